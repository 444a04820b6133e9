"""Scalars of the operators beside the attention that the library would take for something else.  No GPU is needed."""
import pytest
import torch

from paper_2602_12128_b200 import binding as b


def test_heads_without_eps_are_refused():
    """0 stands for 1e-6 in the library; rows of a mean square near 1e-6 would be normalised by another number than the caller's."""
    with pytest.raises(ValueError):
        b.Heads(1, 2, 24, 64, norm=True, eps=0.0, device=None)
    with pytest.raises(ValueError):
        b.Heads(1, 2, 24, 64, norm=True, eps=0, device=None)
    b.Heads(1, 2, 24, 64, norm=False, eps=0.0, device=None)            # not read
    b.Heads(1, 2, 24, 64, norm=True, eps=1e-30, device=None)


def test_places_beyond_32_bits_are_refused():
    """They would come out 2^32 away."""
    make = lambda **kw: b.Heads(1, 2, 24, 64, device=None, **{**dict(axes=(24, 20, 20), grid=(2, 3, 4)), **kw})
    for kw in (dict(start=(1 << 31, 0, 0)), dict(start=(0, -(1 << 31) - 1, 0)), dict(start=((1 << 32) + 5, 0, 0)), dict(grid=((1 << 32) + 2, 3, 4)), dict(axes=((1 << 32) + 24, 20, 20))):
        with pytest.raises(ValueError):
            make(**kw)
    make(start=(-(1 << 31), (1 << 31) - 4, 0))


TINY = 1e-46        # not 0, but 0 as fp32


def test_scalars_that_are_zero_as_fp32_are_refused():
    """0 as fp32 stands for a default (1e-6, 1, 1, 1) or, as max_norm, for no norm at all."""
    for kw in (dict(norm=True, eps=TINY), dict(q_scale=TINY), dict(q_scale=-TINY)):
        with pytest.raises(ValueError):
            b.Heads(1, 2, 24, 64, device=None, **kw)
    step = b.AdamW.step.__get__(_Step())
    for kw in (dict(grad_scale=TINY), dict(max_norm=TINY)):
        with pytest.raises(ValueError):
            step(1e-3, **kw)
    p = [torch.zeros(10)]
    with pytest.raises(ValueError, match="lr_mul"):
        b.AdamW(p, [torch.zeros(10)], lr_mul=TINY, device="cpu")


class _Step:
    """What AdamW.step looks at before it refuses."""
    _norm, steps, _on = 0, 0, -1


@pytest.mark.parametrize("device", ["cpu", pytest.param("cuda", marks=pytest.mark.gpu)])
def test_a_rate_and_a_number_on_the_device_are_one_element(device):
    """A tensor without elements has no address, which stood for the number beside it: a rate of 0, the step 1."""
    step = b.AdamW.step.__get__(_Step())
    for n in (0, 2):
        with pytest.raises(ValueError, match="one element"):
            step(torch.zeros(n, device=device))
        with pytest.raises(ValueError, match="one element"):
            step(1e-3, step=torch.zeros(n, dtype=torch.int64, device=device))


@pytest.mark.gpu
def test_the_norm_is_one_element():
    p, g = [torch.zeros(64, device="cuda")], [torch.ones(64, device="cuda")]
    for n in (0, 2):
        with pytest.raises(ValueError, match="one element"):
            b.AdamW(p, g, norm=torch.zeros(n, device="cuda"))
    for shape in ((), (1,)):
        norm, lr, step = torch.zeros(shape, device="cuda"), torch.full(shape, 1e-3, device="cuda"), torch.ones(shape, dtype=torch.int64, device="cuda")
        opt = b.AdamW(p, g, norm=norm)
        opt.step(lr, step, max_norm=100.0)
        assert norm.item() == 8.0
