"""Scalars of the operators beside the attention that the library would take for something else.  No GPU is needed."""
import pytest

from paper_2602_12128_b200 import binding as b


def test_heads_without_eps_are_refused():
    """0 stands for 1e-6 in the library; rows of a mean square near 1e-6 would be normalised by another number than the caller's."""
    with pytest.raises(ValueError):
        b.Heads(1, 2, 24, 64, norm=True, eps=0.0, device=None)
    with pytest.raises(ValueError):
        b.Heads(1, 2, 24, 64, norm=True, eps=0, device=None)
    b.Heads(1, 2, 24, 64, norm=False, eps=0.0, device=None)            # not read
    b.Heads(1, 2, 24, 64, norm=True, eps=1e-30, device=None)
