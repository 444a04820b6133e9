"""Tensors with more than 2^31 elements: parts of the results at both ends and around the places where 32-bit offsets would wrap."""
import pytest
import torch

import ops_reference as ref
from paper_2602_12128_b200 import binding

pytestmark = pytest.mark.gpu
BF = torch.bfloat16


@pytest.fixture(autouse=True)
def room():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of device memory")
    yield
    torch.cuda.empty_cache()


def test_heads():
    B, H, N, d, axes = 1, 40, 430_000, 128, (44, 42, 42)
    assert B * H * N * d > 1 << 31
    g = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(B, N, H, d, generator=g, device="cuda", dtype=BF)
    w = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(BF)
    op = binding.Heads(B, H, N, d, axes=axes, grid=(430, 25, 40), norm=True)
    Q = op.forward(q=x, wq=w)[0]
    places = torch.tensor([0, 1, 209_713, 209_715, 209_716, 419_430, 419_431, N - 1], device="cuda")
    ang = ref.angles(ref.grid_positions((430, 25, 40))[places.cpu()], axes).cuda()
    want = ref.heads(x[:, places].double(), w.double(), ang, 1.0, "interleaved", 1e-6)
    assert ((Q[:, :, places].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all()
    dx = torch.empty_like(x)
    op.backward(dQ=Q, q=x, dq=dx, wq=w)
    want, _ = ref.heads_backward(Q[:, :, places].double(), x[:, places].double(), w.double(), ang, 1.0, "interleaved", 1e-6)
    assert ((dx[:, places].double() - want).abs() <= 2.0 ** -8 * want.abs() + 1e-4).all()


def test_scan():
    B, N, C = 2, 70_000, 16_000
    assert B * N * C > 1 << 31
    x = torch.randn(B, N, C, device="cuda", dtype=BF)
    z = torch.randn(B, N, C, device="cuda", dtype=BF)
    op = binding.Scan(B, N, C, gate="sigmoid")
    h, last = op.forward(x, z)
    some = torch.tensor([0, 1, 7999, C - 2, C - 1], device="cuda")
    for b in range(B):      # the last tokens of some channels, from a state that the tokens before have made
        t0 = N - 60
        want = ref.scan(x[b:b + 1, t0:, some].double(), z[b:b + 1, t0:, some].double(), h[b:b + 1, t0 - 1, some].double(), "sigmoid", False)
        assert ((h[b:b + 1, t0:, some].double() - want).abs() <= 2.0 ** -7 * (want.abs() + 8)).all()
        assert ((last[b, some].double() - want[0, -1]).abs() <= 2.0 ** -7 * (want[0, -1].abs() + 8)).all()
    dx, dg, _ = op.backward(x, z, h, x)
    for b in range(B):      # the last tokens are where the backward starts
        t0 = N - 60
        wx, wg, _ = ref.scan_backward(x[b:b + 1, t0:, some].double(), z[b:b + 1, t0:, some].double(), h[b:b + 1, t0 - 1, some].double(),
                                      h[b:b + 1, t0:, some].double(), x[b:b + 1, t0:, some].double(), None, "sigmoid", False)
        assert ((dx[b:b + 1, t0:, some].double() - wx).abs() <= 2.0 ** -8 * wx.abs() + 1e-5).all()
        assert ((dg[b:b + 1, t0:, some].double() - wg).abs() <= 2.0 ** -8 * wg.abs() + 1e-4).all()
    assert torch.isfinite(dx[0, :100]).all() and torch.isfinite(dg[1, :100]).all()


def test_adamw():
    n = (1 << 31) + 1000
    g = torch.Generator(device="cuda").manual_seed(0)
    p, grad = (torch.randn(n, generator=g, device="cuda", dtype=BF) for _ in range(2))
    keep = torch.cat([p[:2000], p[(1 << 31) - 1000:]])
    opt = binding.AdamW([p], [grad], state="q8", seed=9)
    opt.step(1e-3, max_norm=float("inf"))
    some = torch.cat([grad[:2000], grad[(1 << 31) - 1000:]]).double()
    want = keep.double() - 1e-3 * some / (some.abs() + 1e-8)
    got = torch.cat([p[:2000], p[(1 << 31) - 1000:]]).double()
    assert ((got - want).abs() <= 2.0 ** -7 * want.abs() + 1e-8).all()
    for codes, scales, moment in ((opt.ms[0], opt.m_scales[0], 0.1 * grad[-1000:].double()), (opt.vs[0], opt.v_scales[0], 1e-3 * grad[-1000:].double().square())):
        tail = (1000 + 127) // 128                     # (2^31 is a multiple of 128: the last groups begin there)
        off = (ref.decode_q8(codes[-1000:], scales[-tail:]) - moment).abs()
        assert (off <= moment.abs() / 8 + scales[-tail:].double().repeat_interleave(128)[:1000] * 2.0 ** -9 * 1.001).all()
    parts = [grad[i:i + (1 << 28)].float().norm().double().square() for i in range(0, n, 1 << 28)]
    assert abs(opt.norm.item() - torch.stack(parts).sum().sqrt().item()) <= 1e-4 * opt.norm.item()
