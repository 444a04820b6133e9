"""Head preparation against its formulas in 64 bits.

Tolerances count roundings, in units of 2^-24 of the largest quantity that enters.  Forward: the sum of squares (8 additions in a lane, 5
shuffles, mean, eps: 15 units, half of them after the root), rsqrtf (4), two factors (2), cos and sin with their angle (6), scale and the
rotation (4): 24 units of the pair's length, 32 are allowed.  Backward: the same for r and the rotation, the second sum (20 units of the
mean of |g w xh|), four more products: 64 units.  The result is rounded once to its type."""
import math

import pytest
import torch

import ops_reference as ref
from paper_2602_12128_b200 import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def make(B, H, grid, d, dtype, axes, pairing="interleaved", norm=True, fused=False, seed=0, **kw):
    g = torch.Generator(device="cuda").manual_seed(seed)
    N = math.prod(grid)
    dt = DT[dtype]
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").to(dt)
    if fused:
        X = rnd(B, N, 3, H, d)
        xs = [X[:, :, i] for i in range(3)]
    else:
        xs = [rnd(B, N, H, d) for _ in range(3)]
    ws = [(1 + 0.3 * torch.randn(d, generator=g, device="cuda")).to(dt) for _ in range(2)] if norm else [None, None]
    ds = [rnd(B, H, N, d) for _ in range(3)]
    op = binding.Heads(B, H, N, d, dtype=dtype, axes=axes, grid=grid if kw.pop("use_grid", True) else None, pairing=pairing, norm=norm, **kw)
    return op, xs, ws, ds


def pair_length(x, R, pairing):
    """For every channel of x [..., d] the length of its pair."""
    y = x.abs().clone()
    a, b = ((x[..., 0:R:2], x[..., 1:R:2]) if pairing == "interleaved" else (x[..., :R // 2], x[..., R // 2:R]))
    n = torch.hypot(a, b)
    if pairing == "interleaved":
        y[..., 0:R:2] = y[..., 1:R:2] = n
    else:
        y[..., :R // 2] = y[..., R // 2:R] = n
    return y


def check(got, want, size, dtype, units):
    half = ref.HALF_STEP[DT[dtype]]
    err = (got.double() - want).abs()
    bound = half * want.abs() + (1 + half) * units * U * size + 1e-40
    assert torch.isfinite(got).all()
    assert (err <= bound).all(), float((err / bound).max())


def verify(op, xs, ws, ds, ang, pairing, norm, scale, dtype, axes, positions=None, eps=1e-6, dX=None):
    R = sum(axes)
    got = op.forward(*xs, *ws, positions=positions)
    ang = ang.cuda()
    e = eps if norm else None
    dbl = lambda t: None if t is None else t.double()
    for i, s in ((0, scale), (1, 1.0)):
        want = ref.heads(dbl(xs[i]), dbl(ws[i]), ang, s, pairing, e)
        size = pair_length(ref.heads(dbl(xs[i]), dbl(ws[i]), ang * 0, s, pairing, e), R, pairing)
        check(got[i], want, size, dtype, 32)
    assert torch.equal(got[2], xs[2].permute(0, 2, 1, 3))
    out = [torch.full_like(x, float("nan")) for x in xs] if dX is None else dX
    dws = op.backward(*ds, *xs, *out, *ws, positions=positions)
    for i, s in ((0, scale), (1, 1.0)):
        dx, dw = ref.heads_backward(dbl(ds[i]), dbl(xs[i]), dbl(ws[i]), ang, s, pairing, e)
        g = pair_length(ref.heads_backward(dbl(ds[i]), None, None, ang * 0, s, pairing, None)[0], R, pairing)
        if norm:
            x = dbl(xs[i])
            r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
            gw = g * (ws[i].double().abs() if ws[i] is not None else 1.0)
            size = r * (gw + (x * r).abs() * (gw * (x * r).abs()).mean(-1, keepdim=True))
            # a lane's terms follow one another: at most all rows there are
            rows = xs[i].shape[0] * xs[i].shape[1] * xs[i].shape[2]
            total = (g * (x * r).abs()).sum((0, 1, 2))
            assert ((dws[i].double() - dw).abs() <= (64 + min(rows, 512)) * U * total).all()
        else:
            size = g
            assert dws[i] is None
        check(out[i], dx, size, dtype, 64)
    assert torch.equal(out[2], ds[2].permute(0, 2, 1, 3))


CASES = [
    # B, H, grid, d, dtype, axes
    (1, 1, (1, 1, 1), 128, "bf16", (44, 42, 42)),
    (1, 12, (1, 1, 1), 128, "bf16", (44, 42, 42)),
    (2, 3, (3, 5, 7), 128, "bf16", (44, 42, 42)),
    (1, 40, (2, 3, 11), 128, "bf16", (44, 42, 42)),
    (3, 5, (2, 9, 4), 64, "bf16", (24, 20, 20)),
    (1, 2, (4, 8, 8), 16, "f32", (8, 4, 4)),
    (2, 7, (1, 3, 43), 128, "f32", (44, 42, 42)),
    (1, 3, (5, 2, 2), 20, "f32", (8, 6, 6)),
    (2, 2, (33, 1, 1), 36, "f32", (12, 12, 12)),
    (1, 4, (2, 2, 17), 8, "bf16", (4, 2, 2)),
    (1, 9, (3, 2, 10), 48, "bf16", (16, 16, 16)),
    (1, 3, (1, 41, 1), 80, "bf16", (28, 26, 26)),
    (2, 1, (2, 2, 2), 4, "f32", (4, 0, 0)),
]


@pytest.mark.parametrize("pairing", ["interleaved", "half"])
@pytest.mark.parametrize("norm", [True, False])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}x{c[1]}x{math.prod(c[2])}x{c[3]}{c[4]}" for c in CASES])
def test_forward_and_backward(case, norm, pairing):
    B, H, grid, d, dtype, axes = case
    op, xs, ws, ds = make(B, H, grid, d, dtype, axes, pairing, norm, fused=H % 2 == 1, q_scale=0.25, seed=d + H)
    verify(op, xs, ws, ds, ref.angles(ref.grid_positions(grid), axes), pairing, norm, 0.25, dtype, axes)


@pytest.mark.parametrize("axes", [(), (64,), (32, 16), (16, 16, 16), (0, 64, 0)])
def test_axes_that_leave_channels_alone(axes):
    grid = (35,) if len(axes) == 1 else (5, 7) if len(axes) == 2 else (5, 7, 1)
    for pairing in ("interleaved", "half"):
        op, xs, ws, ds = make(2, 3, grid, 128, "bf16", axes, pairing, True, use_grid=bool(axes))
        verify(op, xs, ws, ds, ref.angles(ref.grid_positions(grid), axes), pairing, True, 1.0, "bf16", axes)


def test_far_positions_start_and_frequencies():
    """An angle of 2^31 radians: in 32 bits nothing of it would be left."""
    axes, N = (44, 42, 42), 60
    freq = [0.9 ** j for j in range(64)]
    op, xs, ws, ds = make(1, 2, (3, 4, 5), 128, "f32", axes, start=(2**31 - 10, -(2**31), 12345), inv_freq=freq)
    verify(op, xs, ws, ds, ref.angles(ref.grid_positions((3, 4, 5), (2**31 - 10, -(2**31), 12345)), axes, inv_freq=freq), "interleaved", True, 1.0, "f32", axes)
    g = torch.Generator(device="cuda").manual_seed(5)
    pos = torch.randint(-2**31, 2**31, (2, N, 3), generator=g, device="cuda", dtype=torch.int64).to(torch.int32)
    op, xs, ws, ds = make(2, 3, (3, 4, 5), 128, "bf16", axes, "half", use_grid=False)
    verify(op, xs, ws, ds, ref.angles(pos.cpu(), axes), "half", True, 1.0, "bf16", axes, positions=pos)
    verify(op, xs, ws, ds, ref.angles(pos[:1].cpu(), axes), "half", True, 1.0, "bf16", axes, positions=pos[0])      # shared by the sequences
    with pytest.raises(binding.HlaError):
        op.forward(*xs)                                                     # no grid, no positions


def test_weights_of_ones_and_a_row_of_zeros():
    op, xs, _, ds = make(1, 3, (2, 3, 4), 64, "bf16", (24, 20, 20))
    xs[0][0, 5] = 0
    xs[1][0, 7, 1] = 0
    verify(op, xs, [None, None], ds, ref.angles(ref.grid_positions((2, 3, 4)), (24, 20, 20)), "interleaved", True, 1.0, "bf16", (24, 20, 20))


def test_infinities_and_nan_stay_in_their_row():
    op, xs, ws, ds = make(1, 4, (2, 3, 4), 128, "bf16", (44, 42, 42))
    ok = op.forward(*xs, *ws)
    xs[0][0, 3, 1, 17] = float("inf")
    xs[1][0, 8, 2, 5] = float("nan")
    got = op.forward(*xs, *ws)
    for i, (n, h) in ((0, (3, 1)), (1, (8, 2))):
        same = torch.ones_like(got[i], dtype=torch.bool)
        same[0, h, n] = False
        assert torch.equal(got[i][same], ok[i][same]) and not torch.isfinite(got[i][0, h, n]).all()


def test_gradients_go_into_one_projection_and_nothing_else_is_written():
    B, H, grid, d = 2, 3, (2, 5, 3), 64
    op, xs, ws, ds = make(B, H, grid, d, "bf16", (24, 20, 20), fused=True)
    N = 30
    buf = torch.full((B, N + 4, 3, H + 2, d), 7.0, device="cuda", dtype=torch.bfloat16)
    dX = [buf[:, 2:2 + N, i, :H] for i in range(3)]
    verify(op, xs, ws, ds, ref.angles(ref.grid_positions(grid), (24, 20, 20)), "interleaved", True, 1.0, "bf16", (24, 20, 20), dX=dX)
    keep = torch.ones_like(buf, dtype=torch.bool)
    keep[:, 2:2 + N, :, :H] = False
    assert (buf[keep] == 7).all()


@pytest.mark.parametrize("B,N", [(3, 30), (5, 1)])
def test_tokens_outside_the_batches(B, N):
    """[N][B][3][H][d]: the batches of a token lie behind one another, of inputs and gradients."""
    H, d, grid = 3, 64, (1, 1, N)
    op, xs, ws, ds = make(B, H, grid, d, "bf16", (24, 20, 20))
    outside = lambda: torch.full((N, B + 1, 3, H, d), 7.0, device="cuda", dtype=torch.bfloat16)
    X, dX = outside(), outside()
    parts = lambda t: [t[:, :B, i].transpose(0, 1) for i in range(3)]
    for to, x in zip(parts(X), xs):
        to.copy_(x)
    verify(op, parts(X), ws, ds, ref.angles(ref.grid_positions(grid), (24, 20, 20)), "interleaved", True, 1.0, "bf16", (24, 20, 20), dX=parts(dX))
    assert (dX[:, B:] == 7).all()


def test_each_tensor_alone():
    op, xs, ws, ds = make(2, 6, (2, 5, 3), 128, "bf16", (44, 42, 42))
    Q, K, V = op.forward(*xs, *ws)
    assert torch.equal(op.forward(q=xs[0], wq=ws[0])[0], Q) and torch.equal(op.forward(k=xs[1], wk=ws[1])[1], K) and torch.equal(op.forward(v=xs[2])[2], V)
    out = [torch.empty_like(x) for x in xs]
    dwq, dwk = op.backward(*ds, *xs, *out, *ws)
    for i, (a, b) in enumerate((("q", "dQ"), ("k", "dK"))):
        dx = torch.empty_like(xs[i])
        dw = op.backward(**{b: ds[i], a: xs[i], "d" + a: dx, "w" + a: ws[i]})
        assert torch.equal(dx, out[i]) and dw[1 - i] is None
        torch.testing.assert_close(dw[i], (dwq, dwk)[i], rtol=1e-5, atol=1e-4)
    dv = torch.empty_like(xs[2])
    assert op.backward(dV=ds[2], dv=dv) == (None, None) and torch.equal(dv, out[2])


def test_one_token_with_strides_of_nothing():
    op, xs, ws, ds = make(1, 4, (1, 1, 1), 64, "bf16", (24, 20, 20))
    want = op.forward(*xs, *ws)
    odd = [x.as_strided(x.shape, (1, 3, 64, 1)) for x in xs]
    assert all(torch.equal(a, b) for a, b in zip(op.forward(*odd, *ws), want))


def test_repeats_streams_and_graphs():
    op, xs, ws, ds = make(2, 12, (3, 11, 13), 128, "bf16", (44, 42, 42))
    def call():
        out = [torch.empty_like(x) for x in xs]
        return [*op.forward(*xs, *ws), *op.backward(*ds, *xs, *out, *ws), *out]
    want = call()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    xs[0].neg_()
    ds[0].neg_()
    graph.replay()
    torch.cuda.synchronize()
    new = call()
    assert all(torch.equal(a, b) for a, b in zip(got, new)) and not torch.equal(new[0], want[0])


def test_very_many_heads_of_one_token():
    """More runs of heads than a grid has rows of blocks."""
    H = 60000
    op, xs, ws, ds = make(1, H, (1, 1, 1), 8, "bf16", (4, 2, 2))
    verify(op, xs, ws, ds, ref.angles(ref.grid_positions((1, 1, 1)), (4, 2, 2)), "interleaved", True, 1.0, "bf16", (4, 2, 2))


@pytest.mark.parametrize("H,grid,d,dtype", [(24, (5, 39, 40), 128, "bf16"), (5, (7, 30, 31), 64, "f32")])
def test_longer_sequences(H, grid, d, dtype):
    axes = {128: (44, 42, 42), 64: (24, 20, 20)}[d]
    op, xs, ws, ds = make(1, H, grid, d, dtype, axes, fused=True, q_scale=d ** -0.5)
    verify(op, xs, ws, ds, ref.angles(ref.grid_positions(grid), axes), "interleaved", True, d ** -0.5, dtype, axes)


def test_refusals_of_tensors():
    op, xs, ws, ds = make(2, 3, (2, 3, 4), 64, "bf16", (24, 20, 20))
    with pytest.raises(ValueError):
        op.forward(xs[0].float())
    with pytest.raises(ValueError):
        op.forward(xs[0].transpose(1, 2))
    with pytest.raises(ValueError):
        op.forward(torch.empty(2, 24, 64, 3, device="cuda", dtype=torch.bfloat16).transpose(2, 3))
    with pytest.raises(ValueError):
        op.forward(xs[0], wq=ws[0].float())
    with pytest.raises(ValueError):
        op.forward(xs[0], positions=torch.zeros(24, 2, device="cuda", dtype=torch.int32))
    with pytest.raises(ValueError):
        op.forward(xs[0], positions=torch.zeros(24, 3, device="cuda", dtype=torch.int64))
    with pytest.raises(binding.HlaError):
        op.forward(xs[0][:1].expand(2, -1, -1, -1))            # sequences that share memory are not read: strides must lead on
    with pytest.raises(binding.HlaError):
        op.backward(dQ=ds[0], q=xs[0], dq=xs[0])               # over the input
    with pytest.raises(binding.HlaError):
        op.backward(dQ=ds[0], dq=torch.empty_like(xs[0]))      # the norm needs q
