"""Gated recurrence against token-by-token sums in 64 bits.

The bound follows the recurrence itself: a step adds at most 16 units of 2^-24 of |a h| + |u| (expf 4, 1 / (1 + e) 2, 1 - a 4, the step 2,
and as much again for the products of the composed maps), and carries on a times the error so far; the result is rounded once."""
import pytest
import torch

import ops_reference as ref
from paper_2602_12128_b200 import binding

pytestmark = pytest.mark.gpu
U = 16 * 2.0 ** -24
DT = {"bf16": torch.bfloat16, "f32": torch.float32}
GATES = [("log", False), ("log", True), ("sigmoid", False), ("sigmoid", True)]


def inputs(B, N, C, dtype, gate, seed=0, fused=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    memory = 10 ** (3 * torch.rand(C, generator=g, device="cuda"))
    z = -torch.exp(0.5 * rnd(B, N, C)) / memory if gate == "log" else torch.log(memory) + rnd(B, N, C)
    x = rnd(B, N, C)
    if fused:
        both = torch.empty(B, N, 2, C, device="cuda", dtype=DT[dtype])
        both[:, :, 0], both[:, :, 1] = x, z
        return both[:, :, 0], both[:, :, 1], rnd(B, C), rnd(B, C), rnd(B, N, C).to(DT[dtype])
    return x.to(DT[dtype]), z.to(DT[dtype]), rnd(B, C), rnd(B, C), rnd(B, N, C).to(DT[dtype])


def error_forward(x, z, h0, gate, convex):
    a, rest = ref.gates(z, gate)
    u = (rest * x if convex else x).abs()
    size, err, out = h0.abs(), torch.zeros_like(h0), []
    for t in range(x.shape[1]):
        size = a[:, t] * size + u[:, t]
        err = a[:, t] * err + U * size
        out.append(err)
    return torch.stack(out, 1)


def near(got, want, err, dtype):
    half = ref.HALF_STEP[DT[dtype]]
    off = (got.double() - want).abs() - half * want.abs() - (1 + half) * err
    assert torch.isfinite(got).all() and (off <= 1e-37).all(), float(off.max())


def verify(B, N, C, dtype, gate, convex, carry=True, fused=False, seed=0):
    x, z, h0, dl, dh = inputs(B, N, C, dtype, gate, seed, fused)
    if not carry:
        h0 = dl = None
    op = binding.Scan(B, N, C, dtype=dtype, gate=gate, convex=convex)
    h, last = op.forward(x, z, h0=h0)
    X, Z, D = x.double(), z.double(), dh.double()
    zero = torch.zeros(B, C, device="cuda", dtype=torch.float64)
    H0, DL = (h0.double(), dl.double()) if carry else (zero, zero)
    want = ref.scan(X, Z, H0, gate, convex)
    err = error_forward(X, Z, H0, gate, convex)
    near(h, want, err, dtype)
    near(last, want[:, -1], err[:, -1], "f32")
    dx, dg, dh0 = op.backward(x, z, h, dh, h0=h0, dlast=dl)
    H = h.double()
    wx, wg, w0 = ref.scan_backward(X, Z, H0, H, D, DL, gate, convex)
    a, rest = ref.gates(Z, gate)
    size, e, es, lams = DL.abs(), torch.zeros_like(zero), [], []
    for t in range(N - 1, -1, -1):      # |lambda| and its error, backwards
        lam = D[:, t].abs() + size
        e = e + U * lam
        es.append(e)
        lams.append(lam)
        size, e = a[:, t] * lam, a[:, t] * e + U * a[:, t] * lam
    es, lams = (torch.stack(v[::-1], 1) for v in (es, lams))
    near(dx, wx, (es + U * lams) * (rest if convex else 1.0), dtype)
    before = torch.cat([H0[:, None], H[:, :-1]], 1)
    slope = a if gate == "log" else a * rest
    diff = (before - X).abs() if convex else before.abs()
    near(dg, wg, (es + U * lams) * diff * slope + (U * lams * (before.abs() + X.abs()) * slope if convex else 0.0), dtype)
    if carry:
        near(dh0, w0, e, "f32")
    else:
        assert dh0 is None


@pytest.mark.parametrize("gate,convex", GATES)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N", [1, 2, 7, 8, 9, 127, 128, 129, 255, 257, 1023, 1024, 1025])
def test_lengths(N, dtype, gate, convex):
    verify(2, N, 40, dtype, gate, convex, carry=N % 2 == 1, seed=N)


@pytest.mark.parametrize("C", [1, 2, 3, 31, 32, 33, 63, 64, 65, 257, 1000])
@pytest.mark.parametrize("fused", [False, True])
def test_channels(C, fused):
    verify(3, 150, C, "bf16", "sigmoid", True, fused=fused, seed=C)
    verify(1, 70, C, "f32", "log", False, fused=fused, seed=C)


@pytest.mark.parametrize("B,N,C,dtype,gate,convex", [(1, 5000, 64, "bf16", "log", True), (1, 9001, 8, "f32", "sigmoid", False), (2, 4097, 130, "f32", "log", True),
                                                     (5, 2300, 96, "bf16", "sigmoid", False)])
def test_many_pieces(B, N, C, dtype, gate, convex):
    verify(B, N, C, dtype, gate, convex)


@pytest.mark.parametrize("B,N,C,dtype,gate,convex", [(4, 700, 1540, "bf16", "log", False), (3, 300, 2001, "f32", "sigmoid", True), (2, 2100, 1536, "bf16", "sigmoid", True),
                                                     (20, 140, 1000, "f32", "log", True), (2, 1025, 1601, "bf16", "log", True), (16, 1100, 1024, "bf16", "sigmoid", False)])
def test_many_channels(B, N, C, dtype, gate, convex):
    """More tiles of channels than clusters of eight blocks run at once."""
    verify(B, N, C, dtype, gate, convex, fused=C == 1536, carry=C != 1024)


@pytest.mark.parametrize("B,N,C,dtype,gate,convex", [(1, 20000, 33, "bf16", "log", True), (2, 9000, 64, "bf16", "sigmoid", True), (1, 8200, 1, "f32", "log", False),
                                                     (1, 16385, 257, "bf16", "log", False), (3, 6000, 20, "f32", "sigmoid", True)])
@pytest.mark.parametrize("carry", [False, True])
def test_long_sequences_of_few_channels_run_in_parts(B, N, C, dtype, gate, convex, carry):
    assert binding.Scan(B, N, C, dtype=dtype).workspace is not None
    verify(B, N, C, dtype, gate, convex, carry=carry, fused=C == 257)


def test_the_state_may_stay_in_its_buffer_when_a_sequence_runs_in_parts():
    B, N, C = 1, 30000, 64
    x, z, h0, dl, dh = inputs(B, N, C, "bf16", "sigmoid")
    op = binding.Scan(B, N, C, gate="sigmoid")
    h, last = op.forward(x, z, h0=h0)
    state = h0.clone()
    for _ in range(3):
        state.copy_(h0)
        got, out = op.forward(x, z, h0=state, h_last=state)
        assert out is state and torch.equal(got, h) and torch.equal(state, last)
    first = op.forward(x[:, :1].expand(1, N, C).contiguous(), z, h0=h0)      # (another call on the same workspace)
    assert torch.equal(op.forward(x, z, h0=h0)[0], h) and not torch.equal(first[0], h)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_pieces_continue_a_sequence(dtype):
    """One pass and pieces with the state handed on give the same up to the roundings of both; the state may stay in one buffer."""
    B, N, C = 2, 700, 48
    x, z, h0, _, _ = inputs(B, N, C, dtype, "sigmoid")
    want, last = binding.Scan(B, N, C, dtype=dtype, gate="sigmoid", convex=True).forward(x, z, h0=h0)
    state, parts = h0.clone(), []
    for n in (1, 1, 130, 1, 567):
        at = sum(p.shape[1] for p in parts)
        op = binding.Scan(B, n, C, dtype=dtype, gate="sigmoid", convex=True)
        parts.append(op.forward(x[:, at:at + n], z[:, at:at + n], h0=state, h_last=state)[0])
    err = error_forward(x.double(), z.double(), h0.double(), "sigmoid", True)
    half = ref.HALF_STEP[DT[dtype]]
    assert ((torch.cat(parts, 1).double() - want.double()).abs() <= 2 * (1 + half) * err + 2 * half * want.double().abs()).all()
    assert ((state.double() - last.double()).abs() <= 2 * err[:, -1]).all()


def test_gates_at_their_ends():
    """exp(-inf) and sigmoid(-inf) forget everything, exp(0) and sigmoid(inf) nothing."""
    B, N, C = 1, 300, 32
    x = torch.randn(B, N, C, device="cuda")
    for gate, off, on in (("log", float("-inf"), 0.0), ("sigmoid", float("-inf"), float("inf"))):
        z = torch.full((B, N, C), on, device="cuda")
        z[:, 100] = off
        op = binding.Scan(B, N, C, dtype="f32", gate=gate)
        h, last = op.forward(x, z)
        assert torch.equal(h[:, 100], x[:, 100])
        torch.testing.assert_close(h[:, 101:].double(), torch.cumsum(x[:, 100:].double(), 1)[:, 1:], rtol=1e-5, atol=1e-4)
        dx, dg, _ = op.backward(x, z, h, torch.ones_like(x))
        torch.testing.assert_close(dx[:, :100].double(), torch.arange(100, 0, -1, device="cuda", dtype=torch.float64)[None, :, None].expand(1, 100, C), rtol=1e-6, atol=0)
        assert (dg[:, 100] == 0).all() and torch.isfinite(dg).all()
        conv, _ = binding.Scan(B, N, C, dtype="f32", gate=gate, convex=True).forward(x, z, h0=torch.ones(B, C, device="cuda"))
        assert (conv[:, :100] == 1).all() and torch.equal(conv[:, 100:], x[:, 100:101].expand(1, 200, C))


def test_a_channel_with_nan_or_infinity_leaves_the_others_alone():
    B, N, C = 2, 260, 40
    x, z, h0, dl, dh = inputs(B, N, C, "bf16", "log")
    op = binding.Scan(B, N, C, dtype="bf16")
    want = op.forward(x, z, h0=h0)
    x[0, 30, 7], x[1, 200, 12] = float("nan"), float("inf")
    got = op.forward(x, z, h0=h0)
    for w, g in zip(want, got):
        keep = torch.ones_like(w, dtype=torch.bool)
        keep[0, ..., 7] = keep[1, ..., 12] = False
        assert torch.equal(w[keep], g[keep])
    assert got[0][0, 30:, 7].isnan().all() and torch.equal(got[0][0, :30, 7], want[0][0, :30, 7])
    assert torch.equal(got[0][1, :200, 12], want[0][1, :200, 12]) and not torch.isfinite(got[0][1, 200:, 12]).any()


def test_nothing_behind_the_outputs_is_written():
    B, N, C = 1, 131, 33
    x, z, h0, dl, dh = inputs(B, N, C, "bf16", "log")
    op = binding.Scan(B, N, C, dtype="bf16")
    room = [torch.full((B * N * C + 64,), 5.0, device="cuda", dtype=torch.bfloat16) for _ in range(3)]
    h, dx, dg = (r[:B * N * C].view(B, N, C) for r in room)
    op.forward(x, z, h0=h0, h=h)
    op.backward(x, z, h, dh, h0=h0, dlast=dl, dx=dx, dg=dg)
    assert all((r[B * N * C:] == 5).all() for r in room)


def test_repeats_streams_and_graphs():
    B, N, C = 2, 1500, 200
    x, z, h0, dl, dh = inputs(B, N, C, "bf16", "sigmoid")
    op = binding.Scan(B, N, C, dtype="bf16", gate="sigmoid", convex=True)
    def call():
        h, last = op.forward(x, z, h0=h0)
        return [h, last, *op.backward(x, z, h, dh, h0=h0, dlast=dl)]
    want = call()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = call()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    x.neg_()
    graph.replay()
    torch.cuda.synchronize()
    new = call()
    assert all(torch.equal(a, b) for a, b in zip(got, new)) and not torch.equal(new[0], want[0])


def test_two_calls_at_once():
    """Contexts on streams of their own share nothing."""
    sets = [inputs(1, 2000, 256, "bf16", "log", seed=s) for s in range(2)]
    ops = [binding.Scan(1, 2000, 256, dtype="bf16") for _ in range(2)]
    want = [op.forward(*s[:2], h0=s[2]) for op, s in zip(ops, sets)]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for op, s, st in zip(ops, sets, streams):
        with torch.cuda.stream(st):
            got.append([op.forward(*s[:2], h0=s[2]) for _ in range(5)][-1])
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for w, g in zip(want, got) for a, b in zip(w, g))


def test_strides_are_followed_and_bad_ones_refused():
    op = binding.Scan(2, 20, 16, dtype="f32")
    a, b = inputs(2, 20, 16, "f32", "log"), inputs(2, 20, 16, "f32", "log", fused=True)
    assert torch.equal(op.forward(*a[:2])[0], op.forward(*b[:2])[0]) and torch.equal(op.forward(*a[:2])[0], op.forward(b[0], a[1])[0])
    with pytest.raises(ValueError):
        op.forward(a[0][:, :1].expand(2, 20, 16), a[1])
    with pytest.raises(ValueError):
        op.forward(a[0][:1].expand(2, 20, 16), a[1])
    with pytest.raises(ValueError):
        op.forward(torch.empty(2, 16, 20, device="cuda").transpose(1, 2), a[1])
    with pytest.raises(ValueError):
        op.forward(*a[:2], h0=a[2].bfloat16())
    with pytest.raises(binding.HlaError):
        op.forward(*a[:2], h=a[0])
