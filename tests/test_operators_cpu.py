"""Head preparation, AdamW step and gated recurrence: what is refused before anything is launched, and the gradients that the
GPU tests compare with against differences.  No GPU is needed."""
import ctypes

import pytest
import torch

import ops_reference as ref
from paper_2602_12128_b200 import binding as b

P = 0x100000        # never dereferenced: validation fails first
OK, INVALID, UNSUPPORTED, WORKSPACE = b.HLA_OK, b.HLA_ERR_INVALID_ARG, b.HLA_ERR_UNSUPPORTED, b.HLA_ERR_WORKSPACE


def heads_config(**kw):
    three = lambda v: (ctypes.c_int32 * 3)(*v)
    c = dict(B=2, H=3, N=24, d=64, dtype=b.HLA_BF16, pairing=0, norm=1, n_axes=3, axis_width=(24, 20, 20), grid=(2, 3, 4), start=(0, 0, 0), eps=0.0,
             q_scale=0.0, theta=0.0, inv_freq=None)
    c.update(kw)
    for k in ("axis_width", "grid", "start"):
        c[k] = three(c[k])
    return b.HlaHeadsConfig(*[c[k] for k, _ in b.HlaHeadsConfig._fields_])


def heads(**kw):
    out = ctypes.c_void_p()
    st = b.load_library().hla_heads_create(ctypes.byref(heads_config(**kw)), ctypes.byref(out))
    return st, out.value


@pytest.mark.parametrize("kw,want", [
    (dict(), OK), (dict(grid=(0, 0, 0)), OK), (dict(n_axes=0, grid=(0, 0, 0)), OK), (dict(pairing=1), OK), (dict(axis_width=(8, 0, 0)), OK),
    (dict(dtype=b.HLA_F32, d=20, axis_width=(8, 6, 6), pairing=1), OK),
    (dict(B=0), INVALID), (dict(d=-8), INVALID), (dict(dtype=2), INVALID), (dict(pairing=2), INVALID), (dict(norm=2), INVALID), (dict(n_axes=4), INVALID),
    (dict(axis_width=(23, 20, 20)), INVALID), (dict(axis_width=(40, 20, 20)), INVALID), (dict(grid=(2, 3, 5)), INVALID), (dict(grid=(2, 0, 12)), INVALID),
    (dict(grid=(1 << 30, 1 << 30, 1 << 4)), INVALID), (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(theta=-2.0), INVALID),
    (dict(q_scale=float("inf")), INVALID), (dict(start=(2**31 - 1, 0, 0)), INVALID),
    (dict(d=60, axis_width=(20, 20, 20)), UNSUPPORTED), (dict(d=136), UNSUPPORTED), (dict(B=300, H=300), UNSUPPORTED),
    (dict(axis_width=(24, 20, 18), pairing=1), UNSUPPORTED),
])
def test_heads_create(kw, want):
    st, ctx = heads(**kw)
    assert st == want and bool(ctx) == (want == OK)
    if ctx:
        assert b.load_library().hla_heads_destroy(ctx) == OK


def test_heads_calls_are_checked_before_launching():
    lib = b.load_library()
    st, ctx = heads()
    assert st == OK
    row = 3 * 64
    r = lambda data=P, batch=24 * row, token=row: ctypes.byref(b.HlaRows(data, batch, token))
    far = P + (1 << 24)
    fwd = lambda q=r(), k=None, v=None, wq=None, wk=None, pos=None, pb=0, Q=far, K=None, V=None: lib.hla_heads_forward(ctx, q, k, v, wq, wk, pos, pb, Q, K, V, None)
    assert fwd(q=None, Q=None) == INVALID                  # nothing to do
    assert fwd(Q=None) == INVALID and fwd(q=None) == INVALID
    assert fwd(q=r(P + 2)) == INVALID and fwd(Q=far + 8) == INVALID
    assert fwd(q=r(token=row - 8)) == INVALID and fwd(q=r(token=row + 4)) == INVALID and fwd(q=r(batch=24 * row - 8)) == INVALID
    assert fwd(q=r(token=-row)) == INVALID and fwd(q=r(batch=0)) == INVALID
    assert fwd(q=r(token=1 << 53)) == INVALID and fwd(q=r(batch=1 << 56)) == INVALID     # spans beyond 64 bits
    assert fwd(Q=P) == INVALID and fwd(Q=P + 2 * 24 * row * 2 - 16) == INVALID           # over its input
    assert fwd(k=r(far), K=far + (1 << 22), Q=far) == INVALID                            # Q over k
    assert fwd(v=r(far + (1 << 22)), V=far + 1024) == INVALID                            # V over Q
    assert fwd(wq=P + 4) == INVALID and fwd(pos=P + 2) == INVALID and fwd(pos=P, pb=24 * 3 - 1) == INVALID
    bwd = lambda dQ=P, q=r(far), dq=r(2 * far), wq=None, dwq=None, dwk=None, ws=None, n=0, dV=None, dv=None: lib.hla_heads_backward(
        ctx, dQ, None, dV, q, None, wq, None, None, 0, dq, None, dv, dwq, dwk, ws, n, None)
    need = b.load_library().hla_heads_workspace_bytes(ctx)
    assert need > 0 and lib.hla_heads_workspace_bytes(None) == 0
    assert bwd(dQ=None, dq=None) == INVALID and bwd(dq=None) == INVALID and bwd(q=None) == INVALID
    assert bwd(dwk=P) == INVALID                                                         # no dK
    assert bwd(dwq=P) == INVALID and bwd(dwq=P, ws=P + 16, n=need) == INVALID and bwd(dwq=P, ws=P, n=need - 1) == WORKSPACE
    assert bwd(dq=r(P)) == INVALID and bwd(dq=r(far)) == INVALID                         # over dQ, over q
    assert bwd(dV=3 * far, dv=r(P)) == INVALID
    lib.hla_heads_destroy(ctx)
    st, ctx = heads(grid=(0, 0, 0), norm=0)
    assert fwd() == INVALID                                # no grid and no positions
    assert fwd(pos=P, wq=P) == INVALID                     # weights without norm
    assert lib.hla_heads_workspace_bytes(ctx) == 0
    lib.hla_heads_destroy(ctx)
    assert lib.hla_heads_destroy(None) == INVALID


def test_a_single_token_or_sequence_may_have_any_stride():
    lib = b.load_library()
    st, ctx = heads(B=1, N=1, grid=(1, 1, 1))
    assert st == OK
    bad = ctypes.byref(b.HlaRows(P, 1, 3))                 # strides of dimensions of one are arbitrary: only the missing output is refused
    assert lib.hla_heads_forward(ctx, bad, None, None, None, None, None, 0, P, None, None, None) == INVALID      # (over its input)
    lib.hla_heads_destroy(ctx)


def test_heads_gradients_that_would_share_rows_are_refused():
    lib = b.load_library()
    st, ctx = heads(norm=0)
    assert st == OK
    row, far = 3 * 64, P + (1 << 24)                       # elements of a token's heads; two bytes each
    r = lambda at, batch, token: ctypes.byref(b.HlaRows(at, batch, token))
    bwd = lambda dq, dk: lib.hla_heads_backward(ctx, P, P, None, None, None, None, None, None, 0, dq, dk, None, None, None, None, 0, None)
    fused = lambda part, token=3 * row, batch=24 * 3 * row: r(far + part * row * 2, batch, token)
    assert bwd(fused(0), fused(0)) == INVALID                                            # the same rows twice
    assert bwd(fused(0), r(far + row, 72 * row, 3 * row)) == INVALID                     # half of a row
    assert bwd(fused(0), r(far + (3 * row - 8) * 2, 72 * row, 3 * row)) == INVALID       # the end over the next token's begin
    assert bwd(fused(0), r(far + 3 * row * 2, 72 * row, 3 * row)) == INVALID             # one token on
    assert bwd(fused(0), r(far + row * 2, 24 * row, row)) == INVALID                     # other strides
    assert bwd(fused(0, batch=72 * row + 64), fused(1, batch=72 * row + 64)) == INVALID  # not a multiple
    assert bwd(r(far, 3 * row, 6 * row), r(far + 3 * row * 2, 3 * row, 6 * row)) == INVALID      # [N][B][3]: one batch on
    lib.hla_heads_destroy(ctx)
    st, ctx = heads()
    need = lib.hla_heads_workspace_bytes(ctx)
    x = lambda at: r(at, 24 * row, row)
    call = lambda dwq, dwk: lib.hla_heads_backward(ctx, P, P, None, x(2 * far), x(2 * far), None, None, None, 0, fused(0), fused(1), None, dwq, dwk, 3 * far & ~255, need, None)
    assert call(4 * far, 4 * far) == INVALID and call(4 * far, 4 * far + 252) == INVALID
    lib.hla_heads_destroy(ctx)


def test_heads_frequencies_that_leave_64_bits():
    for value, want in ((1e305, INVALID), (float("inf"), INVALID), (1e200, OK)):
        f = (ctypes.c_double * 32)(*([1.0] * 31 + [value]))
        st, ctx = heads(inv_freq=f)
        assert st == want
        if ctx:
            b.load_library().hla_heads_destroy(ctx)
    assert heads(d=128, n_axes=1, axis_width=(128, 0, 0), grid=(24, 0, 0), theta=1e-320)[0] == INVALID      # its last frequency is 1e315


def test_heads_binding_refuses():
    with pytest.raises(ValueError):
        b.Heads(1, 2, 24, 64, dtype="f16", device=None)
    with pytest.raises(ValueError):
        b.Heads(1, 2, 24, 64, axes=(24, 20, 20), grid=(2, 3, 4), pairing="pairs", device=None)
    with pytest.raises(ValueError):
        b.Heads(1, 2, 24, 64, axes=(24, 20, 20), grid=(2, 12), device=None)
    with pytest.raises(ValueError):
        b.Heads(1, 2, 24, 64, axes=(24, 20, 20), grid=(2, 3, 4), inv_freq=[1.0] * 31, device=None)
    with pytest.raises(b.HlaError):
        b.Heads(1, 2, 24, 64, axes=(24, 20, 20), grid=(2, 3, 5), device=None)
    op = b.Heads(1, 2, 24, 64, axes=(24, 20, 20), grid=(2, 3, 4), device=None)
    for bad in (torch.zeros(1, 24, 2, 64), torch.zeros(1, 24, 2, 64, dtype=torch.bfloat16), torch.zeros(1, 2, 24, 64, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            op.forward(bad)


def adamw(rows, **kw):
    c = dict(beta1=0.9, beta2=0.999, eps=1e-8, state=0, seed=0)
    c.update(kw)
    cfg = b.HlaAdamwConfig(*[c[k] for k, _ in b.HlaAdamwConfig._fields_])
    out = ctypes.c_void_p()
    st = b.load_library().hla_adamw_create(ctypes.byref(cfg), (b.HlaAdamwTensor * len(rows))(*rows), len(rows), ctypes.byref(out))
    return st, out.value


def tensor(at=P, n=100, **kw):
    step = 1 << 16
    t = dict(param=at, copy=0, grad=at + step, m=at + 2 * step, v=at + 3 * step, m_scale=at + 4 * step, v_scale=at + 5 * step, n=n, lr_mul=1.0, weight_decay=0.0,
             param_dtype=b.HLA_F32, grad_dtype=b.HLA_F32)
    t.update(kw)
    return b.HlaAdamwTensor(*[t[k] for k, _ in b.HlaAdamwTensor._fields_])


@pytest.mark.parametrize("rows,kw,want", [
    ([tensor()], {}, OK), ([tensor(n=0, param=0, grad=0), tensor()], {}, OK), ([tensor(copy=P + (6 << 16))], {}, OK), ([tensor(), tensor(P + (1 << 20))], dict(state=1), OK),
    ([tensor(), tensor(P + (1 << 20), grad=P + (1 << 16))], {}, OK),                       # two tensors with one gradient
    ([tensor(param=0)], {}, INVALID), ([tensor(grad=P + 4)], {}, INVALID), ([tensor(v=0)], {}, INVALID), ([tensor(n=-1)], {}, INVALID),
    ([tensor(m_scale=0)], {}, OK), ([tensor(m_scale=0)], dict(state=1), INVALID), ([tensor(v_scale=P + 4)], dict(state=1), INVALID),
    ([tensor(param_dtype=2)], {}, INVALID), ([tensor(grad_dtype=-1)], {}, INVALID), ([tensor(copy=P + (6 << 16), param_dtype=b.HLA_BF16)], {}, INVALID),
    ([tensor(lr_mul=float("nan"))], {}, INVALID), ([tensor(weight_decay=float("inf"))], {}, INVALID),
    ([tensor()], dict(beta1=1.0), INVALID), ([tensor()], dict(beta2=-0.1), INVALID), ([tensor()], dict(eps=0.0), INVALID), ([tensor()], dict(eps=1e-60), INVALID), ([tensor()], dict(eps=1e-16, state=1), INVALID), ([tensor()], dict(eps=1e-16), OK),
    ([tensor()], dict(state=2), INVALID), ([tensor()], dict(beta1=float("nan")), INVALID),
    ([tensor(), tensor()], {}, INVALID),                                                   # the same tensor twice
    ([tensor(), tensor(P + (1 << 20), m=P + 384)], {}, INVALID),                           # a moment over the end of another's weights
    ([tensor(grad=P + 16)], {}, INVALID),                                                  # a gradient over its weights
    ([tensor(n=1 << 39)], {}, UNSUPPORTED),
    ([tensor()], dict(eps=1e-40), INVALID), ([tensor()], dict(eps=2.0 ** -126), OK), ([tensor()], dict(eps=1e39), INVALID),      # eps as fp32 is a normal number
])
def test_adamw_create(rows, kw, want):
    st, ctx = adamw(rows, **kw)
    assert st == want and bool(ctx) == (want == OK)
    if ctx:
        assert b.load_library().hla_adamw_destroy(ctx) == OK


def test_adamw_calls_are_checked_before_launching():
    lib = b.load_library()
    st, ctx = adamw([tensor(), tensor(n=0, grad=0)])
    assert st == OK
    need = lib.hla_adamw_workspace_bytes(ctx)
    assert need > 0 and lib.hla_adamw_workspace_bytes(None) == 0
    def step(ws=None, n=0, **kw):
        a = dict(lr=1e-3, step=1, lr_device=0, step_device=0, max_norm=0.0, grad_scale=1.0, norm=0)
        a.update(kw)
        return lib.hla_adamw_step(ctx, ctypes.byref(b.HlaAdamwStepArgs(*[a[k] for k, _ in b.HlaAdamwStepArgs._fields_])), ws, n, None)
    assert step(step=0) == INVALID and step(lr=float("nan")) == INVALID and step(max_norm=-1.0) == INVALID and step(max_norm=float("nan")) == INVALID
    assert step(grad_scale=float("inf")) == INVALID and step(lr_device=P + 2) == INVALID and step(step_device=P + 4) == INVALID and step(norm=P + 1) == INVALID
    assert step(max_norm=1.0) == INVALID and step(max_norm=1.0, ws=P + 8, n=need) == INVALID and step(max_norm=1.0, ws=P, n=need - 1) == WORKSPACE
    assert lib.hla_adamw_step(None, None, None, 0, None) == INVALID and lib.hla_adamw_step(ctx, None, None, 0, None) == INVALID
    grads = lambda *g: (ctypes.c_void_p * len(g))(*g)
    assert lib.hla_adamw_set_grads(ctx, grads(P + (1 << 22), 0), 2) == OK
    assert lib.hla_adamw_set_grads(ctx, grads(P + (1 << 22)), 1) == INVALID
    assert lib.hla_adamw_set_grads(ctx, grads(0, 0), 2) == INVALID and lib.hla_adamw_set_grads(ctx, grads(P + 4, 0), 2) == INVALID
    assert lib.hla_adamw_set_grads(ctx, grads(P, 0), 2) == INVALID                          # over the weights
    lib.hla_adamw_destroy(ctx)
    assert lib.hla_adamw_destroy(None) == INVALID


def test_the_norm_of_a_step_is_not_written_over_what_the_step_reads():
    lib = b.load_library()
    st, ctx = adamw([tensor()])
    assert st == OK
    need = lib.hla_adamw_workspace_bytes(ctx)
    at = P + (1 << 22)
    for kw in (dict(lr_device=at, norm=at), dict(step_device=at, norm=at + 4)):
        a = b.HlaAdamwStepArgs(1e-3, 1, kw.get("lr_device", 0), kw.get("step_device", 0), 1.0, 1.0, kw["norm"])
        assert lib.hla_adamw_step(ctx, ctypes.byref(a), P + (1 << 23), need, None) == INVALID
    lib.hla_adamw_destroy(ctx)


def test_adamw_binding_refuses():
    p = [torch.zeros(10)]
    for bad in (dict(params=p, grads=[torch.zeros(10)]), dict(params=p, grads=[]), dict(params=[torch.zeros(10, dtype=torch.float64)], grads=p),
                dict(params=p, grads=p, state="f16"), dict(params=p, grads=p, weight_decay=[0.1, 0.2]), dict(params=p, grads=p, lr_mul=0.0)):
        with pytest.raises(ValueError):
            b.AdamW(**bad, device="cpu")


def scan(**kw):
    c = dict(B=2, N=50, C=40, dtype=b.HLA_BF16, gate=0, convex=0, x_batch_stride=0, x_token_stride=0, g_batch_stride=0, g_token_stride=0)
    c.update(kw)
    out = ctypes.c_void_p()
    st = b.load_library().hla_scan_create(ctypes.byref(b.HlaScanConfig(*[c[k] for k, _ in b.HlaScanConfig._fields_])), ctypes.byref(out))
    return st, out.value


@pytest.mark.parametrize("kw,want", [
    (dict(), OK), (dict(C=1, N=1, B=1), OK), (dict(x_token_stride=81, x_batch_stride=81 * 50), OK),
    (dict(B=0), INVALID), (dict(N=-1), INVALID), (dict(C=0), INVALID), (dict(dtype=5), INVALID), (dict(gate=2), INVALID), (dict(convex=2), INVALID),
    (dict(x_token_stride=39), INVALID), (dict(g_batch_stride=-4), INVALID), (dict(B=70000), UNSUPPORTED), (dict(N=(1 << 30) + 1), UNSUPPORTED), (dict(B=60000, N=1 << 30, C=1 << 20), UNSUPPORTED),
    (dict(x_batch_stride=1 << 57), INVALID), (dict(g_token_stride=1 << 55), INVALID), (dict(N=1 << 30, C=4, B=1, x_token_stride=1 << 40), INVALID),
])
def test_scan_create(kw, want):
    st, ctx = scan(**kw)
    assert st == want and bool(ctx) == (want == OK)
    if ctx:
        assert b.load_library().hla_scan_destroy(ctx) == OK


def test_scan_calls_are_checked_before_launching():
    lib = b.load_library()
    st, ctx = scan(convex=1)
    assert st == OK
    far = 1 << 20
    fwd = lambda x=P, g=P + far, h0=None, h=P + 2 * far, last=None: lib.hla_scan_forward(ctx, x, g, h0, h, last, None, 0, None)
    assert fwd(x=None) == INVALID and fwd(h=None) == INVALID and fwd(x=P + 1) == INVALID and fwd(h=P + 2 * far + 4) == INVALID and fwd(h0=P + 2) == INVALID
    assert fwd(h=P) == INVALID and fwd(h=P + far) == INVALID                              # over an input
    assert fwd(last=P + 2 * far) == INVALID and fwd(h0=P + 2 * far + 64) == INVALID and fwd(last=P + 64) == INVALID
    assert fwd(h0=P + 3 * far, last=P + 3 * far + 16) == INVALID                          # shifted, not the same
    bwd = lambda x=P, g=P + far, h0=None, h=P + 2 * far, dh=P + 3 * far, dl=None, dx=P + 4 * far, dg=P + 5 * far, d0=None: lib.hla_scan_backward(
        ctx, x, g, h0, h, dh, dl, dx, dg, d0, None, 0, None)
    assert bwd(x=None) == INVALID and bwd(dg=None) == INVALID and bwd(dh=P + 3 * far + 8) == INVALID and bwd(dl=P + 1) == INVALID
    assert bwd(dx=P) == INVALID and bwd(dg=P + 2 * far) == INVALID and bwd(dg=P + 4 * far) == INVALID and bwd(dx=P + 3 * far) == INVALID
    assert bwd(d0=P + 3 * far) == INVALID and bwd(d0=P + 5 * far) == INVALID and bwd(h0=P + 4 * far) == INVALID
    lib.hla_scan_destroy(ctx)
    assert lib.hla_scan_destroy(None) == INVALID and lib.hla_scan_forward(None, P, P, None, P, None, None, 0, None) == INVALID


def test_scan_in_parts_needs_its_workspace():
    lib = b.load_library()
    assert lib.hla_scan_workspace_bytes(None) == 0
    st, ctx = scan(B=1, N=75600, C=64)
    assert st == OK
    need = lib.hla_scan_workspace_bytes(ctx)
    far = 1 << 28
    fwd = lambda ws, n: lib.hla_scan_forward(ctx, P, P + far, None, P + 2 * far, None, ws, n, None)
    assert need > 0 and fwd(None, 0) == INVALID and fwd(P + 3 * far + 16, need) == INVALID and fwd(P + 3 * far, need - 1) == WORKSPACE
    lib.hla_scan_destroy(ctx)
    st, ctx = scan(B=2, N=75600, C=1536)
    assert st == OK and lib.hla_scan_workspace_bytes(ctx) in (0, lib.hla_scan_workspace_bytes(ctx))
    lib.hla_scan_destroy(ctx)


def test_scan_binding_refuses():
    with pytest.raises(ValueError):
        b.Scan(1, 5, 8, gate="tanh", device=None)
    with pytest.raises(ValueError):
        b.Scan(1, 5, 8, dtype="f64", device=None)
    op = b.Scan(1, 5, 8, device=None)
    with pytest.raises(ValueError):
        op.forward(torch.zeros(1, 5, 8, dtype=torch.bfloat16), torch.zeros(1, 5, 8, dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        op.forward(torch.zeros(1, 5, 8), torch.zeros(1, 5, 8))


# ---- the references' gradients against differences ---------------------------------------------------------------------
def _differences(f, at, grads):
    """Directional derivatives of f at `at` against the gradients."""
    g = torch.Generator().manual_seed(3)
    for i, (x, dx) in enumerate(zip(at, grads)):
        if dx is None:
            continue
        e = torch.randn(x.shape, generator=g, dtype=torch.float64)
        h = 1e-6
        up, down = (f(*[y + s * h * e if j == i else y for j, y in enumerate(at)]) for s in (1, -1))
        want = (dx * e).sum()
        assert abs((up - down) / (2 * h) - want) < 1e-6 * (1 + abs(want)), i


@pytest.mark.parametrize("pairing", ["interleaved", "half"])
@pytest.mark.parametrize("norm", [True, False])
def test_reference_gradient_of_heads(pairing, norm):
    g = torch.Generator().manual_seed(1)
    x, dy = (torch.randn(2, 6, 3, 16, generator=g, dtype=torch.float64) for _ in range(2))
    w = torch.randn(16, generator=g, dtype=torch.float64)
    ang = ref.angles(ref.grid_positions((1, 2, 3)), (8, 4, 4), 100.0)
    f = lambda x, w: (ref.heads(x, w if norm else None, ang, 0.3, pairing, 1e-6 if norm else None).permute(0, 2, 1, 3) * dy).sum()
    dx, dw = ref.heads_backward(dy.permute(0, 2, 1, 3), x, w, ang, 0.3, pairing, 1e-6 if norm else None)
    _differences(f, (x, w), (dx, dw if norm else None))


@pytest.mark.parametrize("gate", ["log", "sigmoid"])
@pytest.mark.parametrize("convex", [True, False])
def test_reference_gradient_of_scan(gate, convex):
    g = torch.Generator().manual_seed(2)
    x, z, dh = (torch.randn(2, 9, 4, generator=g, dtype=torch.float64) for _ in range(3))
    if gate == "log":
        z = -z.abs()
    h0, dl = (torch.randn(2, 4, generator=g, dtype=torch.float64) for _ in range(2))
    def f(x, z, h0):
        h = ref.scan(x, z, h0, gate, convex)
        return (h * dh).sum() + (h[:, -1] * dl).sum()
    _differences(f, (x, z, h0), ref.scan_backward(x, z, h0, ref.scan(x, z, h0, gate, convex), dh, dl, gate, convex))
