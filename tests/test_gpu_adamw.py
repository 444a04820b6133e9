"""AdamW step against its formula in 64 bits, in units of 2^-24.

The clipped gradient: its factor has three roundings (norm, sum, quotient), the product one: 4.  First moment: the coefficients and products of the
two terms (2 each), the gradient's 4, the sum 1: 8.  Second moment: twice the gradient's 4, coefficient and products 3, the sum 1: 12.  Weights:
8 for the moment, 6 for the root of the other, root and division 2 each, eps and correction 3, rate and its factors 5: 26, 32 are allowed, of
the update; and two roundings of the weight.  8-bit moments: up to one step of e4m3, an eighth of the value or 2^-9 of the scale.  Weights in
bf16: up to one step, 2^-7."""
import math

import pytest
import torch

import ops_reference as ref
from paper_2602_12128_b200 import binding

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
SIZES = [1, 2, 3, 4, 5, 6, 7, 127, 128, 129, 255, 768, 1000, 2047, 2048, 2049, 4097, 16384, 100003]


def tensors(sizes, param, grad, seed=0, state="f32"):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda n: torch.randn(n, generator=g, device="cuda")
    ps = [0.05 * rnd(n) for n in sizes]
    gs = [(1e-3 * rnd(n) * math.exp(i % 3)).to(grad) for i, n in enumerate(sizes)]
    ms, vs = [3e-4 * rnd(n) for n in sizes], [1e-6 * (0.1 + rnd(n).square()) for n in sizes]
    return [p.to(param) for p in ps], gs, ms, vs


def quantise(x):
    n = x.numel()
    rows = torch.nn.functional.pad(x, (0, -n % 128)).view(-1, 128)
    scale = rows.abs().amax(1) / 448
    return (rows / scale.clamp_min(1e-30)[:, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(-1)[:n].clone(), scale


def check(params, new, m, v, gs, lr, t, gain=1.0, wd=0.0, copies=None, q8=None, mul=None):
    """params = (p, m, v) before; new = (p, m, v) after."""
    for i, (p, m0, v0) in enumerate(params):
        g = gs[i].double() * gain
        rate = lr * (mul[i] if mul else 1.0)
        decay = wd[i] if isinstance(wd, list) else wd
        wp, wm, wv = ref.adamw(p.double(), g, m0, v0, rate, t, wd=decay)
        update = (rate / (1 - 0.9 ** t)) * (0.9 * m0.abs() + 0.1 * g.abs()) / (torch.sqrt(wv / (1 - 0.999 ** t)) + 1e-8)
        slack = 2 * U * p.double().abs() + 32 * U * update + 1e-37
        if p.dtype is torch.bfloat16:
            slack = slack + 2.0 ** -7 * wp.abs()
        assert ((new[i].double() - wp).abs() <= slack).all(), i
        if copies is not None:
            assert torch.equal(copies[i], new[i].bfloat16())
        if q8 is None:
            assert ((m[i].double() - wm).abs() <= 8 * U * (0.9 * m0.abs() + 0.1 * g.abs()) + 1e-44).all(), i
            assert ((v[i].double() - wv).abs() <= 12 * U * wv + 1e-44).all(), i
        else:
            for codes, scale, want in ((m[i], q8[0][i], wm), (v[i], q8[1][i], wv)):
                rows = torch.nn.functional.pad(want.abs(), (0, -want.numel() % 128)).view(-1, 128).amax(1)
                torch.testing.assert_close(scale.double(), rows / 448, rtol=1e-6, atol=0)
                off = (ref.decode_q8(codes, scale) - want).abs()
                step = torch.maximum(want.abs() / 8, scale.double().repeat_interleave(128)[:want.numel()] * 2.0 ** -9)
                assert (off <= step * 1.00001).all(), i
            assert (v[i][wv > 0] != 0).all() and (v[i] < 128).all()


@pytest.mark.parametrize("param,grad", [(torch.float32, torch.float32), (torch.float32, torch.bfloat16), (torch.bfloat16, torch.bfloat16), (torch.bfloat16, torch.float32)])
@pytest.mark.parametrize("q8", [False, True])
@pytest.mark.parametrize("max_norm", [0.0, 0.25, 1e6])
def test_step(param, grad, q8, max_norm):
    ps, gs, ms, vs = tensors(SIZES, param, grad)
    copies = [p.bfloat16() for p in ps] if param is torch.float32 else None
    kw = {}
    if q8:
        (ms, msc), (vs, vsc) = (zip(*[quantise(x) for x in xs]) for xs in (ms, vs))
        ms, vs, kw = list(ms), list(vs), dict(m_scales=list(msc), v_scales=list(vsc))
        before = [(p.clone(), ref.decode_q8(m, a), ref.decode_q8(v, b)) for p, m, v, a, b in zip(ps, ms, vs, msc, vsc)]
    else:
        before = [(p.clone(), m.double(), v.double()) for p, m, v in zip(ps, ms, vs)]
    wd = [0.1 * (i % 2) for i in range(len(ps))]
    mul = [1.0 + i % 4 for i in range(len(ps))]
    opt = binding.AdamW(ps, gs, ms, vs, copies=copies, weight_decay=wd, lr_mul=mul, seed=11, **kw)
    opt.step(1e-2, 5, max_norm=max_norm, grad_scale=0.5)
    norm = 0.5 * math.sqrt(sum(g.double().square().sum().item() for g in gs))
    gain = 0.5
    if max_norm:
        assert abs(opt.norm.item() - norm) <= 2 * U * norm
        gain *= min(1.0, max_norm / (norm + 1e-6))
        assert (max_norm < norm) == (max_norm == 0.25)
    check(before, ps, ms, vs, gs, 1e-2, 5, gain, wd, copies, (kw["m_scales"], kw["v_scales"]) if q8 else None, mul)


def test_states_made_here_and_steps_counted():
    for state in ("f32", "q8"):
        ps, gs, _, _ = tensors([300, 6], torch.float32, torch.float32)
        p0 = [p.clone() for p in ps]
        opt = binding.AdamW(ps, gs, state=state, betas=(0.9, 0.999))
        opt.step(1e-3)
        assert opt.steps == 1
        # the first step moves every weight by lr against the sign of its gradient, but for eps: g / (|g| + eps) is eps / |g| off it
        for p, q, g in zip(ps, p0, gs):
            assert ((p - q + 1e-3 * torch.sign(g)).abs() <= 1e-3 * (1e-8 / g.abs() + 32 * U) + 2 * U * q.abs()).all()
        opt.step(1e-3)
        assert opt.steps == 2


@pytest.mark.parametrize("count", [1, 40, 41, 360, 361, 800])
def test_many_tensors(count):
    """Launches know a limited number of tensors; weights with a gradient of zero and no moment stay."""
    sizes = [1 + (37 * i) % 300 for i in range(count)]
    for q8 in (False, True):
        ps, gs, ms, vs = tensors(sizes, torch.float32, torch.float32, seed=count)
        before = [(p.clone(), torch.zeros(n, device="cuda", dtype=torch.float64), torch.zeros(n, device="cuda", dtype=torch.float64)) for p, n in zip(ps, sizes)]
        opt = binding.AdamW(ps, gs, state="q8" if q8 else "f32")
        opt.step(1e-3, 1, max_norm=0.01)
        norm = math.sqrt(sum(g.double().square().sum().item() for g in gs))
        assert abs(opt.norm.item() - norm) <= 2 * U * norm
        check(before, ps, opt.ms, opt.vs, gs, 1e-3, 1, min(1.0, 0.01 / (norm + 1e-6)), q8=(opt.m_scales, opt.v_scales) if q8 else None)


def test_empty_tensors_are_passed_over():
    p, g = torch.randn(300, device="cuda"), torch.randn(300, device="cuda")
    empty = torch.empty(0, device="cuda")
    ps = [empty, p.clone(), empty.clone()]
    opt = binding.AdamW(ps, [empty.clone(), g, empty.clone()], state="q8", seed=3)
    opt.step(1e-3, max_norm=1.0)
    alone = [torch.zeros(1, device="cuda"), p.clone()]      # the random numbers go by the place in the list
    one = binding.AdamW(alone, [torch.zeros(1, device="cuda"), g], state="q8", seed=3)
    one.step(1e-3, max_norm=1.0)
    assert torch.equal(alone[1], ps[1]) and torch.equal(one.ms[1], opt.ms[1]) and torch.equal(one.vs[1], opt.vs[1])
    none = binding.AdamW([empty], [empty.clone()])
    none.norm.fill_(3.0)
    none.step(1e-3, max_norm=1.0)
    assert none.norm.item() == 0.0


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_step_whose_norm_is_not_finite_changes_nothing(bad):
    for state in ("f32", "q8"):
        ps, gs, _, _ = tensors([5000, 6], torch.float32, torch.bfloat16)
        copies = [p.bfloat16() for p in ps]
        opt = binding.AdamW(ps, gs, state=state, copies=copies)
        opt.step(1e-3, max_norm=1.0)
        keep = [t.clone() for t in (*ps, *copies, *opt.ms, *opt.vs)]
        gs[0][4321] = bad
        opt.step(1e-3, max_norm=1.0)
        assert not math.isfinite(opt.norm.item())
        assert all(torch.equal(a, b) for a, b in zip(keep, (*ps, *copies, *opt.ms, *opt.vs)))


def test_without_a_norm_bad_gradients_show():
    g = torch.full((300,), 1e-3, device="cuda")
    g[130] = float("nan")
    p = torch.ones(300, device="cuda")
    opt = binding.AdamW([p], [g], state="q8")
    opt.step(1e-3)
    assert p[130].isnan() and torch.isfinite(p[:130]).all() and torch.isfinite(p[131:]).all()
    m = ref.decode_q8(opt.ms[0], opt.m_scales[0])
    assert opt.m_scales[0].isnan().tolist() == [False, True, False] and opt.v_scales[0].isnan().tolist() == [False, True, False]
    assert torch.isfinite(m[:128]).all() and m[128:256].isnan().all() and torch.isfinite(m[256:]).all()


@pytest.mark.parametrize("size", [1e-25, 1e-12, 1.0, 1e15, 3e19])
def test_gradients_of_any_size(size):
    """Squares of large and small gradients leave the range of fp32; the norm does not."""
    n = 1000
    gs = [size * torch.randn(n, device="cuda")]
    p = [torch.zeros(n, device="cuda")]
    opt = binding.AdamW(p, gs, state="q8", betas=(0.0, 0.999))
    opt.step(1e-3, max_norm=1.0)
    norm = gs[0].double().norm().item()
    assert abs(opt.norm.item() - norm) <= 2 * U * norm
    assert torch.isfinite(p[0]).all()
    assert torch.isfinite(opt.m_scales[0]).all() and torch.isfinite(opt.v_scales[0]).all()


def test_second_moments_below_the_normal_numbers_with_an_eps_that_does_not_cover_them():
    """The first step moves a weight by -lr g / (|g| + eps) whatever the size of g.  Second moments from 1e-39 on are held in multiples of 2^-149;
    two products round to them, half a multiple each, and a root halves the relative error."""
    g = (1 + 9 * torch.rand(1000, device="cuda")) * 1e-18
    g[::2] *= -1
    g[::100] = 0
    p = torch.zeros(1000, device="cuda")
    opt = binding.AdamW([p], [g], eps=2.0 ** -126)
    opt.step(1e-3)
    want = -1e-3 * g.double().sign()
    slack = (32 * U + 2.0 ** -149 / (2 * 1e-3 * g.double().square()).clamp_min(1e-45)) * want.abs()
    assert ((p.double() - want).abs() <= slack).all()


@pytest.mark.parametrize("state", ["f32", "q8"])
def test_a_step_below_one_on_the_device_changes_nothing(state):
    g, p = torch.randn(300, device="cuda"), torch.randn(300, device="cuda")
    before = p.clone()
    opt = binding.AdamW([p], [g], state=state)
    for number in (0, -5):
        opt.step(1e-3, step=torch.tensor(number, device="cuda"), max_norm=1.0)
        assert torch.equal(p, before) and not opt.ms[0].any() and not opt.vs[0].any()
    opt.step(1e-3, step=torch.tensor(1, device="cuda"), max_norm=1.0)
    assert not torch.equal(p, before) and torch.isfinite(p).all()


def test_codes_are_those_of_the_formula():
    """Three steps of 8-bit states on several tensors: every code and scale is what moments formed in single rounded products and sums and the random
    numbers of (seed, step, tensor, element) give, so that another program can follow.  (Below the normal codes a value is first rounded to 2^-20 of
    a step, which the reference does not: one of a million may go the other way.)"""
    sizes, seed = [6, 130, 5000, 128 * 77], 0x123456789AB
    ps, gs, ms, vs = tensors(sizes, torch.bfloat16, torch.bfloat16)
    (ms, msc), (vs, vsc) = (map(list, zip(*[quantise(x) for x in xs])) for xs in (ms, vs))
    opt = binding.AdamW(ps, gs, ms, vs, m_scales=msc, v_scales=vsc, seed=seed)
    f = lambda v: torch.tensor(v, dtype=torch.float32, device="cuda")
    for step in (7, 8, 2**33 + 1):
        held = [(ref.decode_q8(m, a).float(), ref.decode_q8(v, b).float()) for m, v, a, b in zip(ms, vs, msc, vsc)]
        opt.step(1e-3, step)
        for i, n in enumerate(sizes):
            g = gs[i].float()
            m = f(0.9) * held[i][0] + f(1 - 0.9) * g
            v = f(0.999) * held[i][1] + f(1 - 0.999) * g * g
            bits = ref.random_words(n, i, step, seed, "cuda")
            for x, low, codes, scale in ((m, bits & 0xFFFFF, ms[i], msc[i]), (v, bits >> 12, vs[i], vsc[i])):
                want, scales = ref.round_q8(x, low)
                if x is v:
                    want = torch.where(v > 0, want.clamp_min(2.0 ** -9), want)
                assert torch.equal(scale, scales)
                assert (codes.view(torch.float8_e4m3fn).double() != want).sum() <= 1


def test_rounding_keeps_the_mean():
    """Steps of 8-bit moments and bf16 weights are rounded so that their mean is kept: the mean error of n independent roundings,
    each within one step and of variance at most a quarter step squared, is within five standard deviations of zero."""
    n = 1 << 20
    g = torch.full((n,), 1.0, device="cuda")
    g += 0.3 * torch.rand(n, device="cuda")
    p = torch.full((n,), 0.3712, device="cuda").bfloat16()
    p0 = p.double()
    ms, vs = quantise(torch.rand(n, device="cuda") + 0.2), quantise(torch.rand(n, device="cuda") + 0.2)
    m0, v0 = ref.decode_q8(*ms), ref.decode_q8(*vs)
    opt = binding.AdamW([p], [g], [ms[0]], [vs[0]], m_scales=[ms[1]], v_scales=[vs[1]], seed=5)
    opt.step(1e-3, 100)
    wp, wm, wv = ref.adamw(p0, g.double(), m0, v0, 1e-3, 100)
    for got, want, step in ((p.double(), wp, 2.0 ** -8 * 0.25 * 2), (ref.decode_q8(ms[0], ms[1]), wm, None), (ref.decode_q8(vs[0], vs[1]), wv, None)):
        off = got - want
        step = torch.full_like(want, step) if step else 2.0 ** (torch.floor(torch.log2(want)) - 2)
        assert abs((off / step).mean().item()) <= 5 * 0.5 / math.sqrt(n) + 1e-4      # (2^-13 at most from a code at the end of a binade)
    # and a moment moves although its step is far above a change: nearest would never
    v_before = v0.mean()
    for k in range(20):
        opt.step(0.0, 101 + k)
    want = v0.mean() * 0.999 ** 21 + g.double().square().mean() * (1 - 0.999 ** 21)
    assert abs(ref.decode_q8(vs[0], vs[1]).mean() - want) < 0.05 * abs(want - v_before)


def test_a_small_second_moment_never_becomes_zero():
    g = torch.full((128,), 1e-7, device="cuda")
    g[5] = 1.0
    p = torch.zeros(128, device="cuda")
    opt = binding.AdamW([p], [g], state="q8")
    for _ in range(30):
        opt.step(1e-3)
    assert (opt.vs[0] > 0).all() and (p.abs() <= 30 * 1e-3 * 1.01).all()
    none = binding.AdamW([torch.zeros(128, device="cuda")], [torch.zeros(128, device="cuda")], state="q8")
    none.step(1e-3)
    assert (none.ms[0] == 0).all() and (none.vs[0] == 0).all() and (none.m_scales[0] == 0).all() and (none.params[0] == 0).all()


def test_nothing_beside_the_tensors_is_written():
    for state in ("f32", "q8"):
        for n in (1, 5, 127, 130, 2051):
            room = torch.full((n + 64,), 9.0, device="cuda")
            low = torch.full((n + 64,), 9.0, device="cuda", dtype=torch.bfloat16)
            kind = torch.uint8 if state == "q8" else torch.float32
            m, v = (torch.full((n + 64,), 0, device="cuda", dtype=kind) for _ in range(2))
            scales = [torch.full(((n + 127) // 128 + 8,), 0.0, device="cuda") for _ in range(2)]
            k = (n + 127) // 128
            kw = dict(m_scales=[scales[0][:k]], v_scales=[scales[1][:k]]) if state == "q8" else {}
            opt = binding.AdamW([room[:n]], [torch.ones(n, device="cuda")], [m[:n]], [v[:n]], copies=[low[:n]], **kw)
            opt.step(1e-3)
            assert (room[n:] == 9).all() and (low[n:] == 9).all() and (m[n:] == 0).all() and (v[n:] == 0).all() and (m[:n] != 0).all()
            assert all((s[k:] == 0).all() for s in scales)


def test_repeats_streams_other_gradients_and_graphs():
    sizes = [5000, 130, 6, 40000]
    def fresh():
        ps, gs, _, _ = tensors(sizes, torch.bfloat16, torch.bfloat16)
        return ps, gs, binding.AdamW(ps, gs, state="q8", seed=77)
    lr, step = torch.tensor(1e-3, device="cuda"), torch.zeros((), dtype=torch.int64, device="cuda")
    rates = [1e-3, 5e-4, 2e-3]
    ps, gs, opt = fresh()
    for k in range(3):
        opt.step(rates[k], max_norm=0.5)
    want = [t.clone() for t in (*ps, *opt.ms, *opt.vs, opt.norm)]
    side = torch.cuda.Stream()
    ps, gs, opt = fresh()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for k in range(3):
            opt.step(rates[k], max_norm=0.5)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, (*ps, *opt.ms, *opt.vs, opt.norm)))
    # gradients elsewhere
    ps, gs, opt = fresh()
    opt.set_grads([g.clone() for g in gs])
    for g in gs:
        g.zero_()
    for k in range(3):
        opt.step(rates[k], max_norm=0.5)
    assert all(torch.equal(a, b) for a, b in zip(want, (*ps, *opt.ms, *opt.vs, opt.norm)))
    # captured once, replayed with rate and number from the device
    ps, gs, opt = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step.add_(1)
        opt.step(lr, step, max_norm=0.5)
    step.zero_()
    for k in range(3):
        lr.fill_(rates[k])
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want[4:], (*opt.ms, *opt.vs, opt.norm)))
    # (corrections formed on the device in 64 bits and rounded: the weights are the same but for a unit in the last place before their rounding)
    assert all(((a.double() - b.double()).abs() <= 2.0 ** -7 * a.double().abs()).all() and (a != b).double().mean() < 1e-3 for a, b in zip(want, ps))


def test_refusals():
    p = torch.zeros(64, device="cuda")
    with pytest.raises(ValueError):
        binding.AdamW([p], [torch.zeros(63, device="cuda")])
    with pytest.raises(ValueError):
        binding.AdamW([p], [torch.zeros(128, device="cuda")[::2]])
    with pytest.raises(binding.HlaError):
        binding.AdamW([p], [p])
    with pytest.raises(binding.HlaError):
        binding.AdamW([p, p], [torch.zeros(64, device="cuda")] * 2)
    with pytest.raises(binding.HlaError):
        binding.AdamW([torch.zeros(65, device="cuda")[1:]], [torch.zeros(64, device="cuda")])      # not 16-byte aligned
    opt = binding.AdamW([p], [torch.zeros(64, device="cuda")])
    with pytest.raises(ValueError):
        opt.set_grads([torch.zeros(64, device="cuda", dtype=torch.bfloat16)])
    with pytest.raises(ValueError):
        opt.step(1e-3, grad_scale=0.0)
    with pytest.raises(binding.HlaError):
        opt.step(1e-3, step=0)
    with pytest.raises(ValueError):
        opt.step(torch.tensor(1e-3))
