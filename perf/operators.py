"""What the operators around the attention are measured on: the head preparation (norm, rotary positions in several axes,
head-major layout) with its backward, the AdamW step over many tensors, and the gated linear recurrence with its backward.

A case is a plain dict; `op` says which operator one pass runs:

    heads_forward    q, k, v of a projection [B,N,H,d] -> RMS norm per head (q, k), rotation by (time, height, width), scale of q
                     -> Q, K, V [B,H,N,d]
    heads_backward   dQ, dK, dV [B,H,N,d] -> gradients of q, k, v and of the two norm weights
    adamw            one step over all tensors: global gradient norm and clipping (max_norm > 0), both moments, the weights
    scan_forward     h_t = a_t h_{t-1} + u_t over N tokens, a = exp(g) or sigmoid(g), u = x or (1 - a) x
    scan_backward    gradients of x, g and the carried-in state

`own` chooses between the plain form (elementary torch operations) and the calls of the framework."""
from __future__ import annotations

import math
import random

import numpy as np
import torch

own = False
DEVICE = "cuda"
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
THETA, EPS_NORM = 10000.0, 1e-6
BETA1, BETA2, EPS_ADAM, DECAY, LR, FIRST_STEP, SEED = 0.9, 0.999, 1e-8, 0.01, 1e-4, 1000, 1234
BLOCK = 128          # elements that share a scale of the 8-bit states
E4M3_MAX = 448.0
ROUND = 512          # tensors of an arena start at multiples of this many elements


# ---- cases -------------------------------------------------------------------------------------------------------------
def _heads(name, op, B, H, t, h, w, d, dtype="bf16", pairing="interleaved", norm=True, fused=True, positions="grid"):
    return _named(name, {"op": op, "B": B, "H": H, "t": t, "h": h, "w": w, "d": d, "dtype": dtype, "pairing": pairing, "norm": norm,
                         "fused": fused, "positions": positions})


def _adamw(name, kind, layers, width, state, param, grad, max_norm=0.0, sizes=0):
    return _named(name, {"op": "adamw", "kind": kind, "layers": layers, "width": width, "state": state, "param": param, "grad": grad,
                         "max_norm": max_norm, "sizes": sizes})


def _scan(name, op, B, N, C, dtype="bf16", gate="log", convex=False, carry=False, fused=False):
    return _named(name, {"op": op, "B": B, "N": N, "C": C, "dtype": dtype, "gate": gate, "convex": convex, "carry": carry, "fused": fused})


def _named(name, c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # one token of a stream at 12 heads, its position given: what latency is made of
        _heads("heads_token", "heads_forward", 1, 12, 1, 1, 1, 128, positions="given"),
        # the small fp32 configuration of the parity checks, 256 tokens of width 16, the half-split pairing, no norm
        _heads("heads_small_f32", "heads_forward", 1, 2, 4, 8, 8, 16, dtype="f32", pairing="half", norm=False, fused=False),
        # the q, k, v of one attention call of a video DiT, 21x39x40 latent grid
        _heads("heads_dit", "heads_forward", 1, 24, 21, 39, 40, 128),
        # fp32 validation training at a ragged length
        _heads("heads_f32_backward", "heads_backward", 1, 12, 3, 25, 40, 64, dtype="f32", pairing="half", fused=False),
        # backward of the headline training step
        _heads("heads_train_backward", "heads_backward", 2, 24, 21, 39, 40, 128),
        # the four feature networks of one layer: 16 tensors from 6 to 16384 weights, fp32 gradients, bf16 copies for the kernels
        _adamw("adamw_maps", "maps", 1, 128, "f32", "f32", "f32"),
        # eight transformer blocks with their feature networks, clipped, states in fp32
        _adamw("adamw_blocks_f32", "blocks", 8, 1536, "f32", "f32", "bf16", max_norm=1.0),
        # the same blocks trained in little memory: bf16 weights and 8-bit states
        _adamw("adamw_blocks_q8", "blocks", 8, 1536, "q8", "bf16", "bf16", max_norm=1.0),
        # a piece of 500 tokens of a causal stream, the state carried
        _scan("scan_chunk", "scan_forward", 1, 500, 1536, carry=True),
        # a whole video sequence, gate logits and inputs from one projection, convex update
        _scan("scan_video", "scan_forward", 1, 32760, 1536, gate="sigmoid", convex=True, fused=True),
        # fp32 validation training at a ragged length
        _scan("scan_f32_backward", "scan_backward", 1, 3000, 768, dtype="f32", gate="sigmoid", convex=True, carry=True),
        # training step of two video sequences
        _scan("scan_train_backward", "scan_backward", 2, 32760, 1536),
    ]


def _log_between(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["heads", "heads", "adamw", "scan", "scan"])
    dtype = rng.choice(["bf16", "bf16", "f32"])
    if kind == "heads":
        d = rng.choice([64, 128, 128, 16, 32, 48, 80, 96]) if dtype == "bf16" else rng.choice([16, 20, 36, 64, 128])
        B, H = rng.choice([1, 1, 2, 3]), rng.randint(1, 40)
        most = 160_000_000 // (B * H * d) // (1 if dtype == "bf16" else 2)
        t, h, w = rng.randint(1, 21), _log_between(rng, 1, 60), _log_between(rng, 1, 60)
        while t * h * w > most:
            t, h, w = max(1, t // 2), h, max(1, w - 1)
        return _heads(None, rng.choice(["heads_forward", "heads_backward"]), B, H, t, h, w, d, dtype, rng.choice(["interleaved", "half"]),
                      rng.random() < 0.7, rng.random() < 0.6, rng.choice(["grid", "grid", "given"]))
    if kind == "adamw":
        state = rng.choice(["f32", "q8"])
        return _adamw(None, "ragged", rng.randint(1, 300), _log_between(rng, 8, 300_000), state, rng.choice(["f32", "bf16"]),
                      rng.choice(["f32", "bf16"]), rng.choice([0.0, 1.0, 10.0]), rng.randrange(1 << 20))
    B, C, N = rng.choice([1, 1, 2, 4]), rng.choice([64, 257, 768, 1000, 1536, 1536, 2048]), _log_between(rng, 1, 75600)
    N = max(1, min(N, 90_000_000 // (B * C) // (1 if dtype == "bf16" else 2)))
    return _scan(None, rng.choice(["scan_forward", "scan_backward"]), B, N, C, dtype, rng.choice(["log", "sigmoid"]), rng.random() < 0.5,
                 rng.random() < 0.5, rng.random() < 0.5)


def _axes(d):
    """Channels of a head that turn with time, height and width: two sixths each for height and width, the rest for time."""
    side = 2 * (d // 6)
    return d - 2 * side, side, side


def _sizes(case):
    """How many weights each tensor of an AdamW case has."""
    c, w = case, case["width"]
    maps = [128 * 128, 128, 128 * 6, 6] * 4
    if c["kind"] == "maps":
        return maps * c["layers"]
    if c["kind"] == "blocks":
        return (maps + [w * w, w] * 4 + [4 * w * w, 4 * w, 4 * w * w, w]) * c["layers"]
    r = random.Random(c["sizes"])
    return [_log_between(r, 1, 4 * w) for _ in range(c["layers"])]


# ---- inputs ------------------------------------------------------------------------------------------------------------
class _Draw:
    def __init__(self, seed):
        self.g = torch.Generator(device=DEVICE)
        self.g.manual_seed(seed)

    def normal(self, *dims):
        return torch.randn(dims, generator=self.g, device=DEVICE, dtype=torch.float32)

    def uniform(self, *dims):
        return torch.rand(dims, generator=self.g, device=DEVICE, dtype=torch.float32)

    def tokens(self, dtype, *dims):
        return torch.randn(dims, generator=self.g, device=DEVICE, dtype=dtype)


def prepare(case, seed):
    r = _Draw(seed)
    return {"heads": _prepare_heads, "adamw": _prepare_adamw, "scan": _prepare_scan}[case["op"].split("_")[0]](case, r)


def _prepare_heads(c, r):
    B, H, N, d, dt = c["B"], c["H"], c["t"] * c["h"] * c["w"], c["d"], TYPES[c["dtype"]]
    if c["fused"]:                                   # one projection for q, k, v
        X = r.tokens(dt, B, N, 3, H, d)
        xs = [X[:, :, i] for i in range(3)]
    else:
        X = None
        xs = [r.tokens(dt, B, N, H, d) for _ in range(3)]
    s = {"case": c, "X": X, "xs": xs, "w": [None, None], "positions": None}
    if c["norm"]:
        s["w"] = [(1.0 + 0.2 * r.normal(d)).to(dt) for _ in range(2)]
    if c["positions"] == "given":                    # clips cut from long videos: every sequence starts at a time of its own
        first = (r.uniform(B, 1, 1) * 20000).to(torch.int32)
        n = torch.arange(N, device=DEVICE, dtype=torch.int32)
        grid = torch.stack([n // (c["h"] * c["w"]), n // c["w"] % c["h"], n % c["w"]], -1).expand(B, N, 3).clone()
        grid[..., :1] += first
        s["positions"] = grid
    if c["op"] == "heads_backward":
        s["d"] = [r.tokens(dt, B, H, N, d) for _ in range(3)]
    if own:
        from paper_2602_12128_b200 import binding
        s["plan"] = binding.Heads(B, H, N, d, dtype=c["dtype"], axes=_axes(d), grid=(c["t"], c["h"], c["w"]), theta=THETA, pairing=c["pairing"],
                                  norm=c["norm"], eps=EPS_NORM, q_scale=1.0 / math.sqrt(d), device=DEVICE)
    return s


def _prepare_adamw(c, r):
    sizes = _sizes(c)
    starts, total = [], 0
    for n in sizes:
        starts.append(total)
        total += -(-n // ROUND) * ROUND
    real = torch.zeros(total, dtype=torch.bool, device=DEVICE)          # padding between the tensors stays zero
    for o, n in zip(starts, sizes):
        real[o:o + n] = True
    # gradients of a trained network: rows whose size differs, most values small
    size = torch.exp(0.7 * r.normal(total // ROUND, 1)).expand(-1, ROUND).reshape(-1) * (3e-3 / math.sqrt(sum(sizes) / 1e5 + 1))
    p = (0.02 * r.normal(total)) * real
    g = size * r.normal(total) * real
    m = 0.3 * size * r.normal(total) * real
    v = torch.square(size * (0.5 + r.uniform(total))) * real
    s = {"case": c, "sizes": sizes, "starts": starts, "t": FIRST_STEP, "p": p.to(TYPES[c["param"]]), "g": g.to(TYPES[c["grad"]]), "copy": None}
    if c["param"] == "f32":
        s["copy"] = p.to(torch.bfloat16)
    if c["state"] == "q8":
        (s["m"], s["ms"]), (s["v"], s["vs"]) = _nearest_q8(m), _nearest_q8(v)
    else:
        s["m"], s["v"] = m, v
    # the optimiser's view: every tensor by itself
    s["parts"] = {k: [s[k][o:o + n] for o, n in zip(starts, sizes)] if s.get(k) is not None else None for k in ("p", "g", "m", "v", "copy")}
    for k in ("ms", "vs"):
        s["parts"][k] = [s[k][o // BLOCK:o // BLOCK + -(-n // BLOCK)] for o, n in zip(starts, sizes)] if k in s else None
    s["norm"] = torch.zeros((), dtype=torch.float32, device=DEVICE)
    if own:
        from paper_2602_12128_b200 import binding
        q = s["parts"]
        s["plan"] = binding.AdamW(q["p"], q["g"], q["m"], q["v"], m_scales=q["ms"], v_scales=q["vs"], copies=q["copy"], betas=(BETA1, BETA2),
                                  eps=EPS_ADAM, weight_decay=DECAY, seed=SEED, norm=s["norm"], device=DEVICE)
    return s


def _nearest_q8(x):
    """x [total] -> (codes, scales): a state as earlier steps left it."""
    rows = x.view(-1, BLOCK)
    scale = rows.abs().amax(1) / E4M3_MAX
    return (rows / scale.clamp_min(1e-30)[:, None]).to(torch.float8_e4m3fn).view(torch.uint8).view(-1), scale


def _prepare_scan(c, r):
    B, N, C, dt = c["B"], c["N"], c["C"], TYPES[c["dtype"]]
    # each channel has a memory of its own, from two to two thousand tokens; the gates of its tokens scatter around it
    memory = torch.exp(r.uniform(C) * math.log(1000.0) + math.log(2.0))
    pair = torch.empty(B, N, 2, C, dtype=dt, device=DEVICE) if c["fused"] else None
    x, g = (pair[:, :, 0], pair[:, :, 1]) if c["fused"] else (torch.empty(B, N, C, dtype=dt, device=DEVICE) for _ in range(2))
    x.copy_(r.tokens(dt, B, N, C))
    noise = 0.5 * r.normal(B, N, C)
    g.copy_(-torch.exp(noise) / memory if c["gate"] == "log" else torch.log(memory) + noise)
    s = {"case": c, "x": x, "g": g, "h0": r.normal(B, C) if c["carry"] else None}
    if c["op"] == "scan_backward":
        s["h"] = _plain_scan_forward(s)["h"]
        s["dh"] = r.tokens(dt, B, N, C)
        s["dlast"] = r.normal(B, C) if c["carry"] else None
    if own:
        from paper_2602_12128_b200 import binding
        s["plan"] = binding.Scan(B, N, C, dtype=c["dtype"], gate=c["gate"], convex=c["convex"], device=DEVICE)
    return s


# ---- one pass ----------------------------------------------------------------------------------------------------------
def run(state):
    op = state["case"]["op"]
    if op == "adamw":
        return _run_adamw(state)
    if own:
        return {"heads_forward": _own_heads_forward, "heads_backward": _own_heads_backward, "scan_forward": _own_scan_forward,
                "scan_backward": _own_scan_backward}[op](state)
    return {"heads_forward": _plain_heads_forward, "heads_backward": _plain_heads_backward, "scan_forward": _plain_scan_forward,
            "scan_backward": _plain_scan_backward}[op](state)


def _own_heads_forward(s):
    Q, K, V = s["plan"].forward(*s["xs"], *s["w"], positions=s["positions"])
    return {"Q": Q, "K": K, "V": V}


def _own_heads_backward(s):
    if s["X"] is not None:                           # the gradients go where the projection's backward reads them: one tensor
        dX = torch.empty_like(s["X"])
        out = [dX[:, :, i] for i in range(3)]
    else:
        dX, out = None, [torch.empty_like(x) for x in s["xs"]]
    dwq, dwk = s["plan"].backward(*s["d"], *s["xs"], *out, *s["w"], positions=s["positions"])
    return {"dX": dX if dX is not None else out, "dw": [dwq, dwk]}


def _own_scan_forward(s):
    h, last = s["plan"].forward(s["x"], s["g"], h0=s["h0"])
    return {"h": h, "last": last}


def _own_scan_backward(s):
    dx, dg, dh0 = s["plan"].backward(s["x"], s["g"], s["h"], s["dh"], h0=s["h0"], dlast=s["dlast"])
    return {"dx": dx, "dg": dg, "dh0": dh0}


# The head preparation, plainly.
def _cos_sin(s):
    """cos and sin [B or 1, N, 1, d/2] of every token's angles; angles of far positions need 64 bits."""
    c = s["case"]
    if s["positions"] is not None:
        pos = s["positions"].double()
    else:
        n = torch.arange(c["t"] * c["h"] * c["w"], device=DEVICE)
        pos = torch.stack([n // (c["h"] * c["w"]), n // c["w"] % c["h"], n % c["w"]], -1).double()[None]
    turn = []
    for a, width in enumerate(_axes(c["d"])):
        inv = torch.pow(torch.tensor(THETA, dtype=torch.float64, device=DEVICE), -torch.arange(0, width, 2, device=DEVICE, dtype=torch.float64) / max(width, 1))
        turn.append(pos[..., a:a + 1] * inv)
    angle = torch.cat(turn, -1)[:, :, None]
    return torch.cos(angle).float(), torch.sin(angle).float()


def _rotate(x, cos, sin, pairing):
    if pairing == "interleaved":
        a, b = x[..., 0::2], x[..., 1::2]
        return torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    a, b = x.chunk(2, -1)
    return torch.cat([a * cos - b * sin, a * sin + b * cos], -1)


def _plain_heads_forward(s):
    c = s["case"]
    cos, sin = _cos_sin(s)
    out = {}
    for name, x, w, scale in (("Q", s["xs"][0], s["w"][0], 1.0 / math.sqrt(c["d"])), ("K", s["xs"][1], s["w"][1], 1.0)):
        y = x.float()
        if c["norm"]:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS_NORM) * w.float()
        y = _rotate(y, cos, sin, c["pairing"]) * scale
        out[name] = y.to(x.dtype).transpose(1, 2).contiguous()
    out["V"] = s["xs"][2].transpose(1, 2).contiguous()
    return out


def _plain_heads_backward(s):
    c = s["case"]
    cos, sin = _cos_sin(s)
    dxs, dws = [], []
    for dy, x, w, scale in ((s["d"][0], s["xs"][0], s["w"][0], 1.0 / math.sqrt(c["d"])), (s["d"][1], s["xs"][1], s["w"][1], 1.0)):
        g = _rotate(dy.transpose(1, 2).float() * scale, cos, -sin, c["pairing"])
        if c["norm"]:
            x32 = x.float()
            r = torch.rsqrt(x32.square().mean(-1, keepdim=True) + EPS_NORM)
            xh = x32 * r
            dws.append((g * xh).sum((0, 1, 2), dtype=torch.float64).float())
            g = g * w.float()
            g = r * (g - xh * (g * xh).mean(-1, keepdim=True))
        dxs.append(g.to(x.dtype))
    dxs.append(s["d"][2].transpose(1, 2))
    return {"dX": torch.stack(dxs, 2) if s["X"] is not None else [d.contiguous() for d in dxs], "dw": dws if dws else [None, None]}


# The AdamW step, plainly.
def _run_adamw(s):
    c = s["case"]
    s["t"] += 1
    if own:
        s["plan"].step(LR, s["t"], max_norm=c["max_norm"])
    else:
        _plain_adamw(s)
    out = {"p": s["p"], "copy": s["copy"], "norm": s["norm"] if c["max_norm"] > 0 else None}
    if c["state"] == "q8":
        out.update(m=s["m"].view(torch.float8_e4m3fn), m_scale=s["ms"], v=s["v"].view(torch.float8_e4m3fn), v_scale=s["vs"])
    else:
        out.update(m=s["m"], v=s["v"])
    return out


def _mix32(x):
    """A 32-bit mixing function (xor-shift and multiply, twice) on values below 2^32."""
    x = x ^ (x >> 16)
    x = x * 0x7FEB352D & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = x * 0x846CA68B & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random32(n, tensor, step):
    """The random 32 bits of each element of a tensor in a step: two neighbours share the first rounds of the mixing."""
    k = _mix32(SEED & 0xFFFFFFFF)
    k = _mix32(k ^ (SEED >> 32))
    k = _mix32(k ^ (step & 0xFFFFFFFF))
    k = _mix32((k + tensor) & 0xFFFFFFFF)
    i = torch.arange(0, n, 2, device=DEVICE, dtype=torch.int64)
    x = _mix32((k + (i // BLOCK) * 0x9E3779B9) & 0xFFFFFFFF) + (i % BLOCK // 2) * 0x9E3779B9 & 0xFFFFFFFF
    x = x ^ (x >> 16)
    x = x * 0x7FEB352D & 0xFFFFFFFF
    x = (x ^ (x >> 15)) * 0x846CA68B & 0xFFFFFFFF
    y = x * 0xC2B2AE35 & 0xFFFFFFFF
    return torch.stack([x ^ (x >> 16), y ^ (y >> 15)], -1).view(-1)[:n]


def _random_q8(x, bits20):
    """x [n] >= 0 or signed -> (codes, scales), each value rounded up or down to e4m3 with the probability that keeps its mean."""
    n = x.numel()
    rows = torch.nn.functional.pad(x, (0, -n % BLOCK)).view(-1, BLOCK)
    most = rows.abs().amax(1)
    dead, bad = most < 2.0 ** -100, ~torch.isfinite(most)
    scale = torch.where(dead, 0.0, torch.where(bad, math.nan, most / E4M3_MAX))
    y = rows * torch.where(dead | bad, 0.0, E4M3_MAX / most)[:, None]
    y = torch.where(bad[:, None], 0.0, y).view(-1)[:n]
    a = y.abs()
    low = a < 2.0 ** -6                                                  # below the normal numbers the step is 2^-9
    code = (torch.where(low, a + 2.0 ** -6, a).view(torch.int32) + bits20.to(torch.int32) >> 20) - torch.where(low, 121 << 3, 120 << 3)
    return code.clamp_max(126), torch.signbit(y), y != 0, scale


def _plain_adamw(s):
    c, q, t = s["case"], s["parts"], s["t"]
    gain, ok = 1.0, None
    if c["max_norm"] > 0:
        norm = torch.stack([g.double().square().sum() for g in q["g"]]).sum().sqrt()
        s["norm"].copy_(norm)
        gain = torch.clamp_max(c["max_norm"] / (s["norm"] + 1e-6), 1.0)
        ok = torch.isfinite(s["norm"])                                   # a step with such gradients changes nothing
    b1, b2 = np.float32(BETA1).item(), np.float32(BETA2).item()
    r1, r2 = np.float32(1.0 - BETA1).item(), np.float32(1.0 - BETA2).item()
    step_size = LR / -math.expm1(t * math.log(BETA1))
    inv_root = 1.0 / math.sqrt(-math.expm1(t * math.log(BETA2)))
    for i, (p, grad) in enumerate(zip(q["p"], q["g"])):
        n = p.numel()
        g = grad.float() * gain
        if c["state"] == "q8":
            m, v = ((q[k][i].view(torch.float8_e4m3fn).float() * q[k + "s"][i].repeat_interleave(BLOCK)[:n]) for k in ("m", "v"))
        else:
            m, v = q["m"][i], q["v"][i]
        m = b1 * m + r1 * g
        v = b2 * v + r2 * g * g
        new = p.float() * (1.0 - LR * DECAY) - step_size * (m / (torch.sqrt(v) * inv_root + EPS_ADAM))
        if c["state"] == "q8" or c["param"] == "bf16":
            bits = _random32(n, i, t)
        if c["param"] == "bf16":                                         # rounded up or down with the probability that keeps the mean
            low = (bits * 0x9E3779B9 & 0xFFFFFFFF) >> 16
            up = (new.view(torch.int32) + low.to(torch.int32)) >> 16
            new = torch.where(torch.isfinite(new), (up << 16).view(torch.float32), new)
        _keep(p, new, ok)
        if q["copy"] is not None:
            _keep(q["copy"][i], new, ok)
        if c["state"] == "q8":
            code, negative, _, scale = _random_q8(m, bits & 0xFFFFF)
            _keep(q["m"][i], code + negative.to(torch.int32) * 128, ok)
            _keep(q["ms"][i], scale, ok)
            code, _, some, scale = _random_q8(v, bits >> 12)
            _keep(q["v"][i], torch.where(some, code.clamp_min(1), code), ok)     # a second moment is never lost altogether
            _keep(q["vs"][i], scale, ok)
        else:
            _keep(q["m"][i], m, ok)
            _keep(q["v"][i], v, ok)


def _keep(old, new, ok):
    old.copy_(new if ok is None else torch.where(ok, new.to(old.dtype), old))


# The recurrence, plainly.
def _gates(s):
    """a and 1 - a in 32 bits; 1 - a from its own formula, since it is small where the memory is long."""
    g = s["g"].float()
    if s["case"]["gate"] == "log":
        return torch.exp(g), -torch.expm1(g)
    return torch.sigmoid(g), torch.sigmoid(-g)


def _plain_recurrence(a, u):
    """h_t = a_t h_{t-1} + u_t along dim 1 by doubling: after each round h_t holds the contributions of twice as many tokens."""
    a, h, reach = a.clone(), u.clone(), 1
    while reach < h.shape[1]:
        h[:, reach:] += a[:, reach:] * h[:, :-reach]
        a[:, reach:] *= a[:, :-reach].clone()
        reach *= 2
    return h


def _plain_scan_forward(s):
    c = s["case"]
    a, rest = _gates(s)
    u = s["x"].float()
    if c["convex"]:
        u = rest * u
    if s["h0"] is not None:
        u = torch.cat([u[:, :1] + a[:, :1] * s["h0"][:, None], u[:, 1:]], 1)
    h = _plain_recurrence(a, u)
    return {"h": h.to(s["x"].dtype), "last": h[:, -1].clone()}


def _plain_scan_backward(s):
    c = s["case"]
    a, rest = _gates(s)
    # lambda_t = dh_t + a_{t+1} lambda_{t+1}: the same recurrence, backwards
    later = torch.cat([a[:, 1:], torch.ones_like(a[:, :1])], 1)
    dh = s["dh"].float()
    if s["dlast"] is not None:
        dh = torch.cat([dh[:, :-1], dh[:, -1:] + s["dlast"][:, None]], 1)
    lam = _plain_recurrence(later.flip(1), dh.flip(1)).flip(1)
    before = s["h0"][:, None] if s["h0"] is not None else torch.zeros_like(a[:, :1])
    before = torch.cat([before, s["h"][:, :-1].float()], 1)
    if c["convex"]:
        before = before - s["x"].float()
    dg = lam * before * a
    if c["gate"] == "sigmoid":
        dg = dg * rest
    dx = rest * lam if c["convex"] else lam
    return {"dx": dx.to(s["x"].dtype), "dg": dg.to(s["g"].dtype), "dh0": a[:, 0] * lam[:, 0] if s["h0"] is not None else None}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------------------
def exact(case, seed):
    s = prepare(case, seed)
    return {"heads": _exact_heads, "adamw": _exact_adamw, "scan": _exact_scan}[case["op"].split("_")[0]](s)


def _exact_heads(s):
    """The rotation as a product of complex numbers; gradients by automatic differentiation of the definition."""
    c = s["case"]
    B, H, N, d = c["B"], c["H"], c["t"] * c["h"] * c["w"], c["d"]
    pos = s["positions"]
    if pos is None:
        pos = torch.cartesian_prod(*[torch.arange(k, device=DEVICE) for k in (c["t"], c["h"], c["w"])]).view(1, N, 3)
    angle = torch.empty(pos.shape[0], N, 1, d // 2, dtype=torch.float64, device=DEVICE)
    j = 0
    for a, width in enumerate(_axes(d)):
        for i in range(width // 2):
            angle[:, :, 0, j] = pos[..., a].double() * math.exp(-2 * i / width * math.log(THETA))
            j += 1
    turn = torch.polar(torch.ones_like(angle), angle)

    def definition(x, w, scale):
        if w is not None:
            x = x / torch.sqrt((x * x).sum(-1, keepdim=True) / d + EPS_NORM) * w
        pairs = x.unflatten(-1, (d // 2, 2)) if c["pairing"] == "interleaved" else x.unflatten(-1, (2, d // 2)).transpose(-1, -2)
        y = torch.view_as_real(torch.complex(pairs[..., 0], pairs[..., 1]) * turn) * scale
        return (y if c["pairing"] == "interleaved" else y.transpose(-1, -2)).flatten(-2).permute(0, 2, 1, 3)

    if c["op"] == "heads_forward":
        Q, K = (definition(x.double(), w if w is None else w.double(), k).contiguous() for x, w, k in zip(s["xs"], s["w"], (d ** -0.5, 1.0)))
        return {"Q": Q, "K": K, "V": s["xs"][2].double().permute(0, 2, 1, 3).contiguous()}
    dx, dw = [], []
    for x, w, k, dy in zip(s["xs"], s["w"], (d ** -0.5, 1.0), s["d"]):
        x = x.double().requires_grad_()
        w = w if w is None else w.double().requires_grad_()
        with torch.enable_grad():
            got = torch.autograd.grad(definition(x, w, k), [x] if w is None else [x, w], dy.double())
        dx.append(got[0])
        dw.append(got[1] if w is not None else None)
        del got, x
    dx.append(s["d"][2].double().permute(0, 2, 1, 3))
    return {"dX": torch.stack(dx, 2) if s["X"] is not None else dx, "dw": dw}


def _exact_adamw(s):
    """Moments and weights before they are rounded; what the 8-bit states hold depends on the rounding and has no such value."""
    c, t = s["case"], s["t"] + 1
    g = s["g"].double()
    out = {"copy": None, "norm": None}
    if c["max_norm"] > 0:
        norm = torch.linalg.vector_norm(g)
        out["norm"] = norm
        g = g * min(1.0, c["max_norm"] / (norm.item() + 1e-6))
    if c["state"] == "q8":
        m, v = ((s[k].view(torch.float8_e4m3fn).double().view(-1, BLOCK) * s[k + "s"].double()[:, None]).view(-1) for k in ("m", "v"))
    else:
        m, v = s["m"].double(), s["v"].double()
    m, v = BETA1 * m + (1 - BETA1) * g, BETA2 * v + (1 - BETA2) * g ** 2
    p = s["p"].double()
    out["p"] = p - LR * DECAY * p - LR * (m / (1 - BETA1 ** t)) / ((v / (1 - BETA2 ** t)) ** 0.5 + EPS_ADAM)
    if s["copy"] is not None:
        out["copy"] = out["p"]
    if c["state"] == "q8":
        return dict(out, m=None, v=None, m_scale=m.view(-1, BLOCK).abs().amax(1) / E4M3_MAX, v_scale=v.view(-1, BLOCK).amax(1) / E4M3_MAX)
    return dict(out, m=m, v=v)


def _exact_scan(s):
    """Token by token."""
    c, N = s["case"], s["case"]["N"]
    g, x = s["g"].double(), s["x"].double()
    a = torch.exp(g) if c["gate"] == "log" else 1 / (1 + torch.exp(-g))
    share = (-torch.expm1(g) if c["gate"] == "log" else 1 / (1 + torch.exp(g))) if c["convex"] else torch.ones_like(a)
    zero = torch.zeros(c["B"], c["C"], dtype=torch.float64, device=DEVICE)
    if c["op"] == "scan_forward":
        u, h = share * x, torch.empty_like(x)
        now = s["h0"].double() if s["h0"] is not None else zero
        for t in range(N):
            now = torch.addcmul(u[:, t], a[:, t], now)
            h[:, t] = now
        return {"h": h, "last": now}
    lam, dh = torch.empty_like(x), s["dh"].double()
    now = s["dlast"].double() if s["dlast"] is not None else zero
    for t in range(N - 1, -1, -1):
        now = dh[:, t] + now
        lam[:, t] = now
        now = a[:, t] * now
    before = torch.empty_like(x)
    before[:, 0] = s["h0"].double() if s["h0"] is not None else zero
    before[:, 1:] = s["h"][:, :-1].double()
    slope = a if c["gate"] == "log" else a * (1 / (1 + torch.exp(g)))
    return {"dx": lam * share, "dg": lam * (before - x if c["convex"] else before) * slope, "dh0": now if s["h0"] is not None else None}


# ---- what a pass cannot do without -------------------------------------------------------------------------------------
def work(case):
    """Inputs read once, results written once."""
    c = case
    if c["op"].startswith("heads"):
        n, elt = c["B"] * c["H"] * c["t"] * c["h"] * c["w"] * c["d"], 2 if c["dtype"] == "bf16" else 4
        extra = c["B"] * c["t"] * c["h"] * c["w"] * 12 if c["positions"] == "given" else 0
        if c["op"] == "heads_forward":
            return {"bytes": 6 * n * elt + extra, "flops": 2 * n * (8 if c["norm"] else 4)}
        return {"bytes": (8 if c["norm"] else 6) * n * elt + extra, "flops": 2 * n * (16 if c["norm"] else 4)}
    if c["op"] == "adamw":
        n, wide = sum(_sizes(c)), {"bf16": 2, "f32": 4}
        by = wide[c["grad"]] + 2 * wide[c["param"]] + (2 if c["param"] == "f32" else 0)
        by += 16 if c["state"] == "f32" else 4 + 4 * 4 / BLOCK
        return {"bytes": n * by, "flops": n * (16 if c["max_norm"] > 0 else 14)}
    n, elt = c["B"] * c["N"] * c["C"], 2 if c["dtype"] == "bf16" else 4
    state = c["B"] * c["C"] * 4 * (2 if c["carry"] else 1)
    if c["op"] == "scan_forward":
        return {"bytes": 3 * n * elt + state, "flops": n * (8 if c["convex"] else 6)}
    return {"bytes": (6 if c["convex"] else 5) * n * elt + state, "flops": n * (12 if c["convex"] else 9)}
