"""Head preparation and gated recurrence in 64 bits, straight from their formulas; the AdamW step too.  For the tests."""

import torch


def grid_positions(grid, start=(0, 0, 0)):
    return torch.cartesian_prod(*[torch.arange(n, dtype=torch.int64) + s for n, s in zip(grid, start)]).view(-1, len(grid))


def angles(positions, widths, theta=10000.0, inv_freq=None):
    """positions [..., axes] -> angles [..., pairs]."""
    cols, pair = [], 0
    for a, width in enumerate(widths):
        for j in range(width // 2):
            f = inv_freq[pair] if inv_freq is not None else theta ** (-j / (width // 2))
            cols.append(positions[..., a].double() * f)
            pair += 1
    return torch.stack(cols, -1) if cols else positions.new_zeros(positions.shape[:-1] + (0,), dtype=torch.float64)


def turn(x, ang, pairing):
    """x [B,N,H,d], ang [N or B,N, pairs]."""
    c, s = torch.cos(ang)[..., None, :].to(x.device), torch.sin(ang)[..., None, :].to(x.device)
    R = 2 * ang.shape[-1]
    y = x.clone()
    a, b = ((x[..., 0:R:2], x[..., 1:R:2]) if pairing == "interleaved" else (x[..., :R // 2], x[..., R // 2:R]))
    ya, yb = a * c - b * s, a * s + b * c
    if pairing == "interleaved":
        y[..., 0:R:2], y[..., 1:R:2] = ya, yb
    else:
        y[..., :R // 2], y[..., R // 2:R] = ya, yb
    return y


def heads(x, w, ang, scale, pairing, eps):
    """x [B,N,H,d] -> [B,H,N,d]; eps None: no norm; w None: ones."""
    if eps is not None:
        x = x / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
        if w is not None:
            x = x * w
    return (turn(x, ang, pairing) * scale).permute(0, 2, 1, 3)


def heads_backward(dY, x, w, ang, scale, pairing, eps):
    """dY [B,H,N,d] -> dx [B,N,H,d], dw [d] (None without norm)."""
    g = turn(dY.permute(0, 2, 1, 3) * scale, -ang, pairing)
    if eps is None:
        return g, None
    r = 1 / torch.sqrt(x.square().mean(-1, keepdim=True) + eps)
    xh = x * r
    gw = g * (w if w is not None else 1.0)
    return r * (gw - xh * (gw * xh).mean(-1, keepdim=True)), (g * xh).sum((0, 1, 2))


def gates(z, gate):
    return (torch.exp(z), -torch.expm1(z)) if gate == "log" else (torch.sigmoid(z), torch.sigmoid(-z))


def scan(x, z, h0, gate, convex):
    a, rest = gates(z, gate)
    u = rest * x if convex else x
    h, now = [], h0 if h0 is not None else torch.zeros_like(x[:, 0])
    for t in range(x.shape[1]):
        now = a[:, t] * now + u[:, t]
        h.append(now)
    return torch.stack(h, 1)


def scan_backward(x, z, h0, h, dh, dl, gate, convex):
    a, rest = gates(z, gate)
    zero = torch.zeros_like(x[:, 0])
    lam, mu = torch.empty_like(x), dl if dl is not None else zero
    for t in range(x.shape[1] - 1, -1, -1):
        lam[:, t] = dh[:, t] + mu
        mu = a[:, t] * lam[:, t]
    before = torch.cat([(h0 if h0 is not None else zero)[:, None], h[:, :-1]], 1)
    slope = a if gate == "log" else a * rest
    return lam * rest if convex else lam, lam * (before - x if convex else before) * slope, mu


def adamw(p, g, m, v, lr, t, b1=0.9, b2=0.999, eps=1e-8, wd=0.0):
    m, v = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    return p - lr * wd * p - lr * (m / (1 - b1 ** t)) / (torch.sqrt(v / (1 - b2 ** t)) + eps), m, v


def mix32(x):
    x = x ^ (x >> 16)
    x = x * 0x7FEB352D & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = x * 0x846CA68B & 0xFFFFFFFF
    return x ^ (x >> 16)


def random_words(n, tensor, step, seed, device):
    """The 32 random bits of each element of a tensor in a step."""
    M = 0xFFFFFFFF
    k = mix32((mix32(mix32(mix32(seed & M) ^ seed >> 32) ^ step & M) + tensor) & M)
    i = torch.arange(0, n, 2, dtype=torch.int64, device=device)
    x = mix32((k + i // 128 * 0x9E3779B9) & M) + i % 128 // 2 * 0x9E3779B9 & M
    x = (x ^ x >> 16) * 0x7FEB352D & M
    x = (x ^ x >> 15) * 0x846CA68B & M
    y = x * 0xC2B2AE35 & M
    return torch.stack([x ^ x >> 16, y ^ y >> 15], -1).view(-1)[:n]


def round_q8(x, bits20):
    """Codes (as signed magnitudes in units of the code) and scales of x, rounded by 20 random bits: the code below, or the one above where the
    random number is within the remainder.  In 64 bits, from the products in 32 that the formula names."""
    n = x.numel()
    rows = torch.nn.functional.pad(x, (0, -n % 128)).view(-1, 128)
    most = rows.abs().amax(1)
    y = (rows * (most.reciprocal() * 448.0)[:, None]).view(-1)[:n].abs().double()
    binade = torch.frexp(y.clamp_min(2.0 ** -6))[1].to(torch.int64) - 1
    step = (binade - 3 + 1023 << 52).view(torch.float64)                 # (powers of two by their bits: 2.0 ** x is off by a unit on the GPU)
    below = torch.floor(y / step)
    up = ((y / step - below) * 2 ** 20).floor() + bits20 >= 2 ** 20
    value = torch.where(y > 0, ((below + up) * step).clamp_max(448.0), 0.0)
    return value * torch.where(x < 0, -1.0, 1.0), most * (1.0 / torch.tensor(448.0, device=x.device))


def decode_q8(codes, scales):
    n = codes.numel()
    return codes.view(torch.float8_e4m3fn).double() * scales.double().repeat_interleave(128)[:n]


HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float32: 2.0 ** -24}


def bits(t):
    return t.view(torch.int16 if t.element_size() == 2 else torch.int32)


