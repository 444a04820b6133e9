"""The operators in a row, as a training step of one attention layer runs them: projection -> heads -> HLA -> merge, and back, then the feature
networks' gradients into AdamW; eager and as one captured graph."""
import math

import pytest
import torch

import ops_reference as ref
from paper_2602_12128_b200 import binding

pytestmark = pytest.mark.gpu


class Layer:
    def __init__(self, state, seed=0):
        self.B, self.H, self.grid, self.d = 1, 2, (2, 9, 10), 128
        B, H, N, d = self.B, self.H, math.prod(self.grid), self.d
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.X = rnd(B, N, 3, H, d).bfloat16()
        self.w = [(1 + 0.1 * rnd(d)).bfloat16() for _ in range(2)]
        self.dY = rnd(B, N, H, d).bfloat16()
        self.heads = binding.Heads(B, H, N, d, axes=(44, 42, 42), grid=self.grid, norm=True, q_scale=1.0)
        self.merge = binding.Heads(B, H, N, d)
        self.op = binding.Hla(B, H, N, d)
        self.master = [[rnd(d, d) / math.sqrt(d), 0.1 * rnd(d), rnd(d, 6) / math.sqrt(d), 0.3 + 0.1 * rnd(6)] for _ in range(4)]
        self.weights = [[w.bfloat16() for w in m] for m in self.master]
        self.op.set_phi(tuple(self.weights[0]), [tuple(w) for w in self.weights[1:]])
        self.grads = [[torch.empty_like(w) for w in m] for m in self.master]
        flat = lambda t: [x for m in t for x in m]
        self.opt = binding.AdamW(flat(self.master), flat(self.grads), copies=flat(self.weights), state=state, weight_decay=0.01)
        self.lr, self.number = torch.tensor(1e-3, device="cuda"), torch.zeros((), dtype=torch.int64, device="cuda")

    def step(self):
        xs = [self.X[:, :, i] for i in range(3)]
        Q, K, V = self.heads.forward(*xs, *self.w)
        O = self.op.forward(Q, K, V)
        Y = torch.empty_like(self.dY)
        self.merge.backward(dV=O, dv=Y)                                  # head-major to token-major, for the output projection
        dO = self.merge.forward(v=self.dY)[2]
        dQ, dK, dV = self.op.backward(Q, K, V, O, dO)
        dX = torch.empty_like(self.X)
        dws = self.heads.backward(dQ, dK, dV, *xs, *[dX[:, :, i] for i in range(3)], *self.w)
        binding.hla_backward_weights(self.op.ctx, Q, K, tuple(self.grads[0]), [tuple(g) for g in self.grads[1:]], self.op.workspace)
        self.number.add_(1)
        self.opt.step(self.lr, self.number, max_norm=1.0)
        return {"Q": Q, "K": K, "V": V, "O": O, "Y": Y, "dO": dO, "dQ": dQ, "dK": dK, "dV": dV, "dX": dX, "dwq": dws[0], "dwk": dws[1], "norm": self.opt.norm}


@pytest.mark.parametrize("state", ["f32", "q8"])
def test_step_of_a_layer(state):
    layer = Layer(state)
    before = [w.clone() for m in layer.master for w in m]
    got = layer.step()
    torch.cuda.synchronize()
    assert layer.op.device_status() == binding.HLA_OK
    ang = ref.angles(ref.grid_positions(layer.grid), (44, 42, 42)).cuda()
    half = 2.0 ** -8
    for name, i in (("Q", 0), ("K", 1)):
        want = ref.heads(layer.X[:, :, i].double(), layer.w[i].double(), ang, 1.0, "interleaved", 1e-6)
        assert ((got[name].double() - want).abs() <= half * want.abs() + 1e-4).all()
        dx, dw = ref.heads_backward(got["d" + name].double(), layer.X[:, :, i].double(), layer.w[i].double(), ang, 1.0, "interleaved", 1e-6)
        assert ((got["dX"][:, :, i].double() - dx).abs() <= half * dx.abs() + 1e-4 * dx.abs().max()).all()
        torch.testing.assert_close(got["dw" + name.lower()].double(), dw, rtol=1e-4, atol=1e-4 * dw.abs().max().item())
    assert torch.equal(got["V"], layer.X[:, :, 2].transpose(1, 2)) and torch.equal(got["Y"], got["O"].transpose(1, 2))
    assert torch.equal(got["dO"], layer.dY.transpose(1, 2)) and torch.equal(got["dX"][:, :, 2], got["dV"].transpose(1, 2))
    grads = [g for m in layer.grads for g in m]
    norm = math.sqrt(sum(g.double().square().sum().item() for g in grads))
    assert abs(got["norm"].item() - norm) <= 1e-6 * norm
    gain = min(1.0, 1.0 / (norm + 1e-6))
    for w, b, g, low in zip((w for m in layer.master for w in m), before, grads, (w for m in layer.weights for w in m)):
        want, _, _ = ref.adamw(b.double(), g.double() * gain, torch.zeros_like(b, dtype=torch.float64), torch.zeros_like(b, dtype=torch.float64), 1e-3, 1, wd=0.01)
        assert ((w.double() - want).abs() <= 1e-3 * 2e-5 + 2.0 ** -23 * b.double().abs()).all()
        assert torch.equal(low, w.bfloat16())


@pytest.mark.parametrize("state", ["f32", "q8"])
def test_captured_steps_are_the_eager_ones(state):
    eager, layer = Layer(state), Layer(state)
    layer.step()                                                         # (first calls look device addresses and attributes up)
    layer = Layer(state)
    layer.op.forward(*layer.heads.forward(*[layer.X[:, :, i] for i in range(3)], *layer.w))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = layer.step()
    for _ in range(3):
        want = eager.step()
        graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(got[k], want[k]) for k in want)
    for a, b in zip((w for m in eager.master for w in m), (w for m in layer.master for w in m)):
        assert torch.equal(a, b)


def test_a_causal_layer_with_decay_in_pieces():
    """The scan next to causal HLA: both carry their state from one piece of a sequence to the next."""
    B, H, d, n, pieces = 1, 2, 128, 200, 3
    C = H * d
    g = torch.Generator(device="cuda").manual_seed(1)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
    X = rnd(B, n * pieces, 2, C).bfloat16()
    scan, whole = binding.Scan(B, n, C, gate="sigmoid", convex=True), binding.Scan(B, n * pieces, C, gate="sigmoid", convex=True)
    want, last = whole.forward(X[:, :, 0], X[:, :, 1])
    state, parts = torch.zeros(B, C, device="cuda"), []
    for i in range(pieces):
        part = X[:, i * n:(i + 1) * n]
        parts.append(scan.forward(part[:, :, 0], part[:, :, 1], h0=state, h_last=state)[0])
    assert ((torch.cat(parts, 1).double() - want.double()).abs() <= 2.0 ** -7 * want.double().abs() + 1e-5).all()
    torch.testing.assert_close(state, last, rtol=1e-5, atol=1e-5)
    # its output is the input of the head preparation of a causal HLA
    heads, hla = binding.Heads(B, H, n, d, axes=(128,), grid=None, norm=True), binding.Hla(B, H, n, d, phi="none", causal=True)
    pos = torch.arange(n, device="cuda", dtype=torch.int32)[:, None].contiguous()
    y = parts[0].view(B, n, H, d)
    Q, K, V = heads.forward(y, y, y, positions=pos)
    qf = Q[..., :6].float().abs().contiguous()
    kf = K[..., :18].float().abs().view(B, H, n, 3, 6).permute(0, 1, 3, 2, 4).contiguous()
    O = hla.forward(qf, kf, V)
    torch.cuda.synchronize()
    assert hla.device_status() == binding.HLA_OK and torch.isfinite(O).all()
