"""The recurrence in front of causal HLA: its output, in pieces with the state carried, is prepared for heads and goes through causal HLA, whose
result is held against the masked quadratic definition in 64 bits."""
import numpy as np
import pytest
import torch

import ops_reference as ref
from hla_testlib import TOL, relerr, to_np
from oracle import hla_oracle as orc
from paper_2602_12128_b200 import binding

pytestmark = pytest.mark.gpu


def test_causal_hla_of_a_carried_recurrence():
    B, H, d, n, pieces, eps = 1, 2, 128, 150, 4, 1e-6
    C, N = H * d, n * pieces
    g = torch.Generator(device="cuda").manual_seed(7)
    X = torch.randn(B, N, 2, C, generator=g, device="cuda").bfloat16()
    scan, state, parts = binding.Scan(B, n, C, gate="sigmoid", convex=True), torch.zeros(B, C, device="cuda"), []
    for i in range(pieces):
        part = X[:, i * n:(i + 1) * n]
        parts.append(scan.forward(part[:, :, 0], part[:, :, 1], h0=state, h_last=state)[0])
    y = torch.cat(parts, 1)
    h = ref.scan(X[:, :, 0].double(), X[:, :, 1].double(), None, "sigmoid", True)
    # a rounding to bf16, and before it 32 units of 2^-24 of the largest quantities that enter (gates below 1 on values below 6, sums of a few of them)
    assert ((y.double() - h).abs() <= 2.0 ** -8 * h.abs() + 32 * 2.0 ** -24 * 6).all()
    heads = binding.Heads(B, H, N, d, axes=(d,), grid=(N,), norm=True)
    rows = y.view(B, N, H, d)
    Q, K, V = heads.forward(rows, rows, rows)
    assert torch.equal(V, rows.transpose(1, 2))
    qf = Q[..., :6].float().abs().contiguous()
    kf = K[..., :18].float().abs().view(B, H, N, 3, 6).permute(0, 1, 3, 2, 4).contiguous()
    hla = binding.Hla(B, H, N, d, phi="none", causal=True, eps=eps)
    O = hla.forward(qf, kf, V)
    torch.cuda.synchronize()
    assert hla.device_status() == binding.HLA_OK and scan.device_status() == binding.HLA_OK
    want, _ = orc.hla_core_forward(to_np(qf), to_np(kf), to_np(V), eps, "causal_quadratic")
    assert relerr(to_np(O), want) < TOL["bf16"]
    assert np.isfinite(to_np(O)).all()
