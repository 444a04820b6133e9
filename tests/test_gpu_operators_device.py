"""A device may be given by its number, 0 among them."""
import pytest
import torch

from paper_2602_12128_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("device", [0, "cuda", torch.device("cuda", 0)])
def test_a_device_by_its_number(device):
    B, H, N, d = 1, 2, 24, 64
    heads = binding.Heads(B, H, N, d, axes=(24, 20, 20), grid=(2, 3, 4), norm=True, device=device)
    q, dQ = torch.randn(B, N, H, d, device="cuda").bfloat16(), torch.randn(B, H, N, d, device="cuda").bfloat16()
    dq = torch.full_like(q, float("nan"))
    dwq, _ = heads.backward(dQ=dQ, q=q, dq=dq)
    assert torch.isfinite(dq).all() and torch.isfinite(dwq).all() and dwq.any()
    scan = binding.Scan(1, 30000, 64, device=device)      # (runs in parts)
    x = torch.randn(1, 30000, 64, device="cuda").bfloat16()
    h, _ = scan.forward(x, -x.abs())
    assert torch.isfinite(h).all() and scan.device_status() == binding.HLA_OK
    opt = binding.AdamW([torch.zeros(64, device="cuda")], [torch.ones(64, device="cuda")], device=device)
    opt.step(1e-3, max_norm=1.0)
    assert opt.norm.item() == 8.0
