"""The scratch of the recurrence is what its parts take and no more: nothing where a call has one part, and nothing is written behind it."""
import pytest
import torch

from paper_2602_12128_b200 import binding as b

GUARD = 4096


@pytest.mark.parametrize("B,N,C,dtype,parts", [
    (1, 75600, 64, "bf16", 27),       # 3 x 148 places for blocks, clusters of eight, two tiles of 32 channels
    (1, 75600, 512, "bf16", 3), (1, 75600, 768, "bf16", 1),
    (2, 75600, 1536, "bf16", 1),      # 96 tiles: clusters of four blocks, one part
    (1, 2048, 1, "f32", 1),           # four exchanges: two parts would not be worth their second reading
    (1, 8200, 1, "f32", 8),           # 17 exchanges in clusters of eight, at least two a part
    (1, 1, 1, "bf16", 1),
])
def test_size(B, N, C, dtype, parts):
    op = b.Scan(B, N, C, dtype=dtype, device=None)
    states = (parts + 1) * B * C * 8 if parts > 1 else 0
    assert b.load_library().hla_scan_workspace_bytes(op.ctx) == 256 + -(-states // 256) * 256


@pytest.mark.gpu
@pytest.mark.parametrize("B,N,C,dtype", [(1, 75600, 64, "bf16"), (1, 30000, 33, "bf16"), (1, 75600, 512, "bf16"), (2, 9000, 64, "f32"), (1, 8200, 1, "f32"), (3, 20000, 20, "bf16")])
def test_nothing_behind_it_is_written(B, N, C, dtype):
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    lib, op = b.load_library(), b.Scan(B, N, C, dtype=dtype, gate="sigmoid", convex=True)
    need = lib.hla_scan_workspace_bytes(op.ctx)
    assert need > 256
    room = torch.full((need + GUARD,), 171, dtype=torch.uint8, device="cuda")
    x, z, dh = (torch.randn(B, N, C, device="cuda").to(dt) for _ in range(3))
    h0 = torch.randn(B, C, device="cuda")
    want, last = op.forward(x, z, h0=h0)
    grads = op.backward(x, z, want, dh, h0=h0, dlast=h0)
    h, out, dx, dg, dh0 = torch.empty_like(x), torch.empty_like(h0), torch.empty_like(x), torch.empty_like(x), torch.empty_like(h0)
    s = torch.cuda.current_stream().cuda_stream
    assert lib.hla_scan_forward(op.ctx, x.data_ptr(), z.data_ptr(), h0.data_ptr(), h.data_ptr(), out.data_ptr(), room.data_ptr(), need, s) == b.HLA_OK
    assert lib.hla_scan_backward(op.ctx, x.data_ptr(), z.data_ptr(), h0.data_ptr(), h.data_ptr(), dh.data_ptr(), h0.data_ptr(), dx.data_ptr(), dg.data_ptr(), dh0.data_ptr(),
                                 room.data_ptr(), need, s) == b.HLA_OK
    assert torch.equal(h, want) and torch.equal(out, last) and all(torch.equal(p, q) for p, q in zip((dx, dg, dh0), grads))
    assert (room[need:] == 171).all()
    assert lib.hla_scan_last_device_status(op.ctx, room.data_ptr(), s) == b.HLA_OK
