"""A wait of the recurrence that runs out is recorded in the workspace and can be read, as for the attention.  The wait is one for what
never comes, with a limit of a millisecond."""
import pytest
import torch

from paper_2602_12128_b200 import binding as b


def test_status_calls_are_checked():
    lib = b.load_library()
    op = b.Scan(1, 50, 64, device=None)
    P = 0x100000        # never dereferenced
    assert lib.hla_scan_last_device_status(None, P, None) == b.HLA_ERR_INVALID_ARG
    for bad in (None, P + 16):
        assert lib.hla_scan_last_device_status(op.ctx, bad, None) == b.HLA_ERR_INVALID_ARG
        assert lib.hla_scan_selftest_bounded_wait(op.ctx, bad, 256, None) == b.HLA_ERR_INVALID_ARG
    assert lib.hla_scan_selftest_bounded_wait(None, P, 256, None) == b.HLA_ERR_INVALID_ARG
    assert lib.hla_scan_selftest_bounded_wait(op.ctx, P, 255, None) == b.HLA_ERR_WORKSPACE
    assert lib.hla_scan_workspace_bytes(op.ctx) >= b.HLA_SCAN_STATUS_BYTES


@pytest.mark.gpu
@pytest.mark.parametrize("N,C", [(3000, 768), (30000, 64)])      # the second one runs in parts
def test_a_wait_that_runs_out_is_recorded(N, C):
    op = b.Scan(1, N, C, gate="sigmoid")
    x, z = (torch.randn(1, N, C, device="cuda").bfloat16() for _ in range(2))
    want, last = op.forward(x, z)
    grads = op.backward(x, z, want, x)
    assert op.device_status() == b.HLA_OK
    assert b.load_library().hla_scan_selftest_bounded_wait(op.ctx, op.workspace.data_ptr(), op.workspace.numel(), torch.cuda.current_stream().cuda_stream) == b.HLA_OK
    got, out = op.forward(x, z)                             # (calls in between leave the record)
    assert op.device_status() == b.HLA_ERR_DEVICE_TIMEOUT
    assert op.device_status() == b.HLA_OK                   # since it was last asked
    assert torch.equal(got, want) and torch.equal(out, last)
    assert all(torch.equal(p, q) for p, q in zip(op.backward(x, z, want, x)[:2], grads)) and op.device_status() == b.HLA_OK
    assert not op.workspace[:b.HLA_SCAN_STATUS_BYTES].any()


@pytest.mark.gpu
def test_a_call_that_needs_no_workspace_can_have_none():
    B, N, C = 1, 500, 1536
    op = b.Scan(B, N, C)
    x, z = (torch.randn(B, N, C, device="cuda").bfloat16() for _ in range(2))
    z = -z.abs()
    want, _ = op.forward(x, z)
    h = torch.full_like(want, 7.0)
    stream = torch.cuda.current_stream().cuda_stream
    assert b.load_library().hla_scan_forward(op.ctx, x.data_ptr(), z.data_ptr(), None, h.data_ptr(), None, None, 0, stream) == b.HLA_OK
    assert torch.equal(h, want)
