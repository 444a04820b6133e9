"""Second moments far below their group's largest, down to the smallest fp32 number."""
import pytest
import torch

from paper_2602_12128_b200 import binding

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("param", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [128, 300, 6000])
def test_a_second_moment_below_the_normal_numbers_keeps_a_positive_code(n, param):
    """v = (1 - 0.999) g^2: 1e-39 is below the normal numbers, 1e-43 is 71 units of 2^-149, 3e-45 two of them; 1e-47 is zero and stays zero."""
    g = torch.full((n,), 1e-18, device="cuda")
    g[1::5], g[2::5], g[3::5] = 1e-20, 1.7e-21, 1e-22
    g[::128] = 1.0                                          # every group lives
    want = torch.tensor(1 - 0.999, dtype=torch.float32, device="cuda") * g * g
    assert set((want.view(torch.int32)[[6, 7, 8]]).tolist()) == {71, 2, 0}
    for seed in range(4):
        opt = binding.AdamW([torch.zeros(n, device="cuda", dtype=param)], [g], state="q8", seed=seed)
        opt.step(1e-3)
        small = g < 1
        assert torch.equal(opt.vs[0][small], (want > 0).to(torch.uint8)[small])
        assert (opt.vs[0][~small] == 0x7e).all()            # 448, the largest code
