"""What psa_norm's description says of rows with a NaN, with an infinity, and with squares that fp32 does not hold."""
import pytest
import torch

from paper_2410_20305_b200 import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("D", [3, 200, 1237, 4096])
@pytest.mark.parametrize("rms", [False, True])
def test_rows_that_are_not_finite(D, rms, dtype):
    x = torch.randn(7, D, generator=torch.Generator().manual_seed(D)).to(dtype).cuda()
    w = torch.ones(D, dtype=dtype, device="cuda")
    clean, clean_stats = B.psa_norm(x, w, rms=rms)
    y = x.clone()
    y[1, D // 2] = float("nan")
    y[3, D - 1] = float("-inf")
    y[5] = 1e30 * (1 - 2 * (torch.arange(D, device="cuda") % 2))
    out, stats = B.psa_norm(y, w, rms=rms)
    fine = [0, 2, 4, 6]
    assert torch.equal(out[fine], clean[fine]) and torch.equal(stats[:, fine], clean_stats[:, fine])
    assert out[1].isnan().all()
    assert stats[1, 5] == 0 and not out[5].any()      # squares of 1e60
    if rms:
        assert stats[1, 3] == 0 and out[3, D - 1].isnan() and not out[3, :D - 1].any()
    else:
        assert out[3].isnan().all()
