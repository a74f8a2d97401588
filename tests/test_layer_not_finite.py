"""The norm of rows that are not finite, as include/triinv.h states it for each kind of result."""
import pytest
import torch

import paper_2605_21325_amd as tri

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("N", [5, 2049])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16, torch.float32])
def test_rows_with_infinities_and_nan(N, dtype):
    D = 512
    x, w = torch.randn(N, D, device="cuda").to(dtype), torch.rand(D, device="cuda").to(dtype) + 1
    x[1, 3], x[2, 200], x[3, 511] = float("nan"), float("inf"), -float("inf")
    y, _ = tri.add_rms_norm(x, w)
    assert torch.isnan(y[1]).all() and torch.isfinite(y[[0, 4]]).all()
    for row, at in ((2, 200), (3, 511)):
        there = torch.arange(D, device="cuda") == at
        assert torch.isnan(y[row][there]).all() and (y[row][~there] == 0).all()
    q, scales, _ = tri.add_rms_norm_fp8(x, w)
    assert torch.isnan(scales[1:4]).all() and torch.isnan(q[1:4].float()).all() and torch.isfinite(scales[[0, 4]]).all()
    q, scales, _ = tri.add_rms_norm_fp8(x, w, group=128)
    assert torch.isnan(scales[1]).all() and torch.isnan(q[1].float()).all()
    for row, at in ((2, 1), (3, 3)):
        there = torch.arange(D // 128, device="cuda") == at
        z = q[row].float().view(-1, 128)
        assert torch.isnan(scales[row][there]).all() and (scales[row][~there] == 1).all() and torch.isnan(z[there]).all() and (z[~there] == 0).all()


def test_rows_whose_squares_pass_fp32():
    x = torch.full((2, 256), 1e25, device="cuda")
    x[1] = 1.0
    y, _ = tri.add_rms_norm(x, torch.ones(256, device="cuda"))
    assert (y[0] == 0).all() and torch.isfinite(y[1]).all()
