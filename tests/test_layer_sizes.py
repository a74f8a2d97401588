"""Calls of the layer's operators at the far end of what their entry points take."""
import pytest
import torch

import paper_2605_21325_amd as tri

BF = torch.bfloat16


@pytest.mark.gpu
def test_norm_of_more_rows_than_a_grid_has_threads_for_in_one_dimension():
    """2^26 rows and some: four a workgroup of 256 threads are 2^32 threads."""
    N, D = (1 << 26) + 5, 8
    x = torch.randn(1 << 12, D, device="cuda").to(BF)
    w = torch.rand(D, device="cuda").to(BF)
    want = tri.add_rms_norm(x, w)[0]
    x = x.repeat((1 << 14) + 1, 1)[:N]
    y, _ = tri.add_rms_norm(x, w)
    assert torch.equal(y[:-5].view(-1, *want.shape), want.expand(1 << 14, *want.shape)) and torch.equal(y[-5:], want[:5])
    q, scales, _ = tri.add_rms_norm_fp8(x, w)
    q0, scales0, _ = tri.add_rms_norm_fp8(x[:1 << 12], w)
    assert torch.equal(scales[-5:], scales0[:5]) and torch.equal(q[-5:].view(torch.uint8), q0[:5].view(torch.uint8))
    assert torch.equal(scales[:-5].view(-1, 1 << 12), scales0.view(1, -1).expand(1 << 14, -1))
