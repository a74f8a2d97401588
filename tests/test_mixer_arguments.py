"""Results handed over for what was not given are refused, not left as they were: decided on the host."""
import pytest
import torch

import paper_2605_21325_amd as tri

Q, W = torch.zeros(2, 5, 4, 64), torch.zeros(64)
K = torch.zeros(2, 5, 2, 64)


def test_a_result_for_keys_that_are_not_there():
    with pytest.raises(ValueError, match="k_out without k"):
        tri.qk_norm_rope(Q, None, k_out=K)
    with pytest.raises(ValueError, match="dk without k"):
        tri.qk_norm_rope_bwd(Q, None, Q, None, dk=K)
