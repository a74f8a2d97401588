"""Calls of the layer's operators without a token or a row."""
import pytest
import torch

import paper_2605_21325_amd as tri
from test_layer_gpu import BF, HF, make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens", [[0], [0, 0, 0]])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("delta,state,C", [(True, True, 64), (False, True, 128), (True, False, 16)])
def test_sequences_without_tokens(lens, dtype, delta, state, C):
    x = make(lens, 2, 1, 64, 72, C, dtype, True, delta, state)
    first = torch.zeros(len(lens), 2, 64, 72) if x["state"] is None else x["state"].cpu()
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, W=x["w"], state=x["state"])
    assert o.shape == x["u"].shape and torch.equal(final.cpu(), first)
    got = tri.gdn_chunk_attn_bwd_varlen(x["q"], x["k"], x["u"], x["g"], x["do"], lens, C, W=x["w"], state=x["state"], dstate=x["dstate"])
    assert [None if t is None else t.shape for t in got[:5]] == [None if x[n] is None else x[n].shape for n in ("q", "k", "u", "w", "g")]
    assert (got[5] is None) == (not state) and (not state or torch.equal(got[5].cpu(), x["dstate"].cpu()))


def test_fixed_sequences_without_tokens_and_norms_without_rows():
    x = make([0, 0], 2, 2, 64, 64, 64, BF)
    one = {n: x[n].view(2, 0, *x[n].shape[1:]) for n in ("q", "k", "u", "w", "g", "do")}
    o, final = tri.gdn_chunk_attn(one["q"], one["k"], one["u"], one["g"], 64, W=one["w"], state=x["state"])
    assert o.shape == one["u"].shape and torch.equal(final, x["state"])
    got = tri.gdn_chunk_attn_bwd(one["q"], one["k"], one["u"], one["g"], one["do"], 64, W=one["w"], state=x["state"], dstate=x["dstate"])
    assert torch.equal(got[5], x["dstate"])
    empty, w = torch.zeros(0, 64, device="cuda", dtype=BF), torch.ones(64, device="cuda", dtype=BF)
    y, s = tri.add_rms_norm(empty, w, residual=empty)
    assert y.shape == s.shape == empty.shape
    q, scales, _ = tri.add_rms_norm_fp8(empty, w)
    assert q.shape == empty.shape and scales.shape == (0, 1)
    dx, dw = tri.add_rms_norm_bwd(empty, empty, w)
    assert dx.shape == empty.shape and not dw.any()
    state = torch.ones(3, 2, 64, 64, device="cuda")
    out = tri.gdn_step(empty.view(0, 1, 64), empty.view(0, 1, 64), torch.zeros(0, 2, 64, device="cuda", dtype=BF), None, state)
    assert out.shape == (0, 2, 64) and (state == 1).all()
