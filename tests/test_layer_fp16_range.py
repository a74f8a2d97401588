"""The chunk attention and its gradient in fp16 where scores and values are far from 1: two parts of 16 bits hold 22 bits of an fp32 value
only when a power of two brings it into fp16's range first.  Tolerances as in test_layer_gpu.py, which they do not depend on.

Factors are chosen so that every result in fp16 stays a normal number: one chunk's outputs are scale |q| |u| with |q|, |k| near sqrt(d_k) and 1."""
import numpy as np
import pytest
import torch

import paper_2605_21325_amd as tri
from oracle import layer
from test_layer_gpu import HF, U_OF, check_forward, close, exact, make, split, tol32

pytestmark = pytest.mark.gpu

U = U_OF[HF]


def scaled(lens, H, Hk, d_k, d_v, C, delta, with_state, seed, **by):
    x = make(lens, H, Hk, d_k, d_v, C, HF, True, delta, with_state, seed=seed)
    for name, factor in by.items():
        if x[name] is not None:
            x[name] = (x[name].float() * factor).to(x[name].dtype)
    return x


SMALL = dict(u=2.0 ** 12, do=2.0 ** 12, scale=2.0 ** -20)  # scores near 2^-19
LARGE = dict(u=2.0 ** -12, do=2.0 ** -12, scale=2.0 ** 20)  # scores far beyond 65504


@pytest.mark.parametrize("lens,H,Hk,d_k,d_v,C,delta", [([40], 2, 2, 64, 64, 64, False), ([64, 33], 2, 1, 128, 128, 64, True), ([64], 2, 2, 64, 72, 128, False), ([128], 1, 1, 128, 64, 128, True), ([16, 9], 2, 2, 64, 64, 16, True),
                                                      ([32], 1, 1, 128, 64, 32, False)])
@pytest.mark.parametrize("by", [SMALL, LARGE], ids=["small", "large"])
def test_outputs_of_scores_far_from_one(lens, H, Hk, d_k, d_v, C, delta, by):
    """No state in front and one chunk a sequence: all of an output comes through the scores."""
    by = dict(by)
    scale = by.pop("scale")
    x = scaled(lens, H, Hk, d_k, d_v, C, delta, False, 41, **by)
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, W=x["w"], scale=scale)
    check_forward(o, final, x, lens, C, scale, HF)
    zero = dict(x, u=torch.zeros_like(x["u"]))
    assert not tri.gdn_chunk_attn_varlen(x["q"], x["k"], zero["u"], x["g"], lens, C, W=x["w"], scale=scale)[0].any()


def test_zero_scores_and_zero_values_leave_the_states_outputs():
    """Nothing to add, whose power of two is the largest: the outputs are those of the state."""
    lens, C = [64], 64
    x = scaled(lens, 2, 2, 64, 64, C, False, True, 42, u=0.0)
    x["k"] = torch.zeros_like(x["k"])
    x["state"] = x["state"] * 2.0 ** 30
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, state=x["state"], scale=2.0 ** -28)
    check_forward(o, final, x, lens, C, 2.0 ** -28, HF)


def check_gradient(x, lens, C, scale):
    """Against the statement in 64 bits, with the tolerances of test_gradient in test_layer_gpu.py."""
    H, d_v = x["u"].shape[-2:]
    Hk, d_k = x["q"].shape[-2:]
    got = tri.gdn_chunk_attn_bwd_varlen(x["q"], x["k"], x["u"], x["g"], x["do"], lens, C, W=x["w"], state=x["state"], dstate=x["dstate"], scale=scale)
    t32 = tol32(d_k + d_v, C)
    state, dstate = (lambda s, h=slice(None): None if x["state"] is None else exact(x["state"][s, h])), (lambda s, h=slice(None): None if x["dstate"] is None else exact(x["dstate"][s, h]))
    for s, n in enumerate(lens):
        part = {m: split(x[m], lens, s) for m in ("q", "k", "u", "w", "g", "do")}
        one = lambda h, k: (part["q"][:, k], part["k"][:, k], part["u"][:, h], None if part["w"] is None else part["w"][:, h], part["g"][:, h], C, state(s, h), scale)
        every = slice(None)
        ref = layer.chunk_attn_bwd(*one(every, every), part["do"], dstate(s))
        a = sum(lens[:s])
        for name, mine, r, tol in zip(("dQ", "dK", "dU", "dW"), got[:4], ref[:4], (U, U, U, 2 * U)):
            if r is not None:
                assert np.abs(r).max() < 65504  # (else the inputs would be the test's mistake)
                close(mine[a:a + n], r, tol, f"{name} of sequence {s}")
        rep, size, last = H // Hk, [], []
        for h in range(H):
            args = one(slice(h, h + 1), slice(h // rep, h // rep + 1))
            r = layer.chunk_attn_bwd(*args, part["do"][:, h:h + 1], dstate(s, slice(h, h + 1)))
            size.append((np.abs(part["q"][:, h // rep] * r[0][:, 0]) + np.abs(part["k"][:, h // rep] * r[1][:, 0])).sum(-1))
            final = layer.chunk_attn(*args)[1]
            last.append(0.0 if x["dstate"] is None else np.linalg.norm(final) * np.linalg.norm(dstate(s)[h]) / np.sqrt(d_k * d_v))
        close(got[4][a:a + n].T, ref[4].T, t32, f"dg of sequence {s}", np.stack(size) + np.array(last)[:, None] + np.abs(ref[4].T))
        if x["state"] is not None:
            close(got[5][s].flatten(1), ref[5].reshape(H, -1), t32, f"gradient of the state of sequence {s}")


@pytest.mark.parametrize("lens,H,Hk,d_k,d_v,C,delta", [([40], 2, 2, 64, 64, 64, False), ([64, 33], 2, 1, 128, 128, 64, True), ([128], 1, 1, 128, 64, 128, True), ([16, 9], 2, 2, 64, 64, 16, True),
                                                      ([32], 1, 1, 128, 64, 32, False), ([150], 2, 2, 64, 72, 64, True)])
@pytest.mark.parametrize("by", [SMALL, dict(LARGE, do=2.0 ** -15, dstate=2.0 ** 5)], ids=["small", "large"])
def test_gradients_of_scores_far_from_one(lens, H, Hk, d_k, d_v, C, delta, by):
    """What arrives comes through the outputs (and large scores: little of it through the final state): dU is the scores', and what W hands on to the state."""
    by = dict(dict(u=1.0, dstate=0.0), **{n: f for n, f in by.items() if n != "u"})
    scale = by.pop("scale")
    check_gradient(scaled(lens, H, Hk, d_k, d_v, C, delta, True, 43, **by), lens, C, scale)


@pytest.mark.parametrize("lens,H,Hk,d_k,d_v,C", [([40], 2, 2, 64, 64, 64), ([150, 33], 2, 1, 128, 128, 64), ([200], 1, 1, 128, 72, 128), ([16, 9], 2, 2, 64, 264, 16), ([70], 1, 1, 96, 64, 32)])
@pytest.mark.parametrize("by", [dict(u=2.0 ** -18, state=2.0 ** -18, do=2.0 ** 6, dstate=2.0 ** 6), dict(u=2.0 ** 12, state=2.0 ** 17, dstate=2.0 ** -9, scale=2.0 ** -10)], ids=["small", "large"])
def test_gradients_of_values_far_from_one(lens, H, Hk, d_k, d_v, C, by):
    """V' = U - W S of 2^-18, and of more than 65504 (of a state in fp32)."""
    by = dict(by)
    scale = by.pop("scale", 1.0)
    x = scaled(lens, H, Hk, d_k, d_v, C, True, True, 44, **by)
    check_gradient(x, lens, C, scale)


@pytest.mark.parametrize("C,Hk,delta", [(64, 2, False), (64, 1, False), (64, 2, True), (128, 2, True), (128, 1, True)])
@pytest.mark.parametrize("d_v", [128, 200])
def test_gradients_of_columns_of_zeros_behind_large_ones(C, Hk, delta, d_v):
    """Columns of the state are taken 64 at a time; those behind the first ones hold nothing, whose power of two is the largest there is."""
    lens = [70]
    x = scaled(lens, 2, Hk, 64, d_v, C, delta, True, 45, state=2.0 ** 70, w=0.0, **(dict(k=0.0) if delta else {}))  # (with keys a dW = -dU S^T would be 2^70)
    for name in ("u", "state", "dstate", "do"):
        x[name][..., 64:] = 0
    check_gradient(x, lens, C, 2.0 ** -70)
