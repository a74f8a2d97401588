"""The fp64 statements of the layer's operators (oracle/layer.py): closed forms, differences, and the delta rule through the chunk inverse."""
import numpy as np
import pytest
import torch

import oracle
from oracle import layer

RNG = np.random.default_rng


def inputs(T, H, Hk, d_k, d_v, C, seed, gate=True, delta=True):
    r = RNG(seed)
    x = dict(q=r.normal(size=(T, Hk, d_k)), k=r.normal(size=(T, Hk, d_k)) / np.sqrt(d_k), u=r.normal(size=(T, H, d_v)), w=r.normal(size=(T, H, d_k)) / d_k if delta else None,
             g=None, state=r.normal(size=(H, d_k, d_v)))
    if gate:
        rate = -0.1 * r.random((T, H))
        x["g"] = np.concatenate([rate[a:a + C].cumsum(0) for a in range(0, T, C)])
    return x


def test_without_decay_the_state_is_the_sum_of_outer_products():
    x = inputs(37, 2, 1, 8, 6, 16, 1, gate=False, delta=False)
    o, S = layer.chunk_attn(x["q"], x["k"], x["u"], None, None, 16, x["state"], 0.5)
    for h in range(2):
        scores = np.tril(x["q"][:, 0] @ x["k"][:, 0].T)
        np.testing.assert_allclose(S[h], x["state"][h] + x["k"][:, 0].T @ x["u"][:, h], rtol=1e-12)
        np.testing.assert_allclose(o[:, h], 0.5 * (x["q"][:, 0] @ x["state"][h] + scores @ x["u"][:, h]), rtol=1e-9, atol=1e-12)


@pytest.mark.parametrize("C", [16, 64])
def test_delta_rule_through_the_chunk_inverse_is_the_step_token_by_token(C):
    T, H, d_k, d_v = 100, 2, 32, 8
    r = RNG(3)
    K = torch.nn.functional.normalize(torch.tensor(r.normal(size=(1, T, H, d_k))), dim=-1).float()
    V = torch.tensor(r.normal(size=(1, T, H, d_v))).float()
    beta = torch.tensor(r.random((1, T, H))).float()
    rate = -0.1 * r.random((T, H))
    g = torch.tensor(np.concatenate([rate[a:a + C].cumsum(0) for a in range(0, T, C)]))[None].float()
    U = oracle.gdn_chunk_tri_solve(K, beta, g, V, beta, 0, C)[0]
    W = oracle.gdn_chunk_tri_solve(K, beta, g, K, beta * torch.exp(g), 0, C)[0]
    q, state = r.normal(size=(T, H, d_k)), r.normal(size=(H, d_k, d_v))
    k, v, b, gg = (x[0].numpy().astype(np.float64) for x in (K, V, beta, g))
    o, S = layer.chunk_attn(q, k, np.asarray(U), np.asarray(W), gg, C, state, 0.3)
    for t in range(T):
        ot, state = layer.step(q[t], k[t], v[t], gg[t] if t % C == 0 else gg[t] - gg[t - 1], b[t], state, 0.3)
        np.testing.assert_allclose(o[t], ot, rtol=2e-5, atol=2e-6)  # beta e^g is rounded to fp32 on its way to W
    np.testing.assert_allclose(S, state, rtol=2e-5, atol=2e-6)


@pytest.mark.parametrize("gate,delta", [(True, True), (True, False), (False, True)])
def test_gradient_against_differences(gate, delta):
    C, scale = 8, 0.7
    x = inputs(19, 4, 2, 5, 3, C, 5, gate, delta)
    r = RNG(6)
    do, dS = r.normal(size=x["u"].shape), r.normal(size=x["state"].shape)

    def loss(**kw):
        y = dict(x, **kw)
        o, S = layer.chunk_attn(y["q"], y["k"], y["u"], y["w"], y["g"], C, y["state"], scale)
        return (o * do).sum() + (S * dS).sum()

    got = dict(zip(("q", "k", "u", "w", "g", "state"), layer.chunk_attn_bwd(x["q"], x["k"], x["u"], x["w"], x["g"], C, x["state"], scale, do, dS)))
    for name, grad in got.items():
        if x[name] is None:
            continue
        for i in range(4):
            d = r.normal(size=x[name].shape)
            e = 1e-5
            diff = (loss(**{name: x[name] + e * d}) - loss(**{name: x[name] - e * d})) / (2 * e)
            # third-order remainder and the cancellation of ~1e2 in 64 bits over 2e-5
            assert abs(diff - (grad * d).sum()) <= 1e-6 * (1 + np.abs(grad * d).sum()), name


def test_norm_gradient_against_differences():
    r = RNG(8)
    s, w, dy = r.normal(size=(5, 24)), r.normal(size=24), r.normal(size=(5, 24))
    ds, dw = layer.rms_norm_bwd(dy, s, w, 1e-3)
    for i in range(4):
        a, b, e = r.normal(size=s.shape), r.normal(size=w.shape), 1e-6
        diff = ((layer.rms_norm(s + e * a, w, 1e-3) - layer.rms_norm(s - e * a, w, 1e-3)) * dy).sum() / (2 * e)
        assert abs(diff - (ds * a).sum()) <= 1e-7 * (1 + np.abs(ds * a).sum())
        diff = ((layer.rms_norm(s, w + e * b, 1e-3) - layer.rms_norm(s, w - e * b, 1e-3)) * dy).sum() / (2 * e)
        assert abs(diff - (dw * b).sum()) <= 1e-7 * (1 + np.abs(dw * b).sum())
