"""Statements in fp64 of the operators beside the chunk inverse, from their definitions, token by token: the state of linear attention with one decay
per head, its gradient taken back through the tokens, the single token's step, the norm.  numpy only; shares no code with the product.

Shapes: one sequence at a time, q, k [T, H_k, d_k], u, o [T, H, d_v], w [T, H, d_k], g [T, H] (the running sum of the log-decays, beginning again every
C tokens), states [H, d_k, d_v].
"""
from __future__ import annotations

import numpy as np


def _head(x, h, H):
    return x[:, h // (H // x.shape[1])]


def _walk(q, k, u, w, g, C, S, scale):
    """One head: every token's state, the states before the chunks by token, the values, the decays, the outputs."""
    T = q.shape[0]
    states, before, values, decays, out = [], [], np.empty_like(u), np.ones(T), np.empty_like(u)
    for t in range(T):
        if t % C == 0:
            S0 = S
        if g is not None:
            decays[t] = np.exp(g[t] if t % C == 0 else g[t] - g[t - 1])
        values[t] = u[t] if w is None else u[t] - w[t] @ S0
        S = decays[t] * S + np.outer(k[t], values[t])
        states.append(S)
        before.append(S0)
        out[t] = scale * (q[t] @ S)
    return states, before, values, decays, out, S


def chunk_attn(q, k, u, w, g, C, state, scale):
    """(o, final state)."""
    H, d_k, d_v = u.shape[1], q.shape[2], u.shape[2]
    o, final = np.zeros_like(u), np.zeros((H, d_k, d_v))
    for h in range(H):
        S = np.zeros((d_k, d_v)) if state is None else state[h]
        *_, o[:, h], final[h] = _walk(_head(q, h, H), _head(k, h, H), u[:, h], None if w is None else w[:, h], None if g is None else g[:, h], C, S, scale)
    return o, final


def chunk_attn_bwd(q, k, u, w, g, C, state, scale, do, dfinal):
    """Gradients of q, k, u, w, g and of the initial state."""
    T, H, d_k, d_v = u.shape[0], u.shape[1], q.shape[2], u.shape[2]
    dq, dk, du, dg, dstate = np.zeros_like(q), np.zeros_like(k), np.zeros_like(u), np.zeros((T, H)), np.zeros((H, d_k, d_v))
    dw = None if w is None else np.zeros_like(w)
    for h in range(H):
        hk = h // (H // q.shape[1])
        S_first = np.zeros((d_k, d_v)) if state is None else state[h]
        states, before, values, decays, _, _ = _walk(q[:, hk], k[:, hk], u[:, h], None if w is None else w[:, h], None if g is None else g[:, h], C, S_first, scale)
        dS = np.zeros((d_k, d_v)) if dfinal is None else dfinal[h].copy()
        d_before = np.zeros((d_k, d_v))  # what the chunk's values pass on to the state before it
        for t in reversed(range(T)):
            dS = dS + scale * np.outer(q[t, hk], do[t, h])
            dq[t, hk] += scale * (states[t] @ do[t, h])
            dk[t, hk] += dS @ values[t]
            du[t, h] = k[t, hk] @ dS
            if w is not None:
                dw[t, h] = -(before[t] @ du[t, h])
                d_before -= np.outer(w[t, h], du[t, h])
            step = decays[t] * (dS * (states[t - 1] if t else S_first)).sum()
            dg[t, h] += step
            if t % C:
                dg[t - 1, h] -= step
            dS = decays[t] * dS
            if t % C == 0:
                dS, d_before = dS + d_before, np.zeros((d_k, d_v))
        dstate[h] = dS
    return dq, dk, du, dw, dg, dstate


def step(q, k, v, g, beta, state, scale):
    """One sequence's token: q, k [H_k, d_k], v [H, d_v], g, beta [H] or None, state [H, d_k, d_v] -> (o, state)."""
    H = v.shape[0]
    o, out = np.empty_like(v), np.empty_like(state)
    for h in range(H):
        hk = h // (H // q.shape[0])
        S = state[h] if g is None else np.exp(g[h]) * state[h]
        x = v[h] if beta is None else beta[h] * (v[h] - k[hk] @ S)
        out[h] = S + np.outer(k[hk], x)
        o[h] = scale * (q[hk] @ out[h])
    return o, out


def rms_norm(s, weight, eps):
    return s / np.sqrt((s * s).mean(-1, keepdims=True) + eps) * weight


def rms_norm_bwd(dy, s, weight, eps):
    """(ds, dweight)."""
    ms = (s * s).mean(-1, keepdims=True) + eps
    dn = dy * weight
    return dn / np.sqrt(ms) - s * (dn * s).mean(-1, keepdims=True) / ms ** 1.5, (dy * s / np.sqrt(ms)).sum(0)
