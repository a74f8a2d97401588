"""Statements in fp64 of what stands between a projection and a layer's operators, from their definitions: norms of queries and keys for each head with the
rotation by position, the gated recurrence token by token, and the gradients of both.  numpy only; shares no code with the product.

Shapes: heads x, y [N, H, d], weight [d], positions [N], inv_freq [rot / 2]; one sequence's x, g, h [T, D], states [D].
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

_TURN = 2 * Fraction("3.14159265358979323846264338327950288419716939937510")


def _angles(positions, inv_freq):
    """positions times inv_freq [N, rot / 2] without whole turns, reduced exactly."""
    turns = [[float(Fraction(int(p)) * Fraction(float(f)) / _TURN % 1) for f in inv_freq] for p in positions]
    return 2 * np.pi * np.array(turns, dtype=np.float64).reshape(len(positions), len(inv_freq))


def _pairs(d, rot, interleaved):
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def _rotate(y, positions, inv_freq, interleaved, way):
    if positions is None:
        return y
    rot = 2 * len(inv_freq)
    a, b = _pairs(y.shape[-1], rot, interleaved)
    t = way * _angles(positions, inv_freq)[:, None]
    z = (y[..., a] + 1j * y[..., b]) * np.exp(1j * t)
    out = y.copy()
    out[..., a], out[..., b] = z.real, z.imag
    return out


def _length(x, unit, eps):
    sq = np.square(x).sum(-1, keepdims=True)
    return np.sqrt((sq if unit else sq / x.shape[-1]) + eps)


def head_norm(x, weight, positions, inv_freq, unit, interleaved, eps):
    y = x / _length(x, unit, eps)
    return _rotate(y if weight is None else y * weight, positions, inv_freq, interleaved, 1)


def head_norm_bwd(dy, x, weight, positions, inv_freq, unit, interleaved, eps):
    """(dx, dweight); dweight also for a weight of ones."""
    z = _rotate(dy, positions, inv_freq, interleaved, -1)
    n = _length(x, unit, eps)
    hat = x / n
    dweight = (z * hat).sum((0, 1))
    z = z if weight is None else z * weight
    dot = (z * hat).sum(-1, keepdims=True) / (1 if unit else x.shape[-1])
    return (z - hat * dot) / n, dweight


def gates(g, logit):
    """(a, 1 - a)."""
    with np.errstate(over="ignore"):
        if logit:
            return 1 / (1 + np.exp(-g)), 1 / (1 + np.exp(g))
        return np.exp(g), -np.expm1(g)


def gated_scan(x, g, state, logit, mix):
    """(h, final state)."""
    a, rest = gates(g, logit)
    h, S = np.empty_like(x), np.zeros(x.shape[1]) if state is None else state
    for t in range(len(x)):
        S = a[t] * S + (rest[t] * x[t] if mix else x[t])
        h[t] = S
    return h, S


def gated_scan_bwd(x, g, h, state, dh, dstate, logit, mix):
    """(dx, dg, dstate0, r): r the gradient of the state behind each token."""
    a, rest = gates(g, logit)
    r, R = np.empty_like(h), np.zeros(h.shape[1]) if dstate is None else dstate
    for t in reversed(range(len(h))):
        r[t] = dh[t] + R
        R = a[t] * r[t]
    before = np.concatenate([(np.zeros(h.shape[1]) if state is None else state)[None], h[:-1]])[:len(h)]
    dx = r * rest if mix else r
    dg = r * (before - x if mix else before) * a * (rest if logit else 1)
    return dx, dg, R, r
