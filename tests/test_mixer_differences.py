"""Gradients of the head norms and of the gated recurrence against differences of their forward passes, along the gradient itself (every element by its own sign, so that what one
misses is not hidden by others): of the kernels, and, on the CPU, of the fp64 statements with mistakes planted in them, which have to be seen.

Inputs are multiples of 2^-8 and ways multiples of 1/2, so that input + step way is exact.  What a difference may be off by:
  rounding    each result as in test_mixer_gpu.py, times the magnitude of its gradient, over the step
  curvature   the difference in 64 bits at this step and at a quarter of it are 15/16 of it apart; twice that
  gradient    each element as in test_mixer_gpu.py, times the way's
"""
import numpy as np
import pytest
import torch

import paper_2605_21325_amd as tri
from oracle import mixer

E, TINY = 2.0 ** -24, 2.0 ** -126
LINEAR = ("x", "state", "q_weight", "k_weight")  # a long step costs nothing
MODES = [(True, True), (True, False), (False, True), (False, False)]


def coarse(rng, *shape):
    return np.round(rng.standard_normal(shape) * 256) / 256


def f32(x):
    return np.asarray(x, dtype=np.float32).astype(np.float64)


def rounded(ref, err):
    """What a result may be off by that is rounded to fp32."""
    return E * (np.abs(ref) + err) + err + TINY


class Scan:
    """Two sequences of a recurrence, with the gradients of h and of the final states."""
    LENS, D = (9, 5), 16
    names = ("x", "g", "state")

    def __init__(self, logit, mix, seed):
        rng = np.random.default_rng(seed)
        N, self.kind = sum(self.LENS), (logit, mix)
        g = coarse(rng, N, self.D)
        self.at = dict(x=coarse(rng, N, self.D), g=g if logit else -np.abs(g) / 2, state=coarse(rng, len(self.LENS), self.D))
        self.at["g"] = np.round(self.at["g"] * 256) / 256
        self.dh, self.dstate = coarse(rng, N, self.D), coarse(rng, len(self.LENS), self.D)

    def parts(self):
        start = 0
        for s, n in enumerate(self.LENS):
            yield s, slice(start, start + n)
            start += n

    def forward(self, v):
        """(h, final) in 64 bits and what they may be off by."""
        h, off_h, final, off_f = np.empty_like(v["x"]), np.empty_like(v["x"]), np.empty_like(v["state"]), np.empty_like(v["state"])
        for s, r in self.parts():
            a, _ = mixer.gates(v["g"][r], self.kind[0])
            h[r], final[s] = mixer.gated_scan(v["x"][r], v["g"][r], v["state"][s], *self.kind)
            size, _ = mixer.gated_scan(np.abs(v["x"][r]), v["g"][r], np.abs(v["state"][s]), *self.kind)
            e = np.zeros(self.D)
            for t, (at, m) in enumerate(zip(a, size)):
                e = at * e + 16 * E * m
                off_h[r][t] = e
            off_f[s] = e
        return (h, final), (rounded(h, off_h), rounded(final, off_f))

    def ups(self):
        return self.dh, self.dstate

    def backward(self, h, mistake=None):
        """Gradients in 64 bits and what they may be off by; with a mistake."""
        v = self.at
        out, off = {n: np.empty_like(v[n]) for n in self.names}, {n: np.empty_like(v[n]) for n in self.names}
        logit, mix = self.kind
        for s, r in self.parts():
            x, g, S, dS = v["x"][r], v["g"][r], v["state"][s], self.dstate[s]
            dx, dg, d0, R = mixer.gated_scan_bwd(x, g, h[r], 0 * S if mistake == "no state" else S, self.dh[r], 0 * dS if mistake == "no dstate" else dS, logit, mix)
            _, _, m0, m = mixer.gated_scan_bwd(x, g, h[r], S, np.abs(self.dh[r]), np.abs(dS), logit, mix)
            a, rest = mixer.gates(g, logit)
            if mistake == "no 1 - a":
                dg = dg / (rest if logit else 1)
            if mistake == "no x":
                dg = dg + (R * x * a * (rest if logit else 1) if mix else 0)
            err, e = np.empty_like(m), np.zeros(self.D)
            for t in reversed(range(len(m))):
                err[t] = e + 16 * E * m[t]
                e = a[t] * err[t]
            before = np.concatenate([S[None], h[r][:-1]])
            slope, past = a * (rest if logit else 1), before - x if mix else before
            out["x"][r], out["g"][r], out["state"][s] = dx, dg, d0
            off["x"][r] = rounded(dx, err * (rest if mix else 1) + 16 * E * np.abs(dx))
            off["g"][r] = rounded(dg, slope * (err * np.abs(past) + 16 * E * np.abs(R) * (np.abs(before) + (np.abs(x) if mix else 0))))
            off["state"][s] = rounded(d0, e + 16 * E * m0)
        if mistake == "a fifth less":
            out = {n: 0.8 * x for n, x in out.items()}
        if mistake == "a hundredth more":
            out = {n: 1.01 * x for n, x in out.items()}
        return out, off


class Heads:
    """Queries and keys of a few tokens with weights and a rotation."""
    N, H, HK, D, ROT, EPS = 3, 2, 1, 16, 8, 1e-6
    names = ("q", "k", "q_weight", "k_weight")

    def __init__(self, unit, interleaved, seed):
        rng = np.random.default_rng(seed)
        self.kind = (unit, interleaved)
        self.at = dict(q=coarse(rng, self.N, self.H, self.D), k=coarse(rng, self.N, self.HK, self.D), q_weight=1 + coarse(rng, self.D) / 4, k_weight=1 + coarse(rng, self.D) / 4)
        self.at = {n: np.round(x * 256) / 256 for n, x in self.at.items()}
        self.dy = coarse(rng, self.N, self.H, self.D), coarse(rng, self.N, self.HK, self.D)
        self.positions, self.freq = rng.integers(0, 5000, self.N), f32(10000.0 ** (-np.arange(self.ROT // 2) * 2 / self.ROT))

    def lengths(self, y):
        m = np.abs(y).copy()
        a, b = mixer._pairs(self.D, self.ROT, self.kind[1])
        m[..., a] = m[..., b] = np.hypot(y[..., a], y[..., b])
        return m

    def forward(self, v):
        y = [mixer.head_norm(v[n], v[n + "_weight"], self.positions, self.freq, *self.kind, self.EPS) for n in ("q", "k")]
        return y, [rounded(x, 32 * E * self.lengths(x)) for x in y]

    def ups(self):
        return self.dy

    def backward(self, _, mistake=None):
        out, off = {}, {}
        unit, interleaved = self.kind
        for n, dy in zip(("q", "k"), self.dy):
            v, w = self.at[n], self.at[n + "_weight"]
            z = mixer._rotate(dy, self.positions, self.freq, interleaved, 1 if mistake == "turned the other way" else -1)
            length = mixer._length(v, unit, self.EPS)
            hat, m = v / length, 1 if unit else self.D
            out[n + "_weight"] = (z[1:] * hat[1:] if mistake == "weights without a token" else z * hat).sum((0, 1))
            out[n] = (z * w - (0 if mistake == "norm as a constant" else hat * (z * w * hat).sum(-1, keepdims=True) / m)) / length
            zl, ahat = self.lengths(z), np.abs(hat)
            size = (zl * np.abs(w) + ahat * (zl * np.abs(w) * ahat).sum(-1, keepdims=True) / m) / length
            off[n] = rounded(out[n], 64 * E * size)
            off[n + "_weight"] = rounded(out[n + "_weight"], (v.shape[0] * v.shape[1] + 64) * E * (zl * ahat).sum((0, 1)))
        if mistake == "a hundredth more":
            out = {n: 1.01 * x for n, x in out.items()}
        return out, off


def agrees(case, forward, grads, offs, name):
    """Whether a gradient is the slope of `forward` (results as they come, of inputs by name) along itself, and along ways without the half of its elements."""
    return max(ratios(case, forward, grads, offs, name)) <= 1


def ratios(case, forward, grads, offs, name):
    rng = np.random.default_rng(1)
    grad, h = grads[name], 2.0 ** -2 if name in LINEAR else 2.0 ** -8
    for i in range(6):
        way = np.where(grad < 0, -1.0, 1.0) * rng.choice([0.5, 1.0, 1.5, 2.0], grad.shape) * (rng.random(grad.shape) < (1 if i == 0 else 0.5))

        def losses(step, results):
            there = [results(dict(case.at, **{name: case.at[name] + s * step * way})) for s in (1, -1)]
            up, down = (sum((y * d).sum() for y, d in zip(ys, case.ups())) for ys in there)
            return (up - down) / (2 * step)

        exact = lambda v: case.forward(v)[0]
        curvature = 2 * abs(losses(h, exact) - losses(h / 4, exact))
        rounding = max(sum((o * np.abs(d)).sum() for o, d in zip(case.forward(dict(case.at, **{name: case.at[name] + s * h * way}))[1], case.ups())) for s in (1, -1)) / h
        yield abs(losses(h, forward) - (grad * way).sum()) / (curvature + rounding + (offs[name] * np.abs(way)).sum())


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("logit,mix", MODES)
def test_mistakes_in_the_recurrence_are_seen(logit, mix, seed):
    case = Scan(logit, mix, seed)
    forward = lambda v: [f32(y) for y in case.forward(v)[0]]
    h = f32(case.forward(case.at)[0][0])
    right, offs = case.backward(h)
    for name in case.names:
        assert agrees(case, forward, {n: f32(x) for n, x in right.items()}, offs, name), name
    mistakes = [("no state", "g"), ("no dstate", "x"), ("no dstate", "g"), ("no dstate", "state")] + [(m, n) for m in ("a fifth less", "a hundredth more") for n in case.names]
    mistakes += [("no 1 - a", "g")] * logit + [("no x", "g")] * mix
    for mistake, name in mistakes:
        assert not agrees(case, forward, case.backward(h, mistake)[0], offs, name), (mistake, name)


@pytest.mark.parametrize("seed", range(4))
@pytest.mark.parametrize("unit,interleaved", [(False, False), (False, True), (True, False), (True, True)])
def test_mistakes_in_the_norms_are_seen(unit, interleaved, seed):
    case = Heads(unit, interleaved, seed)
    forward = lambda v: [f32(y) for y in case.forward(v)[0]]
    right, offs = case.backward(None)
    for name in case.names:
        assert agrees(case, forward, {n: f32(x) for n, x in right.items()}, offs, name), name
    for mistake, names in [("turned the other way", case.names), ("norm as a constant", ("q", "k")), ("weights without a token", ("q_weight", "k_weight")), ("a hundredth more", case.names)]:
        wrong = case.backward(None, mistake)[0]
        for name in names:
            assert not agrees(case, forward, wrong, offs, name), (mistake, name)


def on_gpu(x, dtype=torch.float32):
    return torch.from_numpy(np.ascontiguousarray(x)).to("cuda", dtype)


def back(x):
    return x.double().cpu().numpy()


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(2))
@pytest.mark.parametrize("logit,mix", MODES)
def test_recurrence(logit, mix, seed):
    case = Scan(logit, mix, seed)
    kind = dict(logit=logit, mix=mix)
    forward = lambda v: [back(y) for y in tri.gated_scan_varlen(on_gpu(v["x"]), on_gpu(v["g"]), list(case.LENS), on_gpu(v["state"]), **kind)]
    x, g, state = (on_gpu(case.at[n]) for n in case.names)
    h, _ = tri.gated_scan_varlen(x, g, list(case.LENS), state, **kind)
    got = tri.gated_scan_bwd_varlen(x, g, h, on_gpu(case.dh), list(case.LENS), state, on_gpu(case.dstate), **kind)
    offs = case.backward(back(h))[1]
    for name in case.names:
        assert agrees(case, forward, dict(zip(case.names, map(back, got))), offs, name), name


@pytest.mark.gpu
@pytest.mark.parametrize("seed", range(2))
@pytest.mark.parametrize("unit,interleaved", [(False, False), (False, True), (True, False), (True, True)])
def test_norms(unit, interleaved, seed):
    case = Heads(unit, interleaved, seed)
    rest = dict(positions=on_gpu(case.positions, torch.int32), inv_freq=on_gpu(case.freq), unit=unit, interleaved=interleaved, eps=case.EPS)
    forward = lambda v: [back(y) for y in tri.qk_norm_rope(*(on_gpu(v[n]) for n in case.names), **rest)]
    got = tri.qk_norm_rope_bwd(*(on_gpu(d) for d in case.dy), *(on_gpu(case.at[n]) for n in case.names), **rest)
    offs = case.backward(None)[1]
    for name in case.names:
        assert agrees(case, forward, dict(zip(case.names, map(back, got))), offs, name), name
