"""The fp64 statements of the head norms and the gated recurrence against differences and against each other."""
import numpy as np
import pytest

from oracle import mixer


def along(f, grads, args, seed=0, step=1e-5):
    """Each gradient along a random way against differences of f."""
    rng = np.random.default_rng(seed)
    for i, grad in grads.items():
        way = rng.standard_normal(args[i].shape)
        up, down = (f(*[a + s * way if j == i else a for j, a in enumerate(args)]) for s in (step, -step))
        assert np.isclose((up - down) / (2 * step), (grad * way).sum(), rtol=1e-7, atol=1e-7), i


@pytest.mark.parametrize("unit", [True, False])
@pytest.mark.parametrize("interleaved", [True, False])
@pytest.mark.parametrize("rot", [0, 4, 10])
def test_heads(unit, interleaved, rot):
    rng = np.random.default_rng(1)
    x, dy, w = rng.standard_normal((4, 3, 10)), rng.standard_normal((4, 3, 10)), rng.standard_normal(10)
    pos, freq = (rng.integers(-50, 50, 4), rng.random(rot // 2)) if rot else (None, None)
    f = lambda x, w: (mixer.head_norm(x, w, pos, freq, unit, interleaved, 1e-3) * dy).sum()
    dx, dw = mixer.head_norm_bwd(dy, x, w, pos, freq, unit, interleaved, 1e-3)
    along(f, {0: dx, 1: dw}, (x, w))
    y = mixer.head_norm(x, None, pos, freq, unit, interleaved, 0.0)
    assert np.allclose(np.square(y).sum(-1), 1 if unit else 10)


def test_a_rotation_adds_up():
    """Scores of rotated heads depend on the distance of their positions."""
    rng = np.random.default_rng(2)
    q, k, freq = rng.standard_normal((1, 1, 8)), rng.standard_normal((1, 1, 8)), np.array([1.0, 0.5, 0.1, 0.01])
    for inter in (True, False):
        dots = [(mixer._rotate(q, np.array([p + 7]), freq, inter, 1) * mixer._rotate(k, np.array([p]), freq, inter, 1)).sum() for p in (0, 5, 2 ** 40)]
        assert np.allclose(dots, dots[0])


@pytest.mark.parametrize("logit,mix", [(True, True), (True, False), (False, True), (False, False)])
def test_scan(logit, mix):
    rng = np.random.default_rng(3)
    x, g, S, dh, dS = rng.standard_normal((6, 5)), rng.standard_normal((6, 5)), rng.standard_normal(5), rng.standard_normal((6, 5)), rng.standard_normal(5)

    def f(x, g, S):
        h, final = mixer.gated_scan(x, g, S, logit, mix)
        return (h * dh).sum() + (final * dS).sum()

    h, final = mixer.gated_scan(x, g, S, logit, mix)
    dx, dg, dS0, _ = mixer.gated_scan_bwd(x, g, h, S, dh, dS, logit, mix)
    along(f, {0: dx, 1: dg, 2: dS0}, (x, g, S))
    first, middle = mixer.gated_scan(x[:2], g[:2], S, logit, mix)
    second, last = mixer.gated_scan(x[2:], g[2:], middle, logit, mix)
    assert np.allclose(np.concatenate([first, second]), h) and np.allclose(last, final)
    # closed form: decays from a token to the next ones
    a, rest = mixer.gates(g, logit)
    b = rest * x if mix else x
    t = 4
    assert np.allclose(h[t], a[:t + 1].prod(0) * S + sum(a[s + 1:t + 1].prod(0) * b[s] for s in range(t + 1)))


def test_nothing():
    e = np.empty((0, 3))
    h, final = mixer.gated_scan(e, e, np.ones(3), False, False)
    assert h.shape == (0, 3) and (final == 1).all()
    dx, dg, d0, _ = mixer.gated_scan_bwd(e, e, e, np.ones(3), e, np.full(3, 2.0), False, False)
    assert dx.shape == (0, 3) and (d0 == 2).all()
