"""Head norms with the rotation and the gated recurrence on the GPU against the fp64 statements of oracle/mixer.py.

Tolerances.  u is half a step of the result's type (bf16 2^-8, fp16 2^-11, fp32 2^-24): one rounding on the way out.  Everything before it is fp32, E = 2^-24:
  heads      the norm: a sum of d squares in a tree (fewer than 16 roundings), a root and a quotient; then three products, and in a rotation a sum and cos and sin of an angle
             that is off by 2 pi 2^-25 turns and their own 2 E: fewer than 32 E of the pair's length.
  weights    sums over tokens and heads of such products in any order: (terms + 32) E of the sum of their magnitudes.
  scan       a decay is off by at most 4 steps (8 E), a token's input too; each of them moves the states behind it by at most 8 E of what it carries, and products of decays
             and joins of segments round as often again: err_t = a_t err_(t-1) + 16 E m_t with m the recurrence of the magnitudes.
"""
import numpy as np
import pytest
import torch

import paper_2605_21325_amd as tri
from oracle import mixer

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
BF, HF, F = torch.bfloat16, torch.float16, torch.float32
U = {BF: 2.0 ** -8, HF: 2.0 ** -11, F: 2.0 ** -24}
TINY = {BF: 2.0 ** -133, HF: 2.0 ** -24, F: 2.0 ** -126}  # a step of the smallest numbers (fp32: they may be taken as zeros)
E = 2.0 ** -24


def exact(x):
    if x is None:
        return None
    x = x.detach().cpu()
    return (x.double() if x.is_floating_point() else x).numpy()


def within(got, ref, tol, dtype, what):
    """Element by element: one rounding of `dtype` and `tol`."""
    got = exact(got)
    assert got.shape == ref.shape, what
    allowed = U[dtype] * (np.abs(ref) + tol) + tol + TINY[dtype]
    over = np.abs(got - ref) / allowed
    assert not np.isnan(over).any(), f"{what}: not a number"
    assert over.size == 0 or over.max() <= 1, f"{what}: {over.max():.2f} of the tolerance at {np.unravel_index(over.argmax(), over.shape)}"


def rand(gen, *shape):
    return torch.randn(*shape, generator=gen, device=DEV)


def generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


# ---------------------------------------------------------------- heads

def make_heads(N, H, Hk, d, rot, weight, dtype, seed=0, joint=False, first=100, pos=torch.int32):
    gen = generator(seed)
    if joint:
        both = rand(gen, N, (H + 2 * Hk) * d + joint).to(dtype)
        q, k = both[:, :H * d].view(N, H, d), both[:, H * d:(H + Hk) * d].view(N, Hk, d)
    else:
        q, k = rand(gen, N, H, d).to(dtype), rand(gen, N, Hk, d).to(dtype)
    x = dict(q=q, k=k if Hk else None, q_weight=(1 + 0.2 * rand(gen, d)).to(dtype) if weight else None, k_weight=(1 + 0.2 * rand(gen, d)).to(dtype) if weight and Hk else None)
    x["positions"] = (first + torch.randint(0, 5000, (N,), generator=gen, device=DEV)).to(pos) if rot else None
    x["inv_freq"] = (10000.0 ** (-torch.arange(rot // 2, device=DEV, dtype=torch.float64) * 2 / rot)).float() if rot else None
    up = dict(dq_out=rand(gen, N, H, d).to(dtype), dk_out=rand(gen, N, Hk, d).to(dtype) if Hk else None)
    return x, up


def lengths_of_pairs(y, rot, interleaved):
    """[N, H, d]: an element's magnitude, or its pair's length."""
    m = np.abs(y).copy()
    if rot:
        a, b = mixer._pairs(y.shape[-1], rot, interleaved)
        m[..., a] = m[..., b] = np.hypot(y[..., a], y[..., b])
    return m


def check_heads(x, got, unit, interleaved, eps=1e-6):
    for n, y in (("q", got[0]), ("k", got[1])):
        if x[n] is None:
            assert y is None
            continue
        ref = mixer.head_norm(exact(x[n]), exact(x[n + "_weight"]), exact(x["positions"]), exact(x["inv_freq"]), unit, interleaved, eps)
        rot = 0 if x["inv_freq"] is None else 2 * len(x["inv_freq"])
        within(y, ref, 32 * E * lengths_of_pairs(ref, rot, interleaved), x[n].dtype, n)


def check_heads_bwd(x, up, got, unit, interleaved, eps=1e-6):
    for n, dx, dw in (("q", got[0], got[2]), ("k", got[1], got[3])):
        if x[n] is None:
            assert dx is None and dw is None
            continue
        v, w, dy = exact(x[n]), exact(x[n + "_weight"]), exact(up[f"d{n}_out"])
        pos, freq = exact(x["positions"]), exact(x["inv_freq"])
        ref, dweight = mixer.head_norm_bwd(dy, v, w, pos, freq, unit, interleaved, eps)
        rot = 0 if freq is None else 2 * len(freq)
        z = lengths_of_pairs(mixer._rotate(dy, pos, freq, interleaved, -1), rot, interleaved)
        hat, length = np.abs(v) / mixer._length(v, unit, eps), mixer._length(v, unit, eps)
        zw = z if w is None else z * np.abs(w)
        size = (zw + hat * (zw * hat).sum(-1, keepdims=True) / (1 if unit else v.shape[-1])) / length
        within(dx, ref, 64 * E * size, x[n].dtype, "d" + n)
        if w is None:
            assert dw is None
        else:
            assert dw.dtype == F
            within(dw, dweight, (v.shape[0] * v.shape[1] + 64) * E * (z * hat).sum((0, 1)), F, f"d{n}_weight")


HEADS = [
    # N, H, Hk, d, rot, interleaved, unit, weight, dtype
    (1, 16, 4, 128, 128, False, False, True, BF),
    (7, 4, 4, 64, 0, False, True, False, HF),
    (33, 3, 1, 80, 32, True, False, True, BF),
    (5, 5, 5, 96, 96, False, False, False, F),
    (19, 2, 2, 256, 128, True, True, True, BF),
    (10, 8, 2, 192, 192, True, False, True, HF),
    (3, 1, 0, 512, 512, False, False, True, BF),
    (4, 2, 1, 34, 16, False, False, True, F),
    (6, 3, 3, 1, 0, False, False, True, BF),
    (6, 3, 3, 2, 2, False, True, False, F),
    (9, 7, 1, 77, 38, False, False, True, HF),
    (9, 2, 2, 300, 150, True, False, True, F),
    (65, 40, 8, 128, 64, False, False, True, BF),
    (130, 5, 3, 128, 128, True, False, True, F),
    (40, 33, 2, 72, 72, False, False, True, BF),
    (40, 12, 12, 32, 16, False, True, False, BF),
    (12, 4, 4, 128, 6, False, False, True, BF),
    (12, 4, 4, 128, 6, True, False, True, HF),
    (300, 6, 2, 112, 0, False, False, True, BF),
]


@pytest.mark.parametrize("case", range(len(HEADS)))
@pytest.mark.parametrize("joint", [0, 8, 1])
def test_heads(case, joint):
    N, H, Hk, d, rot, inter, unit, weight, dtype = HEADS[case]
    x, up = make_heads(N, H, Hk, d, rot, weight, dtype, seed=case, joint=joint)
    check_heads(x, tri.qk_norm_rope(**x, unit=unit, interleaved=inter), unit, inter)
    check_heads_bwd(x, up, tri.qk_norm_rope_bwd(**up, **x, unit=unit, interleaved=inter), unit, inter)


@pytest.mark.parametrize("pos,first", [(torch.int32, 2 ** 31 - 6000), (torch.int64, 2 ** 52), (torch.int32, -9000), (torch.int64, -2 ** 33)])
def test_angles_of_far_positions(pos, first):
    x, up = make_heads(20, 2, 2, 64, 64, True, F, first=first, pos=pos)
    check_heads(x, tri.qk_norm_rope(**x), False, False)
    check_heads_bwd(x, up, tri.qk_norm_rope_bwd(**up, **x), False, False)


@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("d", [128, 90])
def test_heads_in_place_and_into_columns(dtype, d):
    x, up = make_heads(21, 6, 2, d, 32, True, dtype)
    want, back = tri.qk_norm_rope(**x), tri.qk_norm_rope_bwd(**up, **x)
    wide = torch.full((21, 10 * d + 8), 7.0, dtype=dtype, device=DEV)
    q, k = wide[:, :6 * d].view(21, 6, d), wide[:, 6 * d:8 * d].view(21, 2, d)
    got = tri.qk_norm_rope(**x, q_out=q, k_out=k)
    assert got[0] is q and torch.equal(q, want[0]) and torch.equal(k, want[1]) and (wide[:, 8 * d:] == 7).all()
    got = tri.qk_norm_rope_bwd(**up, **x, dq=q, dk=k)
    assert torch.equal(q, back[0]) and torch.equal(k, back[1]) and (wide[:, 8 * d:] == 7).all()
    q.copy_(x["q"]), k.copy_(x["k"])
    y = dict(x, q=q, k=k)
    tri.qk_norm_rope(**y, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and (wide[:, 8 * d:] == 7).all()
    dq, dk = up["dq_out"].clone(), up["dk_out"].clone()
    tri.qk_norm_rope_bwd(dq, dk, **x, dq=dq, dk=dk)
    assert torch.equal(dq, back[0]) and torch.equal(dk, back[1])


@pytest.mark.parametrize("d,dtype", [(128, BF), (128, F), (65, HF)])
def test_heads_that_are_not_finite_or_nothing(d, dtype):
    x, up = make_heads(6, 4, 4, d, 0, True, dtype)
    clean = tri.qk_norm_rope(**x)
    x["q"][1, 2, 3], x["k"][2, 0, 1], x["q"][4, 3] = torch.nan, torch.inf, 0
    q, k = tri.qk_norm_rope(**x)
    assert q[1, 2].isnan().all() and (q[4, 3] == 0).all()
    inf = torch.zeros(d, dtype=torch.bool, device=DEV)
    inf[1] = True
    assert k[2, 0][inf].isnan().all() and (k[2, 0][~inf] == 0).all()
    keep_q, keep_k = torch.ones(6, 4, dtype=torch.bool, device=DEV), torch.ones(6, 4, dtype=torch.bool, device=DEV)
    keep_q[1, 2] = keep_q[4, 3] = keep_k[2, 0] = False
    assert torch.equal(q[keep_q], clean[0][keep_q]) and torch.equal(k[keep_k], clean[1][keep_k])
    u, _ = tri.qk_norm_rope(x["q"][4:5].contiguous(), None, unit=True)
    assert (u[0, 3] == 0).all()


def test_heads_of_no_tokens():
    x, up = make_heads(0, 4, 2, 64, 64, True, BF)
    q, k = tri.qk_norm_rope(**x)
    assert q.shape == (0, 4, 64) and k.shape == (0, 2, 64)
    dq, dk, dqw, dkw = tri.qk_norm_rope_bwd(**up, **x)
    assert dq.shape == (0, 4, 64) and (dqw == 0).all() and (dkw == 0).all()


def test_heads_gradient_against_differences():
    x, up = make_heads(3, 2, 1, 16, 8, True, F, first=0)

    def loss(v):
        y = tri.qk_norm_rope(**v)
        return sum((exact(a) * exact(b)).sum() for a, b in zip(y, (up["dq_out"], up["dk_out"])))

    got = dict(zip(("q", "k", "q_weight", "k_weight"), tri.qk_norm_rope_bwd(**up, **x)))
    gen = generator(5)
    for name, grad in got.items():
        way = rand(gen, *x[name].shape)
        step = 2.0 ** -7
        there = (loss(dict(x, **{name: x[name] + step * way})) - loss(dict(x, **{name: x[name] - step * way}))) / (2 * step)
        along = (exact(grad) * exact(way)).sum()
        size = (np.abs(exact(grad)) * np.abs(exact(way))).sum()
        # the third derivative's part, step^2 of a smooth function's scale, and the results' rounding over the step
        assert abs(there - along) <= size * (8 * step ** 2 + 200 * 32 * E / step), name


# ---------------------------------------------------------------- scan

def make_scan(lens, D, dtype, gtype, logit, state=True, seed=0, joint=0, slow=7.0, packed=True):
    gen = generator(seed)
    total = sum(lens)
    hold = slow * torch.rand(D, generator=gen, device=DEV)
    g = rand(gen, total, D) + hold if logit else -torch.nn.functional.softplus(rand(gen, total, D)) * torch.exp(-hold)
    x = rand(gen, total, D)
    if joint:
        both = torch.cat([x, g, rand(gen, total, joint)], 1).to(dtype)
        x, g = both[:, :D], both[:, D:2 * D]
    else:
        x, g = x.to(dtype), g.to(gtype)
    shape = lambda t: t if packed else t.view(len(lens), lens[0], *t.shape[1:]) if not joint else t.unflatten(0, (len(lens), lens[0]))
    v = dict(x=shape(x), g=shape(g), state=rand(gen, len(lens), D) if state else None)
    up = dict(dh=shape(rand(gen, total, D).to(dtype)), dstate=rand(gen, len(lens), D) if state else None)
    return v, up


def sequences(lens, *tensors):
    at = 0
    for n in lens:
        yield tuple(None if t is None else exact(t.reshape(-1, t.shape[-1])[at:at + n]) for t in tensors)
        at += n


def running(size, a):
    """err_t = a_t err_(t-1) + 16 E size_t."""
    err, e = np.empty_like(size), np.zeros(size.shape[1])
    for t in range(len(size)):
        e = np.minimum(a[t], 1e30) * e + 16 * E * size[t]
        err[t] = e
    return err, e


def check_scan(lens, v, got, logit, mix):
    dtype = v["x"].dtype
    h, final = got
    assert h.dtype == dtype and final.dtype == F and h.shape == v["x"].shape
    for s, (x, g, y) in enumerate(sequences(lens, v["x"], v["g"], h)):
        S = None if v["state"] is None else exact(v["state"][s])
        ref, last = mixer.gated_scan(x, g, S, logit, mix)
        size, msize = mixer.gated_scan(np.abs(x), g, None if S is None else np.abs(S), logit, mix)
        err, e = running(size, mixer.gates(g, logit)[0])
        within(torch.from_numpy(y), ref, err, dtype, f"h of sequence {s}")
        within(final[s], last, e, F, f"final state of sequence {s}")


def check_scan_bwd(lens, v, h, up, got, logit, mix):
    dtype, gtype = v["x"].dtype, v["g"].dtype
    dx, dg, dstate0 = got
    assert dx.dtype == dtype and dg.dtype == gtype and dx.shape == v["x"].shape and dg.shape == v["x"].shape and (dstate0 is None) == (v["state"] is None)
    for s, (x, g, y, dy, ox, og) in enumerate(sequences(lens, v["x"], v["g"], h, up["dh"], dx, dg)):
        S, dS = (None if t is None else exact(t[s]) for t in (v["state"], up["dstate"]))
        rx, rg, r0, r = mixer.gated_scan_bwd(x, g, y, S, dy, dS, logit, mix)
        a, rest = mixer.gates(g, logit)
        _, _, m0, m = mixer.gated_scan_bwd(x, g, y, S, np.abs(dy), None if dS is None else np.abs(dS), logit, mix)
        err, e = np.empty_like(m), np.zeros(m.shape[1])
        for t in reversed(range(len(m))):
            e = e + 16 * E * m[t]
            err[t] = e
            e = a[t] * e
        e = e + 16 * E * m0
        before = np.concatenate([(np.zeros(g.shape[1]) if S is None else S)[None], y[:-1]])[:len(y)]
        past = before - x if mix else before
        slope = a * (rest if logit else 1)
        within(torch.from_numpy(ox), rx, err * (rest if mix else 1) + 16 * E * np.abs(rx), dtype, f"dx of sequence {s}")
        within(torch.from_numpy(og), rg, slope * (err * np.abs(past) + 16 * E * np.abs(r) * (np.abs(before) + (np.abs(x) if mix else 0))), gtype, f"dg of sequence {s}")
        if dstate0 is not None:
            within(dstate0[s], r0, e, F, f"dstate0 of sequence {s}")


SCAN = [
    # lens, D, dtype, gtype, logit, mix, state
    ([1], 64, BF, BF, True, True, False),
    ([64], 128, HF, HF, False, False, True),
    ([5, 0, 1, 63, 64, 65, 0, 130], 72, BF, BF, True, True, True),
    ([0, 0, 3], 33, BF, F, False, True, True),
    ([700], 130, BF, BF, True, False, True),
    ([1, 1, 1, 1, 1, 1, 1, 1, 1, 1], 256, HF, F, False, False, True),
    ([257, 258], 1, F, F, True, True, False),
    ([511, 2, 513], 200, F, F, False, True, True),
    ([2000], 24, F, F, False, False, False),
    ([300, 0], 1000, HF, F, False, False, True),
    ([33] * 20, 66, BF, BF, True, True, True),
    ([128, 128, 128], 512, BF, F, True, True, False),
    ([1500, 1, 1200], 192, BF, BF, False, False, True),
    ([4100], 320, F, F, True, True, True),
]


@pytest.mark.parametrize("case", range(len(SCAN)))
@pytest.mark.parametrize("joint", [0, 1, 8])
def test_scan(case, joint):
    lens, D, dtype, gtype, logit, mix, state = SCAN[case]
    if joint and gtype != dtype:
        pytest.skip("columns of one projection have one type")
    v, up = make_scan(lens, D, dtype, gtype, logit, state, seed=case, joint=joint)
    got = tri.gated_scan_varlen(v["x"], v["g"], lens, v["state"], logit=logit, mix=mix)
    check_scan(lens, v, got, logit, mix)
    back = tri.gated_scan_bwd_varlen(v["x"], v["g"], got[0], up["dh"], lens, v["state"], up["dstate"], logit=logit, mix=mix)
    check_scan_bwd(lens, v, got[0], up, back, logit, mix)


@pytest.mark.parametrize("B,T,D,dtype,gtype", [(1, 1, 2048, BF, BF), (3, 100, 96, BF, BF), (2, 64, 130, HF, F), (5, 0, 64, BF, BF), (70, 3, 40, F, F), (2, 900, 64, BF, F), (4, 256, 128, HF, HF),
                                              (40, 63, 512, BF, BF), (9, 33, 1000, HF, F), (300, 17, 256, BF, F), (7, 48, 66, F, F), (3, 65, 256, HF, HF)])
@pytest.mark.parametrize("logit,mix", [(True, True), (True, False), (False, True), (False, False)])
def test_scan_of_sequences_of_one_length(B, T, D, dtype, gtype, logit, mix):
    for state in (True, False):
        v, up = make_scan([T] * B, D, dtype, gtype, logit, state, packed=False)
        got = tri.gated_scan(**v, logit=logit, mix=mix)
        check_scan([T] * B, v, got, logit, mix)
        back = tri.gated_scan_bwd(v["x"] if mix else None, v["g"], got[0], up["dh"], v["state"], up["dstate"], logit=logit, mix=mix)
        check_scan_bwd([T] * B, v, got[0], up, back, logit, mix)


def test_scan_forgets_and_holds():
    """Decays of 0 and 1, logits far out: what is behind a token that begins anew does not depend on what was before it, infinities included."""
    v, _ = make_scan([400], 70, F, F, False)
    v["g"][200] = -torch.inf
    got = tri.gated_scan_varlen(**v, seqlens=[400])
    alone = tri.gated_scan_varlen(v["x"][200:].contiguous(), v["g"][200:].contiguous(), [200])
    check_scan([200], dict(x=v["x"][200:], g=v["g"][200:], state=None), (got[0][200:], got[1]), False, False)
    check_scan([200], dict(x=v["x"][200:], g=v["g"][200:], state=None), alone, False, False)
    for far, a in ((200.0, 1.0), (-200.0, 0.0), (torch.inf, 1.0), (-torch.inf, 0.0)):
        g = torch.full((1, 5, 64), far, device=DEV)
        x, s = torch.randn(1, 5, 64, device=DEV), torch.randn(1, 64, device=DEV)
        h, final = tri.gated_scan(x, g, s, logit=True, mix=True)
        assert torch.equal(h, s[:, None].expand_as(h) if a else x) and torch.equal(final, h[:, -1])
        dx, dg, ds = tri.gated_scan_bwd(x, g, h, x, s, logit=True, mix=True)
        assert (dg == 0).all() and (dx == (0 if a else x)).all()
    zero = torch.zeros(1, 300, 64, device=DEV)
    h, final = tri.gated_scan(torch.ones(1, 300, 64, device=DEV), zero)
    assert torch.equal(h[0, :, 5], torch.arange(1, 301, device=DEV).float()) and (final == 300).all()


def test_scan_decays_above_one():
    v, up = make_scan([40, 90], 64, F, F, False)
    v["g"] = 0.2 * torch.randn(130, 64, device=DEV)
    got = tri.gated_scan_varlen(**v, seqlens=[40, 90], mix=False)
    check_scan([40, 90], v, got, False, False)
    check_scan_bwd([40, 90], v, got[0], up, tri.gated_scan_bwd_varlen(v["x"], v["g"], got[0], up["dh"], [40, 90], v["state"], up["dstate"]), False, False)


@pytest.mark.parametrize("dtype,gtype", [(F, F), (BF, F), (BF, BF), (HF, HF)])
def test_scan_decays_beyond_the_range(dtype, gtype):
    """e^g is infinite from 88.73 on, and a finite state becomes infinite by it, not NaN; what comes to nothing is nothing."""
    g = torch.tensor([88.5, -88.5, -87, -60, -30, 45, 89.0, 89.25, 90, 91.5, 95, 100, 127, 300, 1000, 60000, float("inf"), -89, -105, -150, -60000, float("-inf")], device=DEV).to(gtype).view(1, 1, -1)
    x = torch.zeros(g.shape, dtype=dtype, device=DEV)
    _, last = tri.gated_scan(x, g, state=torch.ones(1, g.shape[-1], device=DEV))
    got = exact(last)
    with np.errstate(over="ignore"):
        ref = np.exp(exact(g)).reshape(got.shape)
        ref32 = ref.astype(np.float32).astype(np.float64)
    assert (np.isinf(got) == np.isinf(ref32)).all()
    finite = np.isfinite(ref32)
    assert (np.abs(got[finite] - ref[finite]) <= 16 * E * ref[finite] + TINY[F]).all()
    pool = torch.ones(1, g.shape[-1], device=DEV)
    tri.gated_scan_step(x[0], g[0], pool)
    assert torch.equal(pool, last)


@pytest.mark.parametrize("T", [50, 900])
def test_what_is_not_finite_stays_in_its_sequence_and_channel(T):
    v, _ = make_scan([T, T, T], 64, BF, BF, True)
    clean = tri.gated_scan_varlen(**v, seqlens=[T] * 3, logit=True, mix=True)
    v["x"][T + T // 2, 7], v["state"][0, 3] = torch.nan, torch.inf
    h, final = tri.gated_scan_varlen(**v, seqlens=[T] * 3, logit=True, mix=True)
    hit = torch.zeros(3 * T, 64, dtype=torch.bool, device=DEV)
    hit[T + T // 2:2 * T, 7] = hit[:T, 3] = True
    assert not h[hit].isfinite().any() and torch.equal(h[~hit], clean[0][~hit])
    assert final[1, 7].isnan() and final[0, 3].isinf() and torch.equal(final[2], clean[1][2])


def test_final_state_upon_the_initial_one():
    lens = [300, 0, 1, 1000]
    v, up = make_scan(lens, 96, BF, BF, True)
    want, final = tri.gated_scan_varlen(**v, seqlens=lens, logit=True)
    state = v["state"].clone()
    got, same = tri.gated_scan_varlen(v["x"], v["g"], lens, state, logit=True, final_state=state)
    assert same is state and torch.equal(state, final) and torch.equal(got, want)
    assert torch.equal(final[1], v["state"][1])


def test_scan_into_columns():
    v, up = make_scan([130, 70], 48, BF, BF, True)
    h, final = tri.gated_scan_varlen(**v, seqlens=[130, 70], logit=True, mix=True)
    wide = torch.full((200, 2 * 48 + 2), 7.0, dtype=BF, device=DEV)
    tri.gated_scan_varlen(**v, seqlens=[130, 70], logit=True, mix=True, h=wide[:, 48:96])
    assert torch.equal(wide[:, 48:96], h) and (wide[:, :48] == 7).all() and (wide[:, 96:] == 7).all()
    dx, dg, _ = tri.gated_scan_bwd_varlen(v["x"], v["g"], wide[:, 48:96], up["dh"], [130, 70], v["state"], logit=True, mix=True)
    both = torch.full((200, 2 * 48 + 2), 7.0, dtype=BF, device=DEV)
    tri.gated_scan_bwd_varlen(v["x"], v["g"], h, up["dh"], [130, 70], v["state"], logit=True, mix=True, dx=both[:, :48], dg=both[:, 48:96])
    assert torch.equal(both[:, :48], dx) and torch.equal(both[:, 48:96], dg) and (both[:, 96:] == 7).all()


@pytest.mark.parametrize("logit,mix", [(True, True), (True, False), (False, True), (False, False)])
def test_scan_gradient_against_differences(logit, mix):
    lens = [9, 5]
    v, up = make_scan(lens, 8, F, F, logit, slow=1.0)

    def loss(w):
        h, final = tri.gated_scan_varlen(**w, seqlens=lens, logit=logit, mix=mix)
        return (exact(h) * exact(up["dh"])).sum() + (exact(final) * exact(up["dstate"])).sum()

    h, _ = tri.gated_scan_varlen(**v, seqlens=lens, logit=logit, mix=mix)
    got = dict(zip(("x", "g", "state"), tri.gated_scan_bwd_varlen(v["x"], v["g"], h, up["dh"], lens, v["state"], up["dstate"], logit=logit, mix=mix)))
    gen = generator(5)
    for name, grad in got.items():
        way = rand(gen, *v[name].shape)
        step = 2.0 ** -7
        there = (loss(dict(v, **{name: v[name] + step * way})) - loss(dict(v, **{name: v[name] - step * way}))) / (2 * step)
        along, size = (exact(grad) * exact(way)).sum(), (np.abs(exact(grad)) * np.abs(exact(way))).sum()
        # the third derivative's part (up to 14 decays in a product, each stretched by 1 + 3 step), and the results' rounding over the step
        assert abs(there - along) <= size * (14 ** 2 * step ** 2 + 200 * 32 * E / step), name


@pytest.mark.parametrize("D,dtype,gtype", [(2048, BF, BF), (100, HF, F), (33, F, F), (66, BF, F), (8192, HF, HF)])
@pytest.mark.parametrize("logit,mix", [(True, True), (False, True), (False, False)])
def test_scan_step(D, dtype, gtype, logit, mix):
    B = 9
    v, _ = make_scan([B], D, dtype, gtype, logit)
    pool = rand(generator(3), 12, D)
    slots = torch.tensor([3, 0, -1, 11, 12, 5, 7, 2 ** 30, 1], dtype=torch.int32, device=DEV)
    before = pool.clone()
    h = tri.gated_scan_step(v["x"], v["g"], pool, slots, logit=logit, mix=mix)
    held = set(range(12))
    for b, s in enumerate(slots.tolist()):
        if not 0 <= s < 12:
            assert (h[b] == 0).all()
            continue
        held.discard(s)
        check_scan([1], dict(x=v["x"][b:b + 1], g=v["g"][b:b + 1], state=before[s:s + 1]), (h[b:b + 1], pool[s:s + 1]), logit, mix)
    assert all(torch.equal(pool[s], before[s]) for s in held)
    own = before[:B].clone()
    h = tri.gated_scan_step(v["x"], v["g"], own, logit=logit, mix=mix)
    check_scan([1] * B, dict(v, state=before[:B]), (h, own), logit, mix)


def test_tokens_one_by_one_end_where_the_prompt_ends():
    v, _ = make_scan([40], 96, BF, BF, True)
    h, final = tri.gated_scan_varlen(**v, seqlens=[40], logit=True, mix=True)
    state = v["state"].clone()
    for t in range(40):
        y = tri.gated_scan_step(v["x"][t:t + 1], v["g"][t:t + 1], state, logit=True, mix=True)
    S = exact(v["state"][0])
    size, _ = mixer.gated_scan(np.abs(exact(v["x"])), exact(v["g"]), np.abs(S), True, True)
    _, e = running(size, mixer.gates(exact(v["g"]), True)[0])
    assert (np.abs(exact(state[0]) - exact(final[0])) <= 2 * e).all()
    within(y[0], exact(final[0]), 2 * e, BF, "h")


# ---------------------------------------------------------------- both, as they are used

def test_from_a_projection_to_the_layer_and_on_to_a_token():
    """The recurrence mixes a projection's columns, heads are normed where they stand, the delta rule takes them; a prompt and one token against the prompt with it."""
    B, T, H, d, C = 2, 150, 2, 64, 64
    gen = generator(1)
    D = 3 * H * d
    proj, gate = rand(gen, B, T + 1, D).to(BF), (rand(gen, B, T + 1, D) + 2).to(BF)
    beta, r = torch.sigmoid(rand(gen, B, T + 1, H)), -0.1 * torch.rand(B, T + 1, H, generator=gen, device=DEV)

    def heads(y):
        q, k, v = y.unflatten(-1, (3, H, d)).unbind(-3)
        q, k = tri.qk_norm_rope(q, k, unit=True)
        return q, k, v.contiguous()

    def prompt(n):
        y, mixed = tri.gated_scan(proj[:, :n], gate[:, :n], logit=True, mix=True) if n == T + 1 else tri.gated_scan(proj[:, :n].contiguous(), gate[:, :n].contiguous(), logit=True, mix=True)
        q, k, v = heads(y)
        g = torch.nn.functional.pad(r[:, :n], (0, 0, 0, -n % C)).reshape(B, -1, C, H).cumsum(2).reshape(B, -1, H)[:, :n].contiguous()
        b = beta[:, :n].contiguous()
        u, w = tri.gdn_chunk_tri_solve_multi(k, b, g, [v, k], C, row_scales=[b, b * g.exp()])
        o, state = tri.gdn_chunk_attn(q, k, u, g, C, W=w)
        return y, o, mixed, state

    y, o, mixed, state = prompt(T)
    whole_y, whole, *_ = prompt(T + 1)
    assert torch.equal(whole_y[:, :T], y)
    slots = torch.tensor([1, 0], dtype=torch.int32, device=DEV)
    mixed, state = mixed[[1, 0]].contiguous(), state[[1, 0]].contiguous()
    token = tri.gated_scan_step(proj[:, T], gate[:, T], mixed, slots, logit=True, mix=True)
    q, k, v = heads(token)
    got = tri.gdn_step(q, k, v, r[:, T].contiguous(), state, beta=beta[:, T].contiguous(), slots=slots)
    # inputs to the delta rule are rounded to bf16 after sums in another order: a step of it here and there, and its chunk inverse in bf16 operands
    assert (got.double() - whole[:, T].double()).norm() <= 2.0 ** -5 * whole[:, T].double().norm()
