"""The gated recurrence where products of decays leave fp32's range and the states do not: what a walk token by token gives, forward and against the time.

Channels in turn: 0 as layers have them, 1 nothing until decays of e^20 have passed, 2 decays of e^40 and of e^-40 in turns from a state of 2^-100, 3 as 1 and then a decay of zero.
Tolerances as in test_mixer_gpu.py, which hold for any decays as long as states are finite (with the magnitude of 1 - a, which is negative here)."""
import numpy as np
import pytest
import torch

import paper_2605_21325_amd as tri
from oracle import mixer
from tests.test_mixer_gpu import BF, DEV, E, F, HF, check_scan, exact, generator, make_scan, rand, sequences, within

pytestmark = pytest.mark.gpu


def steep(lens, D, dtype, gtype, back, seed=0):
    """Inputs of the forward pass, or (back) those of the gradient, with the same in the order of its run."""
    v, up = make_scan(lens, D, dtype, gtype, False, seed=seed)
    h = rand(generator(seed + 1), sum(lens), D).to(dtype)
    b, start = (up["dh"], up["dstate"]) if back else (v["x"], v["state"])
    at = 0
    for s, T in enumerate(lens):
        order = torch.arange(at + T - 1, at - 1, -1, device=DEV) if back else torch.arange(at, at + T, device=DEV)
        at += T
        if not T:
            continue
        n = max(1, 3 * T // 4)
        for kind in (1, 2, 3):
            if kind == 2 and dtype == HF:  # (e^51 is not among its numbers)
                continue
            c = torch.arange(kind, D, 4, device=DEV)
            first = order[:n]
            grid = first[:, None], c[None]
            if kind == 2:
                turn = torch.arange(len(first), device=DEV) // 3 % 2
                up_down = 40.0 - 80.0 * turn
                # the last turn is left whole: decays from there on start from 2^-100
                v["g"][grid] = torch.where(torch.arange(len(first), device=DEV) < len(first) // 6 * 6, up_down, -0.1)[:, None].to(gtype).expand(-1, len(c))
                start[s, c] = 2.0 ** -100
            else:
                v["g"][grid] = 20.0
                if kind == 3:
                    v["g"][first[-1], c] = -torch.inf
                start[s, c] = 0
            b[grid] = 0
    return v, up, h


def check_back(lens, v, h, up, got, mix):
    for s, (x, g, y, dy, ox, og) in enumerate(sequences(lens, v["x"], v["g"], h, up["dh"], got[0], got[1])):
        S, dS = exact(v["state"][s]), exact(up["dstate"][s])
        rx, rg, r0, r = mixer.gated_scan_bwd(x, g, y, S, dy, dS, False, mix)
        _, _, m0, m = mixer.gated_scan_bwd(x, g, y, S, np.abs(dy), np.abs(dS), False, mix)
        a, rest = mixer.gates(g, False)
        err, e = np.empty_like(m), np.zeros(m.shape[1])
        for t in reversed(range(len(m))):
            err[t] = e + 16 * E * m[t]
            e = a[t] * err[t]
        past = np.concatenate([S[None], y[:-1]])[:len(y)]
        size = np.abs(past) + (np.abs(x) if mix else 0)
        within(torch.from_numpy(ox), rx, err * (np.abs(rest) if mix else 1) + 16 * E * np.abs(rx), v["x"].dtype, f"dx of sequence {s}")
        within(torch.from_numpy(og), rg, a * (err * np.abs(past - x if mix else past) + 16 * E * np.abs(r) * size), v["g"].dtype, f"dg of sequence {s}")
        within(got[2][s], r0, e + 16 * E * m0, F, f"dstate0 of sequence {s}")


CASES = [
    # lens, D, dtype, gtype: short ones; tiles of a strip each; many; in segments, of odd channels, empty ones among them
    ([50], 64, F, F), ([17, 0, 33, 64], 72, BF, BF), ([300], 66, F, F), ([700, 90], 130, BF, F), ([600] * 40, 512, HF, HF), ([257, 1, 1000], 33, F, F), ([1500] * 12, 2048, BF, BF),
    ([3000], 256, F, F), ([5000, 0, 900], 64, BF, BF), ([2500], 37, HF, F), ([4000, 4000], 320, F, F)]


@pytest.mark.parametrize("mix", [False, True])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_products_of_decays_beyond_the_range(case, mix):
    lens, D, dtype, gtype = CASES[case]
    v, _, _ = steep(lens, D, dtype, gtype, False, seed=case)
    got = tri.gated_scan_varlen(**v, seqlens=lens, mix=mix)
    check_scan(lens, v, got, False, mix)
    v, up, h = steep(lens, D, dtype, gtype, True, seed=case)
    check_back(lens, v, h, up, tri.gated_scan_bwd_varlen(v["x"], v["g"], h, up["dh"], lens, v["state"], up["dstate"], mix=mix), mix)


def test_final_state_upon_the_initial_one_and_the_same_bits():
    lens = [3000, 700]
    v, _, _ = steep(lens, 192, F, F, False)
    want, final = tri.gated_scan_varlen(**v, seqlens=lens)
    state = v["state"].clone()
    got, _ = tri.gated_scan_varlen(v["x"], v["g"], lens, state, final_state=state)
    assert torch.equal(got, want) and torch.equal(state, final) and final.isfinite().all()


@pytest.mark.parametrize("lens,D", [([600] * 6, 64), ([3000, 2000], 128)])
def test_channels_beside_them_stay_within_the_tolerance_and_sequences_as_they_are(lens, D):
    """One sequence of steep decays among others: the others' bits are those of a call without it."""
    v, _ = make_scan(lens, D, F, F, False)
    clean = tri.gated_scan_varlen(**v, seqlens=lens)
    T = lens[0]
    v["g"][:T // 2, 5], v["x"][:T // 2, 5], v["state"][0, 5] = 20.0, 0.0, 0.0
    h, final = tri.gated_scan_varlen(**v, seqlens=lens)
    check_scan(lens, v, (h, final), False, False)
    assert torch.equal(h[T:], clean[0][T:]) and torch.equal(final[1:], clean[1][1:])


def test_whole_sequences_beside_infinite_decays():
    """g = +infinity: its channel is infinite or NaN from that token on; the others go on."""
    v, _ = make_scan([900] * 2, 64, F, F, False, packed=False)
    want, final = tri.gated_scan(**v)
    v["g"][0, 400, 7] = torch.inf
    h, last = tri.gated_scan(**v)
    keep = torch.ones_like(h, dtype=torch.bool)
    keep[0, 400:, 7] = False
    assert not h[~keep].isfinite().any()
    check_scan([900] * 2, dict(x=v["x"][..., 8:], g=v["g"][..., 8:], state=v["state"][:, 8:]), (h[..., 8:], last[:, 8:]), False, False)
    assert torch.equal(h[1], want[1]) and torch.equal(last[1], final[1])
