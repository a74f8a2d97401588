"""The gated recurrence's token at the largest numbers of sequences."""
import os

import pytest
import torch

import paper_2605_21325_amd as tri
from paper_2605_21325_amd import build as tri_build


@pytest.mark.parametrize("B,D,status", [(1 << 26, 1, -9), (1 << 26, 64, -9), ((1 << 26) - 1, 64, -1), (1 << 25, 65, -9), ((1 << 25) - 1, 128, -1), (64, 1 << 20, -1), (0, 64, 0)])
def test_limits_of_a_step(B, D, status):
    """Refused as unsupported from the limit on; up to it the missing result is (no kernel runs)."""
    if not os.path.exists(tri.binding.LIB_PATH):
        tri_build.build()
    at = [(i + 1) << 44 for i in range(3)]
    assert tri.lib().gated_scan_step(at[0], at[1], at[2], None, None, B, 1 << 27, D, D, D, D, tri.F32, tri.F32, 0, None) == status


@pytest.mark.gpu
def test_step_of_more_states_than_a_grid_has_threads_for_in_one_dimension():
    """2^24 sequences and some of one channel, a workgroup of 256 threads each; one of them is padding."""
    B = (1 << 24) + 5
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, g, state = (torch.randn(B, 1, generator=gen, device="cuda") for _ in range(3))
    slots = torch.arange(B - 1, -1, -1, dtype=torch.int32, device="cuda")
    slots[B - 2] = -1  # (slot 1 stays as it is)
    a, before = torch.sigmoid(g.double()), state.double().flip(0)
    want, size = a * before + (1 - a) * x.double(), a * before.abs() + (1 - a) * x.double().abs()
    kept = state[1].clone()
    h = tri.gated_scan_step(x, g, state, slots, logit=True, mix=True)
    # a decay and one less it off by 4 steps (8 2^-24) each, a product and a sum
    good = (h.double() - want).abs() <= 16 * 2.0 ** -24 * size + 2.0 ** -126
    good[B - 2] = h[B - 2] == 0
    assert good.all()
    assert torch.equal(state.flip(0)[:B - 2], h[:B - 2]) and torch.equal(state[0], h[B - 1]) and torch.equal(state[1], kept)
