"""Sequences taken in segments (few heads, many chunks): the state overwritten in place, and the chunk sizes and layers that prompts have."""
import ctypes
import os

import pytest
import torch

import paper_2605_21325_amd as tri
from paper_2605_21325_amd import build as tri_build
from test_layer_gpu import BF, HF, check_forward, make


def workspace(n_seq, chunks, H, d_k, d_v, has_w):
    if not os.path.exists(tri.binding.LIB_PATH):
        tri_build.build()
    n = ctypes.c_int64(-1)
    assert tri.lib().gdn_chunk_attn_workspace(n_seq, chunks, H, d_k, d_v, has_w, ctypes.byref(n)) == 0
    return n.value


@pytest.mark.parametrize("has_w", [0, 1])
def test_the_workspace_has_room_for_the_state_before_the_first_token(has_w):
    """The first segment begins with it while the last one writes the final state, which may be the same memory: a state for every segment, the first one's too."""
    n_seq, H, d_k, d_v = 1, 8, 128, 64
    got = workspace(n_seq, 8 * 16, H, d_k, d_v, has_w)  # 16 segments of 8 chunks
    state, other = 4 * H * d_k * d_v, 4 * H * (d_k * d_k if has_w else 1)
    assert got == 16 * state + 15 * other


PLACES = [
    # lens, H, d_k, d_v, C, dtype, delta
    ([64 * 129], 8, 128, 128, 64, BF, True),  # 16 segments of nine chunks: the last one is empty
    ([64 * 40 + 5], 4, 128, 128, 64, HF, True),
    ([64 * 129 - 3], 8, 128, 128, 64, BF, False),
    ([64 * 100, 70, 0, 3], 2, 64, 128, 64, BF, True),  # short ones beside a long one: all but their first segment are empty
    ([3, 64 * 90 + 1, 0], 2, 128, 64, 64, HF, False),
    ([128 * 33 + 7], 4, 128, 128, 128, BF, True),
    ([16 * 200 + 1], 2, 64, 72, 16, BF, True),
]


@pytest.mark.gpu
@pytest.mark.parametrize("lens,H,d_k,d_v,C,dtype,delta", PLACES)
def test_the_state_in_place(lens, H, d_k, d_v, C, dtype, delta):
    assert workspace(len(lens), sum(-(-n // C) for n in lens), H, d_k, d_v, delta) > 0
    x = make(lens, H, H, d_k, d_v, C, dtype, True, delta, True, seed=31, rate=0.02)
    call = lambda state, final: tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, W=x["w"], state=state, final_state=final, scale=0.3)
    o, final = call(x["state"], None)
    for _ in range(5):
        state = x["state"].clone()
        o1, f1 = call(state, state)
        assert f1 is state and torch.equal(o1, o) and torch.equal(state, final)
    if len(lens) == 1:
        one = {n: None if x[n] is None else x[n][None] for n in ("q", "k", "u", "w", "g")}
        state = x["state"].clone()
        o1, _ = tri.gdn_chunk_attn(one["q"], one["k"], one["u"], one["g"], C, W=one["w"], state=state, final_state=state, scale=0.3)
        assert torch.equal(o1[0], o) and torch.equal(state, final)


@pytest.mark.gpu
@pytest.mark.parametrize("lens,H,Hk,d_k,d_v,C,dtype,gate,delta,state", [
    ([64 * 17 + 5], 2, 1, 128, 128, 64, BF, True, True, True),
    ([64 * 17 + 5], 2, 2, 128, 128, 64, BF, False, True, False),
    ([64 * 24], 2, 2, 128, 128, 64, HF, True, True, False),
    ([64 * 33 + 1, 7], 1, 1, 128, 128, 64, BF, True, False, True),
    ([128 * 17 + 3], 2, 1, 128, 128, 128, BF, False, True, False),
    ([128 * 16 + 65], 1, 1, 128, 64, 128, HF, True, True, True),
    ([128 * 18 + 64], 1, 1, 64, 128, 128, BF, True, False, True),
])
def test_segments_of_a_prompt(lens, H, Hk, d_k, d_v, C, dtype, gate, delta, state):
    """As test_segments of the operators' tests, at the chunk sizes and layers that prompts have."""
    assert workspace(len(lens), sum(-(-n // C) for n in lens), H, d_k, d_v, delta) > 0
    x = make(lens, H, Hk, d_k, d_v, C, dtype, gate, delta, state, seed=33, rate=0.02)
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, W=x["w"], state=x["state"], scale=0.3)
    check_forward(o, final, x, lens, C, 0.3, dtype)


def test_a_prompt_has_segments_from_sixteen_chunks_on():
    """Four at least, of four chunks at least: two segments were slower than none (1024 tokens of 8 heads with W: 60 against 50 us, four 43)."""
    state, other = 4 * 8 * 128 * 128, 4 * 8 * 128 * 128
    count = lambda chunks: (workspace(1, chunks, 8, 128, 128, 1) + other) // (state + other) or 1
    assert [count(n) for n in (1, 15, 16, 24, 64, 127, 128, 200)] == [1, 1, 4, 6, 16, 16, 16, 16]  # (256 / 16 units: 16 at most)
