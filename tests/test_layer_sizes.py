"""Calls of the layer's operators at the far end of what their entry points take."""
import ctypes
import os

import pytest
import torch

import paper_2605_21325_amd as tri
from paper_2605_21325_amd import build as tri_build

BF = torch.bfloat16


@pytest.mark.gpu
def test_norm_of_more_rows_than_a_grid_has_threads_for_in_one_dimension():
    """2^26 rows and some: four a workgroup of 256 threads are 2^32 threads."""
    N, D = (1 << 26) + 5, 8
    x = torch.randn(1 << 12, D, device="cuda").to(BF)
    w = torch.rand(D, device="cuda").to(BF)
    want = tri.add_rms_norm(x, w)[0]
    x = x.repeat((1 << 14) + 1, 1)[:N]
    y, _ = tri.add_rms_norm(x, w)
    assert torch.equal(y[:-5].view(-1, *want.shape), want.expand(1 << 14, *want.shape)) and torch.equal(y[-5:], want[:5])
    q, scales, _ = tri.add_rms_norm_fp8(x, w)
    q0, scales0, _ = tri.add_rms_norm_fp8(x[:1 << 12], w)
    assert torch.equal(scales[-5:], scales0[:5]) and torch.equal(q[-5:].view(torch.uint8), q0[:5].view(torch.uint8))
    assert torch.equal(scales[:-5].view(-1, 1 << 12), scales0.view(1, -1).expand(1 << 14, -1))


@pytest.mark.gpu
def test_step_of_more_columns_than_a_grid_has_threads_for_in_one_dimension():
    """2^24 states and some of one row of four columns, a workgroup of 256 threads each."""
    B, H = (1 << 23) + 3, 2
    gen = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    q, k, v, beta, state = rand(B, 1, 1), rand(B, 1, 1), rand(B, H, 4), torch.rand(B, H, generator=gen, device="cuda"), rand(B, H, 1, 4)
    want = state.double() + k.double()[..., None] * (beta.double()[..., None] * (v.double() - k.double() * state.double()[:, :, 0]))[:, :, None]
    o = tri.gdn_step(q, k, v, None, state, beta=beta, scale=0.5)
    size = 1 + want.abs().amax()  # a handful of fp32 roundings
    assert ((state.double() - want).abs().amax() <= 2.0 ** -21 * size ** 2) and ((o.double() - 0.5 * q.double() * want[:, :, 0]).abs() <= 2.0 ** -21 * size ** 2 * (1 + q.double().abs())).all()


@pytest.mark.parametrize("B,T,H,C,forward,backward", [
    ((1 << 23) - 1, 0, 1, 16, True, False), (1 << 23, 0, 1, 16, False, False), (1 << 22, 0, 1, 16, True, False), (1 << 20, 0, 8, 16, False, False), ((1 << 22) - 1, 0, 1, 16, True, True),
    (1, 16 << 23, 1, 16, True, False), (1, (16 << 23) - 16, 1, 16, True, True), (1, 128 << 22, 1, 128, True, False), (1, (64 << 23) - 64, 1, 64, True, True)])
def test_more_workgroups_than_a_grid_has_threads_for_are_refused(B, T, H, C, forward, backward):
    """Decided on the host; what is taken is refused for its misaligned Q instead, so that no kernel runs."""
    if not os.path.exists(tri.binding.LIB_PATH):
        tri_build.build()
    L, at, room, align, unsupported = tri.lib(), lambda i: (i + 1) << 44, 1 << 62, -6, -9
    sizes = (room, B, T, H, 1, 32, 8, C, tri.BF16, 1.0, None)
    assert L.gdn_chunk_attn(at(0) + 2, at(1), at(2), None, None, None, at(3), None, at(4), *sizes) == (align if forward else unsupported)
    assert L.gdn_chunk_attn_bwd(at(0) + 2, at(1), at(2), None, None, None, at(3), None, at(4), at(5), at(6), None, None, None, at(7), *sizes) == (align if backward else unsupported)


@pytest.mark.parametrize("n_seq,chunks,H,d_k,d_v", [
    (1, 10, 1, 1 << 30, 64), (1, 10, 1, 128, (1 << 31) - 1), (1, 10, 1, 96 + 16, 64), (1, 10, 1, 128, 12), (1 << 30, 10, 1 << 30, 128, 64), (1, 1 << 31, 1, 128, 64), (1, 1 << 62, 4, 128, 64),
    (1, 1 << 20, 1 << 13, 128, 64)])
def test_workspaces_of_what_no_call_takes_are_refused(n_seq, chunks, H, d_k, d_v):
    """Sizes whose products pass 64 bits among them."""
    if not os.path.exists(tri.binding.LIB_PATH):
        tri_build.build()
    n = ctypes.c_int64(-1)
    assert tri.lib().gdn_chunk_attn_workspace(n_seq, chunks, H, d_k, d_v, 1, ctypes.byref(n)) == -5 and n.value == -1
    assert tri.lib().gdn_chunk_attn_bwd_workspace(0, chunks, H << (n_seq > 1), d_k, d_v, 64, 1, ctypes.byref(n)) == -5 and n.value == -1


@pytest.mark.parametrize("tokens,chunks,C,status", [(64 * 3, 3, 64, 0), (64 * 3 + 1, 3, 64, -5), (1 << 62, 3, 64, -5), (3, 3, 48, -2), (3, 3, 0, -2), (0, 0, 128, 0)])
def test_workspace_of_a_gradient_by_its_tokens(tokens, chunks, C, status):
    if not os.path.exists(tri.binding.LIB_PATH):
        tri_build.build()
    n = ctypes.c_int64(-1)
    assert tri.lib().gdn_chunk_attn_bwd_workspace(tokens, chunks, 4, 128, 64, C, 1, ctypes.byref(n)) == status
    assert n.value == (-1 if status else 4 * 4 * (2 * chunks * (2 if C > 64 else 1) * 128 * 64 + tokens * 64))
