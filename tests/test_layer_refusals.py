"""What the entry points of the layer's operators refuse, decided on the host: no kernel runs (every pointer here is made up)."""
import ctypes
import os

import pytest
import torch

import paper_2605_21325_amd as tri
from paper_2605_21325_amd import build as tri_build

OK, NULL, BAD_C, BAD_DTYPE, BAD_SHAPE, ALIGN, ALIAS, UNSUPPORTED = 0, -1, -2, -3, -5, -6, -7, -9


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(tri.binding.LIB_PATH):
        tri_build.build()
    return tri.lib()


def address(i):
    return (i + 1) << 40  # far apart, aligned


ATTN = dict(Q=address(0), K=address(1), U=address(2), W=address(3), g=address(4), state=address(5), O=address(6), final=address(7), ws=address(8), ws_bytes=1 << 36,
            B=1, T=100, H=4, Hk=2, dk=128, dv=64, C=64, dtype=tri.BF16, scale=1.0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(C=48), BAD_C), (dict(C=0), BAD_C), (dict(dtype=7), BAD_DTYPE), (dict(dtype=tri.F32), UNSUPPORTED), (dict(B=0), BAD_SHAPE), (dict(T=-1), BAD_SHAPE), (dict(T=1 << 31), BAD_SHAPE),
    (dict(H=0), BAD_SHAPE), (dict(Hk=3), BAD_SHAPE), (dict(Hk=0), BAD_SHAPE), (dict(dk=100), BAD_SHAPE), (dict(dk=160), BAD_SHAPE), (dict(dv=12), BAD_SHAPE), (dict(dv=520), BAD_SHAPE),
    (dict(dv=0), BAD_SHAPE), (dict(H=1 << 20, Hk=1), UNSUPPORTED), (dict(Q=None), NULL), (dict(K=None), NULL), (dict(U=None), NULL), (dict(O=None), NULL), (dict(Q=address(0) + 2), ALIGN),
    (dict(W=address(3) + 8), ALIGN), (dict(g=address(4) + 2), ALIGN), (dict(state=address(5) + 4), ALIGN), (dict(O=address(2)), ALIAS), (dict(final=address(6)), ALIAS),
    (dict(O=address(4) + 16), ALIAS), (dict(T=100000, ws=None, ws_bytes=0), NULL), (dict(T=100000, ws_bytes=16), BAD_SHAPE)])
def test_chunk_attention(L, change, status):
    a = dict(ATTN, **change)
    assert L.gdn_chunk_attn(*a.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(total=-1), BAD_SHAPE), (dict(chunks=99), BAD_SHAPE), (dict(chunks=1), BAD_SHAPE), (dict(n=0), BAD_SHAPE), (dict(cu=None), NULL), (dict(cc=None), NULL), (dict(cu=address(9) + 4), ALIGN),
    (dict(cc=address(6)), ALIAS), (dict(C=7), BAD_C)])
def test_chunk_attention_packed(L, change, status):
    a = dict(Q=address(0), K=address(1), U=address(2), W=address(3), g=address(4), state=address(5), O=address(6), final=address(7), ws=address(8), ws_bytes=1 << 36,
             cu=address(9), cc=address(10), n=2, total=100, chunks=3, H=4, Hk=2, dk=128, dv=64, C=64, dtype=tri.F16, scale=1.0, stream=None)
    a.update(change)
    assert L.gdn_chunk_attn_varlen(*a.values()) == status


BWD = dict(Q=address(0), K=address(1), U=address(2), W=address(3), g=address(4), state=address(5), dO=address(6), dstate=address(7), dQ=address(8), dK=address(9), dU=address(10),
           dW=address(11), dg=address(12), dstate0=address(13), ws=address(14), ws_bytes=1 << 36, B=1, T=100, H=4, Hk=2, dk=128, dv=64, C=64, dtype=tri.BF16, scale=1.0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(C=20), BAD_C), (dict(dtype=-1), BAD_DTYPE), (dict(dtype=tri.F32), UNSUPPORTED), (dict(Hk=3), BAD_SHAPE), (dict(dO=None), NULL), (dict(dQ=None), NULL), (dict(dK=None), NULL),
    (dict(dU=None), NULL), (dict(dW=None), NULL), (dict(W=None), NULL), (dict(g=None), NULL), (dict(ws=None), NULL), (dict(ws_bytes=1000), BAD_SHAPE), (dict(dQ=address(0)), ALIAS),
    (dict(dU=address(6)), ALIAS), (dict(dK=address(8)), ALIAS), (dict(dstate0=address(5)), ALIAS), (dict(dg=address(12) + 1), ALIGN), (dict(ws=address(14) + 8), ALIGN),
    (dict(H=1 << 17, Hk=1, dk=32), UNSUPPORTED)])
def test_gradient(L, change, status):
    a = dict(BWD, **change)
    assert L.gdn_chunk_attn_bwd(*a.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(B=0), OK), (dict(B=-1), BAD_SHAPE), (dict(n_slot=2, slots=None), BAD_SHAPE), (dict(n_slot=-1), BAD_SHAPE), (dict(n_slot=1 << 32), BAD_SHAPE), (dict(dk=257), BAD_SHAPE),
    (dict(dv=6), BAD_SHAPE), (dict(dv=516), BAD_SHAPE), (dict(Hk=3), BAD_SHAPE), (dict(dtype=9), BAD_DTYPE), (dict(q=None), NULL), (dict(state=None), NULL), (dict(o=None), NULL),
    (dict(v=address(2) + 8), ALIGN), (dict(state=address(5) + 4), ALIGN), (dict(o=address(2)), ALIAS), (dict(state=address(0)), ALIAS)])
def test_step(L, change, status):
    a = dict(q=address(0), k=address(1), v=address(2), g=address(3), beta=address(4), state=address(5), slots=address(6), o=address(7), B=3, n_slot=8, H=4, Hk=2, dk=128, dv=64,
             dtype=tri.BF16, scale=1.0, stream=None)
    a.update(change)
    assert L.gdn_step(*a.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(N=0), OK), (dict(N=-1), BAD_SHAPE), (dict(D=12), BAD_SHAPE), (dict(D=16392), BAD_SHAPE), (dict(D=136), BAD_SHAPE), (dict(group=64), BAD_SHAPE), (dict(group=-2), BAD_SHAPE),
    (dict(dtype=5), BAD_DTYPE), (dict(x=None), NULL), (dict(scales=None), NULL), (dict(sum=None), NULL), (dict(residual=None), NULL), (dict(y=address(3) + 8), ALIGN),
    (dict(y=address(0)), ALIAS), (dict(sum=address(2)), ALIAS)])
def test_norm(L, change, status):
    a = dict(x=address(0), residual=address(1), weight=address(2), y=address(3), scales=address(4), sum=address(5), N=3, D=256, group=128, dtype=tri.BF16, eps=1e-6, stream=None)
    a.update(change)
    assert L.add_rms_norm(*a.values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(N=-1), BAD_SHAPE), (dict(D=4), BAD_SHAPE), (dict(ws_bytes=100), BAD_SHAPE), (dict(dtype=3), BAD_DTYPE), (dict(dy=None), NULL), (dict(dweight=None), NULL), (dict(ws=None), NULL),
    (dict(dx=address(0) + 8), ALIGN), (dict(dx=address(0)), ALIAS), (dict(dweight=address(2)), ALIAS)])
def test_norm_gradient(L, change, status):
    a = dict(dy=address(0), s=address(1), weight=address(2), dsum=address(3), dx=address(4), dweight=address(5), ws=address(6), ws_bytes=1 << 20, N=3, D=256, dtype=tri.BF16, eps=1e-6,
             stream=None)
    a.update(change)
    assert L.add_rms_norm_bwd(*a.values()) == status


def test_workspaces(L):
    n = ctypes.c_int64(-1)
    assert L.gdn_chunk_attn_workspace(1, 2, 4, 128, 128, 1, ctypes.byref(n)) == OK and n.value == 0
    assert L.gdn_chunk_attn_workspace(0, 2, 4, 128, 128, 1, ctypes.byref(n)) == BAD_SHAPE
    assert L.gdn_chunk_attn_workspace(1, 2, 4, 128, 128, 1, None) == NULL
    assert L.gdn_chunk_attn_bwd_workspace(100, 2, 4, 128, 64, 64, 1, ctypes.byref(n)) == OK and n.value == 4 * 4 * (2 * 2 * 128 * 64 + 100 * 64)
    assert L.gdn_chunk_attn_bwd_workspace(-1, 2, 4, 128, 64, 64, 1, ctypes.byref(n)) == BAD_SHAPE


def test_the_binding_refuses_what_a_kernel_would_misread():
    bf = torch.bfloat16
    q, u, g = torch.zeros(1, 10, 2, 64, dtype=bf), torch.zeros(1, 10, 4, 64, dtype=bf), torch.zeros(1, 10, 4)
    state = torch.zeros(1, 4, 64, 64)
    with pytest.raises(ValueError, match="device memory"):
        tri.gdn_chunk_attn(q, q, u, g, 64)
    for bad in (dict(K=q[:, :9]), dict(U=u[:, :9]), dict(g=g[..., :3]), dict(W=q), dict(state=state[:, :3]), dict(final_state=state[..., :8]), dict(O=u[..., :8])):
        a = dict(dict(Q=q, K=q, U=u, g=g, C=64), **bad)
        with pytest.raises(ValueError, match="must be"):
            tri.gdn_chunk_attn(**a)
    for bad in (dict(K=q.half()), dict(U=u.float()), dict(g=g.double()), dict(state=state.to(bf))):
        a = dict(dict(Q=q, K=q, U=u, g=g, C=64), **bad)
        with pytest.raises(TypeError):
            tri.gdn_chunk_attn(**a)
    with pytest.raises(ValueError, match="must be"):
        tri.gdn_chunk_attn_bwd(q, q, u, g, u[:, :9], 64)
    with pytest.raises(ValueError, match="sum to"):
        tri.gdn_chunk_attn_varlen(q[0], q[0], u[0], g[0], [4, 5], 64)
    step = dict(q=q[:, 0], k=q[:, 0], v=u[:, 0], g=g[:, 0], state=state)
    for bad in (dict(k=q[:, 0, :, :32]), dict(v=u[0, :2]), dict(beta=g[:, 0, :2]), dict(state=state[..., :32])):
        with pytest.raises(ValueError):
            tri.gdn_step(**dict(step, **bad))
    with pytest.raises(TypeError):
        tri.gdn_step(**dict(step, slots=torch.zeros(1, dtype=torch.int64)))
    x, w = torch.zeros(4, 64, dtype=bf), torch.zeros(64, dtype=bf)
    for bad in (dict(weight=w[:32]), dict(residual=x[:2])):
        with pytest.raises(ValueError):
            tri.add_rms_norm(**dict(dict(x=x, weight=w), **bad))
    with pytest.raises(TypeError):
        tri.add_rms_norm(x, w.float())
    with pytest.raises(ValueError):
        tri.add_rms_norm_bwd(x[:2], x, w)
