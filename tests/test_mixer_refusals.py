"""What the entry points of the head norms and the gated recurrence refuse, decided on the host: no kernel runs (every pointer here is made up)."""
import ctypes
import os

import pytest
import torch

import paper_2605_21325_amd as tri
from paper_2605_21325_amd import build as tri_build
from paper_2605_21325_amd import mixer

OK, NULL, BAD_DTYPE, BAD_METHOD, BAD_SHAPE, ALIGN, ALIAS, UNSUPPORTED = 0, -1, -3, -4, -5, -6, -7, -9


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(tri.binding.LIB_PATH):
        tri_build.build()
    return tri.lib()


def address(i):
    return (i + 1) << 40  # far apart, aligned


HEADS = dict(q=address(0), k=address(1), qw=address(2), kw=address(3), pos=address(4), freq=address(5), qo=address(6), ko=address(7), N=5, qs=512, ks=256, qos=512, kos=256, H=4, Hk=2, d=128, rot=64,
             dtype=tri.BF16, flags=0, eps=1e-6, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(N=0), OK), (dict(N=-1), BAD_SHAPE), (dict(N=1 << 31), BAD_SHAPE), (dict(H=0), BAD_SHAPE), (dict(Hk=-1), BAD_SHAPE), (dict(d=0), BAD_SHAPE), (dict(d=513), BAD_SHAPE), (dict(rot=130), BAD_SHAPE),
    (dict(rot=63), BAD_SHAPE), (dict(rot=-2), BAD_SHAPE), (dict(dtype=3), BAD_DTYPE), (dict(flags=8), BAD_METHOD), (dict(N=1 << 30), UNSUPPORTED), (dict(qs=-1), BAD_SHAPE), (dict(ks=1 << 32), BAD_SHAPE),
    (dict(qos=511), BAD_SHAPE), (dict(kos=255), BAD_SHAPE), (dict(q=None), NULL), (dict(k=None), NULL), (dict(qo=None), NULL), (dict(ko=None), NULL), (dict(pos=None), NULL), (dict(freq=None), NULL),
    (dict(q=address(0) + 1), ALIGN), (dict(kw=address(3) + 1), ALIGN), (dict(freq=address(5) + 2), ALIGN), (dict(pos=address(4) + 4, flags=4), ALIGN), (dict(qo=address(0) + 1024), ALIAS),
    (dict(qo=address(0), qos=1024), ALIAS), (dict(qo=address(1)), ALIAS), (dict(ko=address(0)), ALIAS), (dict(ko=address(6) + 512), ALIAS), (dict(qo=address(2)), ALIAS), (dict(ko=address(4)), ALIAS),
    # rows of one buffer: q and q_out lie beside each other, k_out begins inside q_out's
    (dict(qs=1000, ks=1000, qos=1000, kos=1000, qo=address(0) + 2 * 512, ko=address(0) + 2 * 500), ALIAS)])
def test_heads(L, change, status):
    assert L.qk_norm_rope(*dict(HEADS, **change).values()) == status


HEADS_BWD = dict(uq=address(0), uk=address(1), q=address(2), k=address(3), qw=address(4), kw=address(5), pos=address(6), freq=address(7), dq=address(8), dk=address(9), dqw=address(10), dkw=address(11),
                 ws=address(12), ws_bytes=1 << 30, N=5, uqs=512, uks=256, qs=512, ks=256, dqs=512, dks=256, H=4, Hk=2, d=128, rot=64, dtype=tri.BF16, flags=0, eps=1e-6, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(N=-1), BAD_SHAPE), (dict(d=600), BAD_SHAPE), (dict(rot=1), BAD_SHAPE), (dict(dtype=-1), BAD_DTYPE), (dict(flags=16), BAD_METHOD), (dict(uq=None), NULL), (dict(uk=None), NULL),
    (dict(q=None), NULL), (dict(dq=None), NULL), (dict(dk=None), NULL), (dict(ws=None), NULL), (dict(qw=None), NULL), (dict(kw=None), NULL), (dict(pos=None), NULL), (dict(ws_bytes=16), BAD_SHAPE),
    (dict(dqs=100), BAD_SHAPE), (dict(uks=-2), BAD_SHAPE), (dict(dqw=address(10) + 2), ALIGN), (dict(ws=address(12) + 8), ALIGN), (dict(uq=address(0) + 1), ALIGN), (dict(dq=address(2)), ALIAS),
    (dict(dk=address(8)), ALIAS), (dict(dkw=address(10)), ALIAS), (dict(dq=address(0), dqs=600), ALIAS), (dict(dq=address(1)), ALIAS), (dict(dqw=address(0)), ALIAS), (dict(ws=address(3)), ALIAS)])
def test_heads_gradient(L, change, status):
    assert L.qk_norm_rope_bwd(*dict(HEADS_BWD, **change).values()) == status


SCAN = dict(x=address(0), g=address(1), state=address(2), h=address(3), final=address(4), ws=address(5), ws_bytes=1 << 40, B=2, T=50, D=100, xs=100, gs=100, hs=100, dtype=tri.BF16, gtype=tri.F32,
            flags=0, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(B=0), BAD_SHAPE), (dict(T=-1), BAD_SHAPE), (dict(T=1 << 31), BAD_SHAPE), (dict(B=1 << 20, T=1 << 12), BAD_SHAPE), (dict(B=1 << 30, T=0, D=128), UNSUPPORTED), (dict(D=0), BAD_SHAPE), (dict(D=(1 << 20) + 1), BAD_SHAPE),
    (dict(dtype=4), BAD_DTYPE), (dict(gtype=tri.F16), BAD_DTYPE), (dict(dtype=tri.F32, gtype=tri.BF16), BAD_DTYPE), (dict(flags=4), BAD_METHOD), (dict(xs=-1), BAD_SHAPE),
    (dict(hs=99), BAD_SHAPE), (dict(gs=(1 << 24) + 1), BAD_SHAPE), (dict(x=None), NULL), (dict(g=None), NULL), (dict(h=None), NULL), (dict(x=address(0) + 1), ALIGN), (dict(g=address(1) + 2), ALIGN),
    (dict(state=address(2) + 2), ALIGN), (dict(ws=address(5) + 8), ALIGN), (dict(h=address(0)), ALIAS), (dict(h=address(1) + 8), ALIAS), (dict(final=address(0)), ALIAS), (dict(final=address(2) + 4), ALIAS),
    (dict(final=address(3)), ALIAS), (dict(state=address(3), final=address(3)), ALIAS)])
def test_scan(L, change, status):
    assert L.gated_scan(*dict(SCAN, **change).values()) == status


def test_scan_packed(L):
    a = dict(x=address(0), g=address(1), state=address(2), h=address(3), final=address(4), ws=address(5), ws_bytes=1 << 40, cu=address(6), n=3, total=100, D=64, xs=64, gs=64, hs=64, dtype=tri.F16,
             gtype=tri.F16, flags=3, stream=None)
    for change, status in [(dict(cu=None), NULL), (dict(cu=address(6) + 4), ALIGN), (dict(cu=address(3)), ALIAS), (dict(n=0), BAD_SHAPE), (dict(total=-1), BAD_SHAPE), (dict(total=1 << 31), BAD_SHAPE)]:
        assert L.gated_scan_varlen(*dict(a, **change).values()) == status


SCAN_BWD = dict(x=address(0), g=address(1), h=address(2), state=address(3), dh=address(4), dstate=address(5), dx=address(6), dg=address(7), dstate0=address(8), ws=address(9), ws_bytes=1 << 40, B=2, T=50,
                D=100, xs=100, gs=100, hs=100, dhs=100, dxs=100, dgs=100, dtype=tri.BF16, gtype=tri.BF16, flags=2, stream=None)


@pytest.mark.parametrize("change,status", [
    (dict(B=0), BAD_SHAPE), (dict(D=0), BAD_SHAPE), (dict(dtype=4), BAD_DTYPE), (dict(flags=8), BAD_METHOD), (dict(x=None), NULL), (dict(h=None), NULL), (dict(dh=None), NULL), (dict(dx=None), NULL),
    (dict(dg=None), NULL), (dict(g=None), NULL), (dict(dgs=99), BAD_SHAPE), (dict(dhs=-1), BAD_SHAPE), (dict(dg=address(7) + 1), ALIGN), (dict(dstate=address(5) + 1), ALIGN), (dict(dx=address(4)), ALIAS),
    (dict(dg=address(1)), ALIAS), (dict(dg=address(6)), ALIAS), (dict(dstate0=address(3)), ALIAS), (dict(dstate0=address(2)), ALIAS), (dict(dstate0=address(5)), ALIAS)])
def test_scan_gradient(L, change, status):
    assert L.gated_scan_bwd(*dict(SCAN_BWD, **change).values()) == status


@pytest.mark.parametrize("change,status", [
    (dict(B=0), OK), (dict(B=-1), BAD_SHAPE), (dict(n_slot=2, slots=None), BAD_SHAPE), (dict(n_slot=-1), BAD_SHAPE), (dict(n_slot=1 << 31), BAD_SHAPE), (dict(D=0), BAD_SHAPE), (dict(dtype=9), BAD_DTYPE),
    (dict(flags=4), BAD_METHOD), (dict(hs=10), BAD_SHAPE), (dict(x=None), NULL), (dict(g=None), NULL), (dict(h=None), NULL), (dict(state=None), NULL), (dict(state=address(2) + 2), ALIGN),
    (dict(slots=address(3) + 2), ALIGN), (dict(h=address(0)), ALIAS), (dict(state=address(1)), ALIAS), (dict(h=address(2) + 400), ALIAS), (dict(B=1 << 27, n_slot=1 << 28), UNSUPPORTED), (dict(xs=(1 << 29) + 1), BAD_SHAPE),
    (dict(xs=1 << 29, gs=1 << 25, h=None), NULL)])
def test_scan_step(L, change, status):
    a = dict(x=address(0), g=address(1), state=address(2), slots=address(3), h=address(4), B=3, n_slot=8, D=100, xs=100, gs=100, hs=100, dtype=tri.BF16, gtype=tri.F32, flags=1, stream=None)
    assert L.gated_scan_step(*dict(a, **change).values()) == status


def test_workspaces(L):
    n = ctypes.c_int64(-1)
    assert L.gated_scan_workspace(100, 2, 64, ctypes.byref(n)) == OK and n.value >= 0
    assert L.gated_scan_workspace(100, 0, 64, ctypes.byref(n)) == BAD_SHAPE
    assert L.gated_scan_workspace(64, 64, 64, ctypes.byref(n)) == OK and n.value == 0
    assert L.gated_scan_workspace(100, 2, 64, None) == NULL
    assert L.qk_norm_rope_bwd_workspace(100, 4, 2, 64, ctypes.byref(n)) == OK and n.value >= 2 * 64 * 4 and n.value % (64 * 4) == 0
    assert L.qk_norm_rope_bwd_workspace(0, 4, 2, 64, ctypes.byref(n)) == OK and n.value == 0
    assert L.qk_norm_rope_bwd_workspace(100, 4, 2, 600, ctypes.byref(n)) == BAD_SHAPE


class Device:
    """A stand-in for a device tensor: what the binding reads of one."""

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return True if name == "is_cuda" else getattr(self.t, name)


@pytest.mark.parametrize("t,inner,step", [
    (torch.zeros(3, 4, 8), 1, 8), (torch.zeros(3, 4, 8), 2, 32), (torch.zeros(3, 4, 20)[..., :8], 1, 20), (torch.zeros(12, 40)[:, 8:24].view(12, 2, 8), 2, 40), (torch.zeros(1, 1, 8), 1, 8),
    (torch.zeros(5, 1, 1, 30)[..., 2:9], 1, 30), (torch.zeros(0, 4, 8), 1, 8), (torch.zeros(2, 1, 9)[:, :, 4:8], 1, 9), (torch.zeros(8).expand(3, 8), 1, 0), (torch.zeros(4, 3)[:, ::3], 1, 3)])
def test_rows(t, inner, step):
    assert mixer._rows(Device(t), "t", inner) == (t.data_ptr(), step)


@pytest.mark.parametrize("t,inner", [(torch.zeros(3, 8)[:, ::2], 1), (torch.zeros(3, 8, 4).transpose(1, 2), 2), (torch.zeros(3, 5, 8)[:, :4], 1), (torch.zeros(3, 2, 10)[..., :8], 2),
                                     (torch.zeros(4, 3, 8).transpose(0, 1), 1)])
def test_rows_that_are_none(t, inner):
    with pytest.raises(ValueError, match="contiguous|one stride"):
        mixer._rows(Device(t), "t", inner)


def test_the_binding_refuses_what_a_kernel_would_misread():
    bf = torch.bfloat16
    q, k, w = torch.zeros(2, 5, 4, 64, dtype=bf), torch.zeros(2, 5, 2, 64, dtype=bf), torch.zeros(64, dtype=bf)
    pos, freq = torch.zeros(2, 5, dtype=torch.int32), torch.zeros(32)
    good = dict(q=q, k=k, q_weight=w, k_weight=w, positions=pos, inv_freq=freq)
    with pytest.raises(ValueError, match="device memory"):
        tri.qk_norm_rope(**good)
    for bad in (dict(k=k[:, :4]), dict(k=k[..., :32]), dict(q_weight=w[:32]), dict(positions=pos[:1]), dict(inv_freq=torch.zeros(40)), dict(positions=None), dict(inv_freq=None), dict(k=None), dict(k=w),
                dict(q=w), dict(inv_freq=torch.zeros(4, 8))):
        with pytest.raises(ValueError):
            tri.qk_norm_rope(**dict(good, **bad))
    for bad in (dict(k=k.half()), dict(k_weight=w.float()), dict(positions=pos.float()), dict(inv_freq=freq.double())):
        with pytest.raises(TypeError):
            tri.qk_norm_rope(**dict(good, **bad))
    for bad in (dict(dq_out=q[:1], dk_out=k), dict(dq_out=q, dk_out=None), dict(dq_out=q.unflatten(0, (1, 2)), dk_out=k)):
        with pytest.raises(ValueError):
            tri.qk_norm_rope_bwd(**bad, **good)
    x, g, s = torch.zeros(2, 5, 64, dtype=bf), torch.zeros(2, 5, 64), torch.zeros(2, 64)
    for bad in (dict(g=g[..., :32]), dict(state=s[:1]), dict(final_state=s[:, :3]), dict(x=x[0]), dict(h=x[:1])):
        with pytest.raises(ValueError):
            tri.gated_scan(**dict(dict(x=x, g=g), **bad))
    for bad in (dict(g=g.half()), dict(g=g.double()), dict(state=s.double())):
        with pytest.raises(TypeError):
            tri.gated_scan(**dict(dict(x=x, g=g), **bad))
    with pytest.raises(ValueError, match="sum to"):
        tri.gated_scan_varlen(x[0], g[0], [2, 2])
    with pytest.raises(ValueError, match="negative"):
        tri.gated_scan_varlen(x[0], g[0], [6, -1])
    with pytest.raises(ValueError, match="needs x"):
        tri.gated_scan_bwd(None, g, x, x, mix=True)
    for bad in (dict(dh=x[:, :4]), dict(state=s[:1]), dict(dstate=s[0]), dict(h=x[0]), dict(x=x[..., :5])):
        with pytest.raises(ValueError):
            tri.gated_scan_bwd(**dict(dict(x=x, g=g, h=x, dh=x), **bad))
    step = dict(x=x[0], g=g[0], state=torch.zeros(7, 64))
    for bad in (dict(g=g[0, :2]), dict(state=torch.zeros(7, 60)), dict(state=torch.zeros(64)), dict(x=x), dict(slots=torch.zeros(4, dtype=torch.int32))):
        with pytest.raises(ValueError):
            tri.gated_scan_step(**dict(step, **bad))
    with pytest.raises(TypeError):
        tri.gated_scan_step(**dict(step, slots=torch.zeros(5, dtype=torch.int64)))
