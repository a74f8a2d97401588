"""The native argument handling of the layer's operators (csrc/fastcall.cpp) without a GPU: host tensors (device -1) and a stand-in for the C-ABI."""
import ctypes
import importlib.util
import shutil

import pytest
import torch

from paper_2605_21325_amd import build as tri_build

P, I, L, F = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float
# as in csrc/fastcall.cpp, struct LayerAbi
ABI = {
    "attn": [P] * 9 + [L, I, L, I, I, I, I, I, I, F, P],
    "attn_varlen": [P] * 9 + [L, P, P, I, L, L, I, I, I, I, I, I, F, P],
    "attn_workspace": [I, L, I, I, I, I, P],
    "attn_bwd": [P] * 15 + [L, I, L, I, I, I, I, I, I, F, P],
    "attn_bwd_varlen": [P] * 15 + [L, P, P, I, L, L, I, I, I, I, I, I, F, P],
    "attn_bwd_workspace": [L, L, I, I, I, I, I, P],
    "step": [P] * 8 + [I, L, I, I, I, I, I, F, P],
    "norm": [P] * 6 + [L, I, I, I, F, P],
    "norm_bwd": [P] * 7 + [L, L, I, I, F, P],
}
bf = torch.bfloat16


class Native:
    def __init__(self, path):
        spec = importlib.util.spec_from_file_location("_fastcall", path)
        self.module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(self.module)
        self.calls, self.status, self.keep = [], 0, []
        for name, types in ABI.items():
            self.keep.append(ctypes.CFUNCTYPE(I, *types)(lambda *a, name=name: self.answer(name, a)))
        self.module.connect_layer(*(ctypes.cast(f, P).value for f in self.keep))
        offsets = ctypes.CFUNCTYPE(I, P, I, I, L, P, P, P)(self.offsets)
        self.keep.append(offsets)
        self.module.connect(*[ctypes.cast(self.keep[0], P).value] * 5, ctypes.cast(offsets, P).value)

    def offsets(self, lens, n, C, total, at, n_chunk, stream):
        lens = ctypes.cast(lens, ctypes.POINTER(L))[:n]
        ctypes.cast(n_chunk, ctypes.POINTER(L))[0] = sum(-(-x // C) for x in lens)
        return 0 if sum(lens) == total else -5

    def answer(self, name, a):
        self.calls.append((name, a))
        if name.endswith("workspace"):
            ctypes.cast(a[-1], ctypes.POINTER(L))[0] = 64
        return self.status


@pytest.fixture
def native(tmp_path):
    if not tri_build._fastcall_current():
        tri_build.build_fastcall()
    copy = str(tmp_path / "_fastcall.so")
    shutil.copy(tri_build.FASTCALL, copy)
    return Native(copy)


def tensors():
    q, u, g = torch.zeros(2, 70, 2, 64, dtype=bf), torch.zeros(2, 70, 4, 72, dtype=bf), torch.zeros(2, 70, 4)
    return q, torch.zeros_like(q), u, g, torch.zeros(2, 70, 4, 64, dtype=bf), torch.zeros(2, 4, 64, 72)


def test_chunk_attention(native):
    Q, K, U, g, W, S = tensors()
    O, final = native.module.chunk_attn(-1, 7, Q, K, U, g, 64, W, S, None, None, None)
    name, a = native.calls[-1]
    assert name == "attn" and a[:9] == (Q.data_ptr(), K.data_ptr(), U.data_ptr(), W.data_ptr(), g.data_ptr(), S.data_ptr(), O.data_ptr(), final.data_ptr(), a[8]) and a[8]
    assert a[9:18] == (64, 2, 70, 4, 2, 64, 72, 64, 2) and a[18] == 0.125 and a[19] == 7
    assert O.shape == U.shape and O.dtype == bf and final.shape == S.shape and final.dtype == torch.float32
    out = native.module.chunk_attn(-1, 7, Q, K, U, None, 64, None, None, 2.0, U.clone(), S)
    assert out[1] is S and native.calls[-1][1][3:6] == (None, None, None) and native.calls[-1][1][18] == 2.0
    dO = torch.zeros_like(U)
    got = native.module.chunk_attn_bwd(-1, 7, Q, K, U, g, dO, 64, W, S, None, None)
    name, a = native.calls[-1]
    assert name == "attn_bwd" and a[6:8] == (dO.data_ptr(), None) and a[8:14] == tuple(x.data_ptr() for x in got) and [x.shape for x in got] == [x.shape for x in (Q, K, U, W, g, S)]
    got = native.module.chunk_attn_bwd(-1, 7, Q, K, U, None, dO, 64, None, None, None, 1.0)
    assert got[3:] == (None, None, None) and native.calls[-1][1][11:14] == (None, None, None)


def test_packed_chunk_attention(native):
    Q, K, U, g, W, S = tensors()
    q, k, u, gg, w = (x.flatten(0, 1) for x in (Q, K, U, g, W))
    O, final = native.module.chunk_attn_varlen(-1, 7, q, k, u, gg, [100, 40], 64, w, S, None, None, None)
    name, a = native.calls[-1]
    assert name == "attn_varlen" and a[12:21] == (2, 140, 3, 4, 2, 64, 72, 64, 2) and a[11] == a[10] + 24 and final._triinv_keepalive[0].data_ptr() == a[10]
    got = native.module.chunk_attn_bwd_varlen(-1, 7, q, k, u, gg, u, (100, 40), 64, w, S, S, None)
    name, a = native.calls[-1]
    assert name == "attn_bwd_varlen" and a[18:27] == (2, 140, 3, 4, 2, 64, 72, 64, 2) and got[0]._triinv_keepalive[0].data_ptr() == a[16]
    assert native.module.chunk_attn_varlen(-1, 7, q, k, u, gg, [100, 41], 64, w, S, None, None, None) is None


def test_step_and_norm(native):
    q, v, g, S = torch.zeros(3, 2, 64), torch.zeros(3, 4, 8), torch.zeros(3, 4), torch.zeros(9, 4, 64, 8)
    slots = torch.zeros(3, dtype=torch.int32)
    o = native.module.step(-1, 7, q, q, v, g, S, g, slots, None, None)
    name, a = native.calls[-1]
    assert name == "step" and a[3:8] == (g.data_ptr(), g.data_ptr(), S.data_ptr(), slots.data_ptr(), o.data_ptr()) and a[8:15] == (3, 9, 4, 2, 64, 8, 0) and a[15] == 0.125
    assert native.module.step(-1, 7, q, q, v, None, S, None, None, 1, o) is o and native.calls[-1][1][3:5] == (None, None)
    x, w = torch.zeros(2, 5, 256, dtype=bf), torch.zeros(256, dtype=bf)
    y, s = native.module.norm(-1, 7, x, w, None, 1e-6, -1)
    assert s is x and y.dtype == bf and native.calls[-1][1][6:9] == (10, 256, -1)
    y, scales, s = native.module.norm(-1, 7, x, w, x.clone(), 1e-6, 128)
    assert y.dtype == torch.float8_e4m3fn and scales.shape == (2, 5, 2) and native.calls[-1][1][3:6] == (y.data_ptr(), scales.data_ptr(), s.data_ptr())
    assert native.module.norm(-1, 7, x, w, None, 1e-6, 0)[1].shape == (2, 5, 1)
    dx, dw = native.module.norm_bwd(-1, 7, x, x, w, 1e-6, None)
    assert dx.shape == x.shape and dw.dtype == torch.float32 and native.calls[-1][1][7:11] == (4 * 10 * 256, 10, 256, 2)


def test_what_is_not_plain_goes_back(native):
    """None, and the C-ABI is not called: the Python route says what is wrong."""
    Q, K, U, g, W, S = tensors()
    ok = [-1, 7, Q, K, U, g, 64, W, S, None, None, None]
    for i, bad in ((3, K[:, :69]), (3, K.half()), (4, U.float()), (5, g.double()), (5, g[..., :3]), (6, 48), (6, 64.0), (7, Q), (8, S[:1]), (9, "1"), (10, U[:1]), (11, S.half()),
                   (2, Q.transpose(0, 1)), (2, None), (4, U[:, :0]), (2, Q[:, :0])):
        a = list(ok)
        a[i] = bad
        n = len(native.calls)
        assert native.module.chunk_attn(*a) is None and len(native.calls) == n, (i, bad)
    q, v, g, S = torch.zeros(3, 2, 64), torch.zeros(3, 4, 8), torch.zeros(3, 4), torch.zeros(9, 4, 64, 8)
    ok = [-1, 7, q, q, v, g, S, g, None, None, None]
    for i, bad in ((3, q[:2]), (4, v[:2]), (5, g.half()), (6, S[..., :4]), (7, g[:, :2]), (8, torch.zeros(3, dtype=torch.int64)), (8, torch.zeros(2, dtype=torch.int32)), (8, [0, 1, 2])):
        a = list(ok)
        a[i] = bad
        n = len(native.calls)
        assert native.module.step(*a) is None and len(native.calls) == n, (i, bad)
    x, w = torch.zeros(4, 256), torch.zeros(256)
    for a in ([x, w[:8], None, 1e-6, -1], [x, w, x[:2], 1e-6, -1], [x, w, None, 1e-6, 64], [x, w.half(), None, 1e-6, 0], [x[:0], w, None, 1e-6, 0], [x, w, None, None, 0]):
        n = len(native.calls)
        assert native.module.norm(-1, 7, *a) is None and len(native.calls) == n
    native.status = -9
    assert native.module.step(*ok) is None and native.module.norm(-1, 7, x, w, None, 1e-6, 0) is None and native.module.norm_bwd(-1, 7, x, x, w, 1e-6, None) is None
