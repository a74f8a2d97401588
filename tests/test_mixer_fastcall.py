"""The native argument handling of the head norms and the gated recurrence (csrc/fastcall.cpp) without a GPU: host tensors (device -1) and a stand-in for the
C-ABI; what it hands on is what the Python route hands on."""
import contextlib
import ctypes
import importlib.util
import shutil
import types

import pytest
import torch

from paper_2605_21325_amd import binding, mixer
from paper_2605_21325_amd import build as tri_build

P, I, L, F, W = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_float, ctypes.c_uint32
# as in csrc/fastcall.cpp, struct MixerAbi
ABI = {
    "qk_norm_rope": [P] * 8 + [L] * 5 + [I] * 5 + [W, F, P],
    "qk_norm_rope_bwd": [P] * 13 + [L] * 8 + [I] * 5 + [W, F, P],
    "qk_norm_rope_bwd_workspace": [L, I, I, I, P],
    "gated_scan": [P] * 6 + [L, I, L, I] + [L] * 3 + [I, I, W, P],
    "gated_scan_varlen": [P] * 6 + [L, P, I, L, I] + [L] * 3 + [I, I, W, P],
    "gated_scan_workspace": [L, I, I, P],
    "gated_scan_bwd": [P] * 10 + [L, I, L, I] + [L] * 6 + [I, I, W, P],
    "gated_scan_bwd_varlen": [P] * 10 + [L, P, I, L, I] + [L] * 6 + [I, I, W, P],
    "gated_scan_step": [P] * 5 + [I, L, I] + [L] * 3 + [I, I, W, P],
}
bf = torch.bfloat16


class Native:
    def __init__(self, path):
        spec = importlib.util.spec_from_file_location("_fastcall", path)
        self.module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(self.module)
        self.calls, self.status, self.keep = [], 0, []
        for name, args in ABI.items():
            self.keep.append(ctypes.CFUNCTYPE(I, *args)(lambda *a, name=name: self.answer(name, a)))
        self.module.connect_mixer(*(ctypes.cast(f, P).value for f in self.keep))
        self.keep.append(ctypes.CFUNCTYPE(I, P, I, I, L, P, P, P)(self.offsets))
        self.module.connect(*[ctypes.cast(self.keep[0], P).value] * 5, ctypes.cast(self.keep[-1], P).value)

    def offsets(self, lens, n, C, total, at, n_chunk, stream):
        return 0 if sum(ctypes.cast(lens, ctypes.POINTER(L))[:n]) == total else -5

    def answer(self, name, a):
        if name.endswith("workspace"):
            ctypes.cast(a[-1], ctypes.POINTER(L))[0] = 64
        else:
            self.calls.append((name, a))
        return self.status


@pytest.fixture
def native(tmp_path):
    if not tri_build._fastcall_current():
        tri_build.build_fastcall()
    copy = str(tmp_path / "_fastcall.so")
    shutil.copy(tri_build.FASTCALL, copy)
    return Native(copy)


@pytest.fixture
def python(monkeypatch):
    """The Python route's calls of the C-ABI, on host tensors."""
    seen = []

    def entry(name):
        def f(*a):
            if name.endswith("workspace"):
                a[-1]._obj.value = 64
            else:
                seen.append((name, tuple(ctypes.c_float(x).value if isinstance(x, float) else x for x in a)))
            return 0
        return f

    library = type("Library", (), {"__getattr__": lambda self, name: entry(name)})()
    monkeypatch.setattr(binding, "lib", lambda: library)
    for name in ("_dev", "_address"):
        monkeypatch.setattr(mixer, name, lambda t, name: t.data_ptr())
    monkeypatch.setattr(mixer, "_opt", lambda t, name: None if t is None else t.data_ptr())
    monkeypatch.setattr(mixer, "_stream_ptr", lambda stream: 7)
    return seen


def same(native, python, results):
    """One call each, alike but for the memory that each made itself: `results` arguments, in both cases given."""
    (name, a), (other, b) = native.calls[-1], python[-1]
    assert name == other and len(a) == len(b)
    for i, (x, y) in enumerate(zip(a, b)):
        if i in results:
            assert x and y, (name, i)
        else:
            assert x == y, (name, i, x, y)


def heads():
    wide = torch.zeros(2, 5, 700, dtype=bf)
    q, k = wide[..., :256].unflatten(-1, (4, 64)), wide[..., 256:384].unflatten(-1, (2, 64))
    return q, k, torch.zeros(64, dtype=bf), torch.zeros(64, dtype=bf), torch.zeros(2, 5, dtype=torch.int32), torch.zeros(16)


def test_heads(native, python):
    q, k, qw, kw, pos, freq = heads()
    for args in ((q, k, qw, kw, pos, freq), (q, None, None, None, None, None), (q, k, None, kw, pos.long(), freq), (q[:1, :1], k[:1, :1], qw, None, pos[:1, :1], freq),
                 (q.contiguous(), k, qw, kw, None, None)):
        got = native.module.heads(-1, 7, *args, True, False, 1e-6, None, None)
        mixer.qk_norm_rope(*args, unit=True, eps=1e-6)
        same(native, python, {6, 7} if args[1] is not None else {6})
        assert got[0].shape == args[0].shape and got[0].is_contiguous() and (got[1] is None) == (args[1] is None) and native.calls[-1][1][6] == got[0].data_ptr()
    got = native.module.heads(-1, 7, q, k, qw, kw, pos, freq, False, True, 1e-6, q, k)
    mixer.qk_norm_rope(q, k, qw, kw, pos, freq, interleaved=True, q_out=q, k_out=k)
    same(native, python, set())
    assert got[0] is q and got[1] is k
    for args in ((q, k, qw, kw, pos, freq), (q, None, qw, None, None, None), (q, k, None, None, pos.long(), freq)):
        uk = None if args[1] is None else torch.zeros_like(args[1])
        got = native.module.heads_bwd(-1, 7, q, uk, *args, False, True, 1e-5, None, None)
        mixer.qk_norm_rope_bwd(q, uk, *args, interleaved=True, eps=1e-5)
        same(native, python, {i for i, t in ((8, q), (9, args[1]), (10, args[2]), (11, args[3]), (12, args[2])) if t is not None})
        assert [x is None for x in got] == [x is None for x in args[:4]] and all(x is None or x.dtype == torch.float32 for x in got[2:])


def test_scan(native, python):
    wide = torch.zeros(2, 30, 150, dtype=bf)
    x, g, state = wide[..., :64], wide[..., 64:128], torch.zeros(2, 64)
    for a, b, s in ((x, g, state), (x.contiguous(), torch.zeros(2, 30, 64), None)):
        h, final = native.module.scan(-1, 7, a, b, s, True, False, None, None)
        mixer.gated_scan(a, b, s, logit=True)
        same(native, python, {3, 4, 5})
        assert h.shape == a.shape and final.shape == (2, 64) and final.dtype == torch.float32
        got = native.module.scan_bwd(-1, 7, a, b, h, h, s, s, True, True, None, None)
        mixer.gated_scan_bwd(a, b, h, h, s, s, logit=True, mix=True)
        same(native, python, {6, 7, 8, 9} if s is not None else {6, 7, 9})
        assert got[0].dtype == bf and got[1].dtype == b.dtype and (got[2] is None) == (s is None)
        native.module.scan_bwd(-1, 7, None, b, h, h, s, None, False, False, x, None)
        mixer.gated_scan_bwd(None, b, h, h, s, dx=x)
        same(native, python, {7, 8, 9} if s is not None else {7, 9})
    assert native.module.scan(-1, 7, x, g, state, False, True, g, state)[1] is state
    mixer.gated_scan(x, g, state, mix=True, h=g, final_state=state)
    same(native, python, {5})


def test_packed_scan(native, python):
    x, g, state = torch.zeros(30, 64, dtype=bf), torch.zeros(30, 64), torch.zeros(3, 64)
    h, final = native.module.scan_varlen(-1, 7, x, g, [10, 0, 20], state, False, True, None, None)
    mixer.gated_scan_varlen(x, g, [10, 0, 20], state, mix=True)
    same(native, python, {3, 4, 5, 7})
    assert h._triinv_keepalive[0].data_ptr() == final._triinv_keepalive[0].data_ptr() == native.calls[-1][1][7]
    got = native.module.scan_bwd_varlen(-1, 7, x, g, x, x, (30, 0, 0), state, None, False, True, None, None)
    mixer.gated_scan_bwd_varlen(x, g, x, x, (30, 0, 0), state, mix=True)
    same(native, python, {6, 7, 8, 9, 11})
    assert all(t._triinv_keepalive[0].data_ptr() == native.calls[-1][1][11] for t in got)
    assert native.module.scan_varlen(-1, 7, x, g, [10, 21], state[:2], False, True, None, None) is None


def test_step(native, python):
    wide = torch.zeros(5, 200)
    x, g, pool, slots = wide[:, :64], wide[:, 100:164], torch.zeros(9, 64), torch.zeros(5, dtype=torch.int32)
    h = native.module.scan_step(-1, 7, x, g, pool, slots, True, True, None)
    mixer.gated_scan_step(x, g, pool, slots, logit=True, mix=True)
    same(native, python, {4})
    assert h.shape == x.shape and h.is_contiguous()
    assert native.module.scan_step(-1, 7, x, g, pool, None, False, True, h) is h
    mixer.gated_scan_step(x, g, pool, mix=True, h=h)
    same(native, python, set())


def test_what_is_not_plain_goes_back(native):
    """None, and the C-ABI is not called: the Python route says what is wrong."""
    def goes_back(f, ok, changes):
        assert f(*ok) is not None
        for i, bad in changes:
            a, n = list(ok), len(native.calls)
            a[i] = bad
            assert f(*a) is None and len(native.calls) == n, (i, bad)

    q, k, qw, kw, pos, freq = heads()
    goes_back(native.module.heads, [-1, 7, q, k, qw, kw, pos, freq, True, False, 1e-6, None, None],
              ((2, q[:1]), (2, q.double()), (2, q.transpose(0, 1)), (2, q[..., ::2]), (2, None), (2, q[:, :0]), (3, k.half()), (3, k[..., :32]), (3, k[0]), (4, qw[:32]), (4, qw.float()), (5, kw[:0]),
               (6, pos[:1]), (6, pos.float()), (6, None), (7, None), (7, freq.double()), (7, torch.zeros(40)), (7, freq[None]), (8, 1), (9, "x"), (10, None), (11, q[:1]), (11, q.float()), (12, q)))
    goes_back(native.module.heads_bwd, [-1, 7, q, k, q, k, qw, kw, pos, freq, True, False, 1e-6, None, None],
              ((2, q[:1]), (3, None), (3, q), (2, q.half()), (5, None), (13, k), (14, q), (10, None)))
    x, g, state = torch.zeros(2, 30, 64, dtype=bf), torch.zeros(2, 30, 64), torch.zeros(2, 64)
    goes_back(native.module.scan, [-1, 7, x, g, state, True, False, None, None],
              ((2, x[0]), (2, x[:, :29]), (2, x[:, :0]), (2, x.transpose(0, 1)), (3, g.half()), (3, g[..., :3]), (4, state[:1]), (4, state.half()), (5, 1), (6, None), (7, x.float()), (8, state[:, :3])))
    goes_back(native.module.scan_bwd, [-1, 7, x, g, x, x, state, state, True, True, None, None],
              ((2, None), (2, x[:1]), (3, g.double()), (4, x[0]), (5, x[:, :3]), (6, state[0]), (7, state.double()), (8, 0), (10, g), (11, x)))
    goes_back(native.module.scan_varlen, [-1, 7, x[0], g[0], [10, 20], state, True, False, None, None],
              ((2, x), (4, [10, 21]), (4, [10, 10, 10]), (4, [10.0, 20.0]), (4, None), (4, [30]), (4, torch.tensor([10, 20]))))
    step = [-1, 7, x[0], g[0], torch.zeros(40, 64), torch.zeros(30, dtype=torch.int32), True, True, None]
    goes_back(native.module.scan_step, step, ((2, x), (2, x[0, :0]), (3, g[0, :2]), (4, state[:0]), (4, torch.zeros(40, 60)), (4, torch.zeros(40, 64, dtype=bf)), (5, torch.zeros(30, dtype=torch.int64)),
                                              (5, torch.zeros(3, dtype=torch.int32)), (6, 1), (8, x[:, 0])))
    native.status = -9
    assert native.module.scan_step(*step) is None and native.module.scan(-1, 7, x, g, state, True, False, None, None) is None
    assert native.module.heads(-1, 7, q, k, qw, kw, pos, freq, True, False, 1e-6, None, None) is None


class Foreign:
    """A stream object of another library."""

    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.mark.parametrize("which", range(7))
@pytest.mark.parametrize("handle,where", [(0x50, 0x50), (0, "default")])
def test_allocations_belong_to_the_stream_of_the_call(python, monkeypatch, which, handle, where):
    force, seen = [None], []

    @contextlib.contextmanager
    def inside(stream):
        force.append(stream.cuda_stream)
        yield
        force.pop()

    def allocating(make):
        def f(*a, **k):
            seen.append(force[-1])
            return make(*a, **k)
        return f

    q, k, qw, kw, pos, freq = heads()
    x, g, s = torch.zeros(2, 30, 64), torch.zeros(2, 30, 64), torch.zeros(2, 64)
    many = [1] * 30 + [0] * 900
    pool = torch.zeros(30, 64)
    monkeypatch.setattr(torch.cuda, "stream", inside)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: types.SimpleNamespace(cuda_stream=handle))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: types.SimpleNamespace(cuda_stream="default"))
    for name in ("empty", "empty_like", "tensor"):
        monkeypatch.setattr(torch, name, allocating(getattr(torch, name)))
    stream = Foreign(handle)
    [lambda: mixer.qk_norm_rope(q, k, qw, kw, pos, freq, stream=stream), lambda: mixer.qk_norm_rope_bwd(q, k, q, k, qw, kw, pos, freq, stream=stream),
     lambda: mixer.gated_scan(x, g, s, stream=stream), lambda: mixer.gated_scan_varlen(x[0], g[0], many, stream=stream), lambda: mixer.gated_scan_bwd(x, g, x, x, s, s, stream=stream),
     lambda: mixer.gated_scan_bwd_varlen(x[0], g[0], x[0], x[0], many, stream=stream), lambda: mixer.gated_scan_step(x[0], g[0], pool, stream=stream)][which]()
    assert seen and all(at == where for at in seen)
