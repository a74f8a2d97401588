"""On which stream the layer's operators allocate what they drop or hand back: that of their kernels.  Without a GPU: host tensors and a stand-in for the library."""
import contextlib
import types

import pytest
import torch

from paper_2605_21325_amd import binding, layer

bf = torch.bfloat16


class Foreign:
    """A stream object of another library."""

    def __init__(self, handle):
        self.cuda_stream = handle


@pytest.fixture
def log(monkeypatch):
    """(what was allocated, on which stream) and ("launch", stream) in order; the stream in force by its handle, None: the current one."""
    seen, force = [], [None]

    @contextlib.contextmanager
    def inside(stream):
        force.append(stream.cuda_stream)
        yield
        force.pop()

    def allocating(make):
        def f(*a, **k):
            seen.append((make.__name__, force[-1]))
            return make(*a, **k)
        return f

    def entry(name):
        def f(*a):
            if name.endswith("workspace"):
                a[-1]._obj.value = 64
            else:
                seen.append(("launch", None))
            return 0
        return f

    monkeypatch.setattr(torch.cuda, "stream", inside)
    monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, device=None: types.SimpleNamespace(cuda_stream=handle))
    monkeypatch.setattr(torch.cuda, "default_stream", lambda device=None: types.SimpleNamespace(cuda_stream="default"))
    for name in ("empty", "empty_like", "tensor"):
        monkeypatch.setattr(torch, name, allocating(getattr(torch, name)))
    library = type("Library", (), {"__getattr__": lambda self, name: entry(name)})()
    monkeypatch.setattr(binding, "lib", lambda: library)
    monkeypatch.setattr(layer, "_dev", lambda t, name: t.data_ptr())
    monkeypatch.setattr(layer, "_stream_ptr", lambda stream: 1)
    return seen


def calls():
    q, u, g = torch.zeros(1, 70, 2, 64, dtype=bf), torch.zeros(1, 70, 4, 64, dtype=bf), torch.zeros(1, 70, 4)
    lens, many = [30, 40], [1] * 70 + [0] * 900
    x, w = torch.zeros(4, 64), torch.zeros(64)
    return [
        ("attention", lambda s: layer.gdn_chunk_attn(q, q, u, g, 64, stream=s)),
        ("gradient", lambda s: layer.gdn_chunk_attn_bwd(q, q, u, g, u, 64, stream=s)),
        ("packed", lambda s: layer.gdn_chunk_attn_varlen(q[0], q[0], u[0], g[0], lens, 64, stream=s)),
        ("many packed", lambda s: layer.gdn_chunk_attn_varlen(q[0], q[0], u[0], g[0], many, 64, stream=s)),
        ("gradient of packed", lambda s: layer.gdn_chunk_attn_bwd_varlen(q[0], q[0], u[0], g[0], u[0], many, 64, stream=s)),
        ("step", lambda s: layer.gdn_step(q[:, 0], q[:, 0], u[:, 0], g[:, 0], torch.zeros(1, 4, 64, 64), stream=s)),
        ("norm", lambda s: layer.add_rms_norm(x, w, residual=x, stream=s)),
        ("norm in 8 bits", lambda s: layer.add_rms_norm_fp8(x, w, residual=x, stream=s)),
        ("gradient of the norm", lambda s: layer.add_rms_norm_bwd(x, x, w, stream=s)),
    ]


@pytest.mark.parametrize("which", range(9))
@pytest.mark.parametrize("handle,where", [(0x50, 0x50), (0, "default")])
def test_a_stream_of_another_library(log, which, handle, where):
    name, call = calls()[which]
    log.clear()
    call(Foreign(handle))
    made = [s for what, s in log if what != "launch"]
    assert ("launch", None) in log and made and all(s == where for s in made), (name, log)


@pytest.mark.parametrize("which", range(9))
def test_the_current_stream(log, which):
    name, call = calls()[which]
    log.clear()
    call(None)
    assert all(s is None for _, s in log), (name, log)


def test_the_offsets_live_as_long_as_any_result(log):
    u, q, g = torch.zeros(70, 4, 64, dtype=bf), torch.zeros(70, 2, 64, dtype=bf), torch.zeros(70, 4)
    for results in (layer.gdn_chunk_attn_varlen(q, q, u, g, [70], 64), layer.gdn_chunk_attn_bwd_varlen(q, q, u, g, u, [70], 64)):
        assert all(x._triinv_keepalive for x in results if x is not None)


@pytest.mark.gpu
def test_a_foreign_stream_gives_the_same():
    import paper_2605_21325_amd as tri

    gen = torch.Generator(device="cuda").manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")
    side = torch.cuda.Stream()
    q, k, u = rand(64 * 20, 2, 64).to(bf), torch.nn.functional.normalize(rand(64 * 20, 2, 64), dim=-1).to(bf), rand(64 * 20, 2, 64).to(bf)
    w, g = 0.3 * k, None
    few, many = [64 * 19, 64], [64 * 19, 1, 63] + [0] * 950
    for lens in (few, many):
        want = tri.gdn_chunk_attn_varlen(q, k, u, g, lens, 64, W=w)
        grads = tri.gdn_chunk_attn_bwd_varlen(q, k, u, g, u, lens, 64, W=w)
        side.wait_stream(torch.cuda.current_stream())
        got = tri.gdn_chunk_attn_varlen(q, k, u, g, lens, 64, W=w, stream=Foreign(side.cuda_stream))
        back = tri.gdn_chunk_attn_bwd_varlen(q, k, u, g, u, lens, 64, W=w, stream=Foreign(side.cuda_stream))
        side.synchronize()
        for a, b in zip((*want, *grads), (*got, *back)):
            assert (a is None) == (b is None) and (a is None or torch.equal(a, b))
    x, weight = rand(5, 256), rand(256)
    side.wait_stream(torch.cuda.current_stream())
    dx, dw = tri.add_rms_norm_bwd(x, x, weight, stream=Foreign(side.cuda_stream))
    dx0, dw0 = tri.add_rms_norm_bwd(x, x, weight, stream=Foreign(0))
    torch.cuda.synchronize()
    assert torch.equal(dx, dx0) and torch.equal(dw, dw0)
