"""The layer's operators beside the chunk inverse on the GPU against the fp64 statements of oracle/layer.py.

Tolerances.  u is the unit roundoff of the operand type (bf16 2^-8, fp16 2^-11).  What ends in that type is rounded once to it; on the way it
is formed from two-part operands (2^-16 and less) and fp32 sums, so its relative error (2-norm, per token and per head) stays below u; dW is the product
of a rounded factor, 2 u.  What ends in fp32 is a chain of sums of d_k + C products per chunk whose operands carry 24 bits (fp16: 22): at most
(d_k + C) 2^-24 + 2^-21 of the magnitudes that are added up, taken twice for the sums' chain through the chunks.
"""
import numpy as np
import pytest
import torch

import paper_2605_21325_amd as tri
from oracle import layer

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
U_OF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float32: 2.0 ** -24}
BF, HF, F = torch.bfloat16, torch.float16, torch.float32


def exact(x):
    return None if x is None else x.detach().double().cpu().numpy()


def make(lens, H, Hk, d_k, d_v, C, dtype, gate=True, delta=True, state=True, seed=0, rate=0.05):
    """Packed inputs of sequences `lens`: W of the size the chunk inverse gives (unit keys times beta)."""
    gen = torch.Generator(device=DEV).manual_seed(seed + 1)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    total = sum(lens)
    x = dict(q=rand(total, Hk, d_k).to(dtype), k=torch.nn.functional.normalize(rand(total, Hk, d_k), dim=-1).to(dtype), u=rand(total, H, d_v).to(dtype))
    x["w"] = (0.5 * torch.nn.functional.normalize(rand(total, H, d_k), dim=-1)).to(dtype) if delta else None
    if gate:
        r = -rate * torch.nn.functional.softplus(rand(total, H)).double()
        x["g"] = torch.cat([part.cumsum(0) for seq in r.split(lens) for part in (seq.split(C) if len(seq) else [seq])]).float() if total else rand(0, H)
    else:
        x["g"] = None
    x["state"] = rand(len(lens), H, d_k, d_v) if state else None
    x["do"], x["dstate"] = rand(total, H, d_v).to(dtype), rand(len(lens), H, d_k, d_v) if state else None
    return x


def close(got, ref, tol, what, size=None):
    """2-norm over the last axis against `tol` of the reference's (or of `size`), with the rounding of what is far below the rest left out; and over everything."""
    got, size = exact(got), np.abs(ref) if size is None else size
    assert got.shape == ref.shape, what
    assert np.isfinite(got).all(), f"{what}: not finite"
    err = np.linalg.norm(got - ref, axis=-1)
    floor = np.sqrt((size ** 2).mean()) * np.sqrt(ref.shape[-1]) * 0.05
    worst = (err / (tol * np.maximum(np.linalg.norm(size, axis=-1), floor) + 1e-30)).max() if ref.size else 0.0
    assert worst <= 1.0, f"{what}: {worst:.2f} of the tolerance"


def tol32(d_k, C):
    return 2 * ((d_k + C) * 2.0 ** -24 + 2.0 ** -21)


def split(x, lens, s):
    a = sum(lens[:s])
    return None if x is None else exact(x[a:a + lens[s]])


def check_forward(o, final, x, lens, C, scale, dtype):
    for s in range(len(lens)):
        part = {n: split(x[n], lens, s) for n in ("q", "k", "u", "w", "g")}
        ro, rf = layer.chunk_attn(part["q"], part["k"], part["u"], part["w"], part["g"], C, None if x["state"] is None else exact(x["state"][s]), scale)
        a = sum(lens[:s])
        if lens[s]:
            close(o[a:a + lens[s]], ro, U_OF[dtype], f"O of sequence {s}")
        # (per head, not per row of the state: its rows are sums of the same length, of which some cancel)
        close(final[s].flatten(1), rf.reshape(rf.shape[0], -1), tol32(x["q"].shape[-1], C), f"state of sequence {s}")


CASES = [
    # lens, H, Hk, d_k, d_v, C, dtype, gate, delta, state
    ([1], 1, 1, 64, 64, 64, BF, True, True, True),
    ([1], 2, 1, 128, 128, 64, HF, True, False, False),
    ([64], 2, 2, 128, 128, 64, BF, True, True, False),
    ([65], 3, 3, 64, 64, 64, BF, True, True, True),
    ([200], 4, 2, 128, 128, 64, BF, True, True, True),
    ([200], 4, 1, 128, 128, 64, HF, True, True, True),
    ([131], 2, 2, 128, 64, 64, BF, False, True, True),
    ([131], 2, 2, 64, 128, 64, HF, False, False, True),
    ([100], 2, 2, 32, 8, 64, BF, True, True, True),
    ([100], 2, 1, 96, 72, 64, HF, True, True, True),
    ([90], 2, 2, 64, 24, 64, BF, True, False, False),
    ([70], 1, 1, 128, 264, 64, BF, True, True, True),
    ([70], 1, 1, 32, 512, 64, HF, True, True, False),
    ([17, 1, 0, 64, 129], 2, 1, 64, 64, 64, BF, True, True, True),
    ([0, 63, 0], 2, 2, 128, 128, 64, HF, True, False, True),
    ([40, 16, 33], 2, 2, 64, 64, 16, BF, True, True, True),
    ([70], 2, 1, 128, 72, 16, HF, True, True, False),
    ([50, 31], 2, 2, 128, 64, 32, BF, True, False, True),
    ([97], 2, 2, 64, 40, 32, HF, True, True, True),
    ([128, 1, 300], 2, 2, 128, 128, 128, BF, True, True, True),
    ([190], 4, 2, 64, 64, 128, HF, True, True, True),
    ([257], 1, 1, 128, 64, 128, HF, False, False, False),
    ([130], 2, 1, 96, 40, 128, BF, True, False, True),
]


@pytest.mark.parametrize("lens,H,Hk,d_k,d_v,C,dtype,gate,delta,state", CASES)
def test_chunk_attention(lens, H, Hk, d_k, d_v, C, dtype, gate, delta, state):
    x = make(lens, H, Hk, d_k, d_v, C, dtype, gate, delta, state)
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, W=x["w"], state=x["state"], scale=0.3)
    check_forward(o, final, x, lens, C, 0.3, dtype)
    if len(lens) == 1:  # the same as one sequence of the fixed layout, bit for bit
        one = {n: None if x[n] is None else x[n][None] for n in ("q", "k", "u", "w", "g")}
        o1, final1 = tri.gdn_chunk_attn(one["q"], one["k"], one["u"], one["g"], C, W=one["w"], state=x["state"], scale=0.3)
        assert torch.equal(o1[0], o) and torch.equal(final1, final)


@pytest.mark.parametrize("lens,H,Hk,d_k,d_v,C,dtype,gate,delta,state", CASES)
def test_gradient(lens, H, Hk, d_k, d_v, C, dtype, gate, delta, state):
    x = make(lens, H, Hk, d_k, d_v, C, dtype, gate, delta, state)
    got = tri.gdn_chunk_attn_bwd_varlen(x["q"], x["k"], x["u"], x["g"], x["do"], lens, C, W=x["w"], state=x["state"], dstate=x["dstate"], scale=0.3)
    u, t32 = U_OF[dtype], tol32(d_k + d_v, C)  # (products over d_v as well)
    for s, n in enumerate(lens):
        part = {m: split(x[m], lens, s) for m in ("q", "k", "u", "w", "g", "do")}
        ref = layer.chunk_attn_bwd(part["q"], part["k"], part["u"], part["w"], part["g"], C, None if x["state"] is None else exact(x["state"][s]), 0.3, part["do"],
                                   None if x["dstate"] is None else exact(x["dstate"][s]))
        a = sum(lens[:s])
        for name, mine, r, tol in zip(("dQ", "dK", "dU", "dW"), got[:4], ref[:4], (u, u, u, 2 * u)):
            assert (mine is None) == (r is None)
            if r is not None and n:
                close(mine[a:a + n], r, tol, f"{name} of sequence {s}")
        if gate and n:  # dg is a difference of <q, dQ> and <k, dK>: against the sizes of what they are summed from, per head and chunk
            rep = H // Hk
            heads = [layer.chunk_attn_bwd(part["q"][:, h // rep:h // rep + 1], part["k"][:, h // rep:h // rep + 1], part["u"][:, h:h + 1], None if part["w"] is None else part["w"][:, h:h + 1],
                                          part["g"][:, h:h + 1], C, None if x["state"] is None else exact(x["state"][s, h:h + 1]), 0.3, part["do"][:, h:h + 1],
                                          None if x["dstate"] is None else exact(x["dstate"][s, h:h + 1])) for h in range(H)]
            size = np.stack([(np.abs(part["q"][:, h // rep] * r[0][:, 0]) + np.abs(part["k"][:, h // rep] * r[1][:, 0])).sum(-1) for h, r in enumerate(heads)])
            arrives = np.zeros(H) if x["dstate"] is None else np.linalg.norm(exact(x["dstate"][s]), axis=(1, 2))
            _, final = layer.chunk_attn(part["q"], part["k"], part["u"], part["w"], part["g"], C, None if x["state"] is None else exact(x["state"][s]), 0.3)
            last = (np.linalg.norm(final, axis=(1, 2)) * arrives)[:, None] / np.sqrt(d_k * d_v)
            close(got[4][a:a + n].T, ref[4].T, t32, f"dg of sequence {s}", size + last + np.abs(ref[4].T))
        if state:
            close(got[5][s].flatten(1), ref[5].reshape(H, -1), t32, f"gradient of the state of sequence {s}")
    if len(lens) == 1:
        one = {m: None if x[m] is None else x[m][None] for m in ("q", "k", "u", "w", "g", "do")}
        same = tri.gdn_chunk_attn_bwd(one["q"], one["k"], one["u"], one["g"], one["do"], C, W=one["w"], state=x["state"], dstate=x["dstate"], scale=0.3)
        for p, q in zip(same, got):
            assert (p is None) == (q is None) and (p is None or torch.equal(p.reshape(q.shape), q))


@pytest.mark.parametrize("delta", [True, False])
def test_gradient_against_differences(delta):
    """The final state is fp32: its directional derivatives by the two fp32 inputs, from the forward kernel itself."""
    C, lens = 64, [150]
    x = make(lens, 2, 2, 64, 64, C, BF, True, delta, True, seed=3)
    gen = torch.Generator(device=DEV).manual_seed(5)
    zero = torch.zeros_like(x["do"])
    got = tri.gdn_chunk_attn_bwd_varlen(x["q"], x["k"], x["u"], x["g"], zero, lens, C, W=x["w"], state=x["state"], dstate=x["dstate"])

    def loss(g, state):
        _, f = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], g, lens, C, W=x["w"], state=state)
        return (f.double() * x["dstate"].double()).sum().item(), f.double().norm().item() * x["dstate"].double().norm().item()

    for name, grad in (("g", got[4]), ("state", got[5])):
        d = torch.randn(x[name].shape, generator=gen, device=DEV)
        e = 2.0 ** -6
        up, size = loss(**{**{"g": x["g"], "state": x["state"]}, name: x[name] + e * d})
        dn, _ = loss(**{**{"g": x["g"], "state": x["state"]}, name: x[name] - e * d})
        # the states' rounding over the step, and in g the third-order remainder (d^3 of exp, at most e^2 max|d|^2 of the derivative's own size)
        bound = 2 * tol32(64, C) * size / (2 * e) + (e * e * d.abs().max().item() ** 2 * (grad * d).abs().sum().item() if name == "g" else 0.0)
        assert abs((up - dn) / (2 * e) - (grad.double() * d.double()).sum().item()) <= bound, name


@pytest.mark.parametrize("delta,dtype", [(True, BF), (False, BF), (True, HF), (False, HF)])
def test_segments(delta, dtype):
    """Few heads and many chunks: the sequence is taken in segments, with one result."""
    lens, C = [16 * 70 + 5], 16
    x = make(lens, 2, 1, 64, 72, C, dtype, True, delta, True, seed=7, rate=0.02)
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, W=x["w"], state=x["state"], scale=0.3)
    check_forward(o, final, x, lens, C, 0.3, dtype)
    lens = [16 * 60, 3, 0, 16 * 150 + 1]  # shares of a long one and of short ones
    x = make(lens, 1, 1, 128, 64, C, dtype, True, delta, False, seed=8, rate=0.02)
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, W=x["w"], scale=0.3)
    check_forward(o, final, x, lens, C, 0.3, dtype)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_strong_decay_and_large_states(dtype):
    """A decay that falls by hundreds within a chunk underflows to zero and nothing else; states far beyond fp16's range are states like others."""
    lens, C = [150], 64
    x = make(lens, 2, 2, 64, 64, C, dtype, True, True, True, seed=9, rate=8.0)
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, W=x["w"], state=x["state"], scale=0.3)
    check_forward(o, final, x, lens, C, 0.3, dtype)
    assert all(torch.isfinite(t).all() for t in tri.gdn_chunk_attn_bwd_varlen(x["q"], x["k"], x["u"], x["g"], x["do"], lens, C, W=x["w"], state=x["state"], dstate=x["dstate"]))
    x = make(lens, 2, 2, 64, 64, C, dtype, True, False, True, seed=10)
    x["state"] = x["state"] * 1e6
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, state=x["state"], scale=1e-4)
    check_forward(o, final, x, lens, C, 1e-4, dtype)


def test_non_finite_values_stay_in_their_head_and_behind_their_chunk():
    lens, C = [200, 100], 64
    x = make(lens, 3, 3, 64, 64, C, BF, True, True, True, seed=11)
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, W=x["w"], state=x["state"])
    for name, bad in (("u", float("nan")), ("k", float("inf")), ("g", float("nan"))):
        y = dict(x, **{name: x[name].clone()})
        y[name][130, 1] = bad  # third chunk of the first sequence, head 1
        p, f = tri.gdn_chunk_attn_varlen(y["q"], y["k"], y["u"], y["g"], lens, C, W=y["w"], state=y["state"])
        keep = torch.ones(300, 3, dtype=torch.bool, device=DEV)
        keep[128:200, 1] = False
        assert torch.equal(p[keep], o[keep]) and not torch.isfinite(p[130:200, 1]).all()
        assert torch.equal(f[:, [0, 2]], final[:, [0, 2]]) and torch.equal(f[1], final[1]) and not torch.isfinite(f[0, 1]).all()


def test_a_sequence_does_not_depend_on_the_others_of_its_call():
    lens, C = [64, 130, 7], 64
    x = make(lens, 70, 70, 64, 64, C, BF, seed=12)
    o, final = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, C, W=x["w"], state=x["state"])
    at = 0
    for s, n in enumerate(lens):
        part = {m: x[m][at:at + n].contiguous() for m in ("q", "k", "u", "w", "g")}
        o1, f1 = tri.gdn_chunk_attn_varlen(part["q"], part["k"], part["u"], part["g"], [n], C, W=part["w"], state=x["state"][s:s + 1].contiguous())
        assert torch.equal(o1, o[at:at + n]) and torch.equal(f1[0], final[s])
        at += n


def test_rows_beyond_four_gigabytes():
    """A short sequence behind one of 5 GB a tensor."""
    H, d, C = 32, 128, 64
    long, short = 640 * 1024, 100
    x = make([short], H, H, d, d, C, BF, gate=True, seed=13)
    big = {n: torch.zeros(long + short, H, d, dtype=BF, device=DEV) for n in ("q", "k", "u", "w")}
    g = torch.zeros(long + short, H, device=DEV)
    for n in big:
        big[n][long:] = x[n]
    g[long:] = x["g"]
    state = torch.cat([torch.zeros_like(x["state"]), x["state"]])
    o, f = tri.gdn_chunk_attn_varlen(big["q"], big["k"], big["u"], g, [long, short], C, W=big["w"], state=state)
    assert not o[:long].any()
    check_forward(o[long:], f[1:], x, [short], C, d ** -0.5, BF)


def test_state_in_place_on_another_stream_and_in_a_graph():
    lens, C = [100], 64
    x = make(lens, 2, 2, 64, 64, C, BF, seed=14)
    one = {n: x[n][None].contiguous() for n in ("q", "k", "u", "w", "g")}
    o, final = tri.gdn_chunk_attn(one["q"], one["k"], one["u"], one["g"], C, W=one["w"], state=x["state"])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    state = x["state"].clone()
    with torch.cuda.stream(side):
        o1, _ = tri.gdn_chunk_attn(one["q"], one["k"], one["u"], one["g"], C, W=one["w"], state=state, final_state=state)
    o2, f2 = tri.gdn_chunk_attn(one["q"], one["k"], one["u"], one["g"], C, W=one["w"], state=x["state"], stream=side)
    side.synchronize()
    assert torch.equal(o1, o) and torch.equal(state, final) and torch.equal(o2, o) and torch.equal(f2, final)
    # a captured call, replayed with other work in between
    run = lambda s: tri.gdn_chunk_attn(one["q"], one["k"], one["u"], one["g"], C, W=one["w"], state=s, final_state=s)[0]
    state, eager = x["state"].clone(), x["state"].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(state)
    for _ in range(3):
        graph.replay()
        want = run(eager)
        torch.cuda.synchronize()
        assert torch.equal(out, want) and torch.equal(state, eager)


@pytest.mark.parametrize("B,H,Hk,d_k,d_v,dtype,gate,delta,pool", [
    (1, 1, 1, 64, 64, BF, True, True, 0), (1, 16, 16, 128, 128, BF, True, True, 3), (3, 4, 2, 128, 64, HF, True, True, 5), (2, 2, 1, 100, 20, BF, True, True, 0),
    (5, 2, 2, 256, 512, F, True, True, 9), (2, 3, 1, 1, 4, F, False, True, 0), (70, 32, 16, 64, 132, BF, True, False, 80), (2, 2, 2, 37, 128, HF, False, False, 4),
    (40, 32, 32, 128, 128, F, True, True, 41)])
def test_step(B, H, Hk, d_k, d_v, dtype, gate, delta, pool):
    gen = torch.Generator(device=DEV).manual_seed(B)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    q, k, v = rand(B, Hk, d_k).to(dtype), torch.nn.functional.normalize(rand(B, Hk, d_k), dim=-1).to(dtype), rand(B, H, d_v).to(dtype)
    g, beta = -rand(B, H).abs() if gate else None, torch.sigmoid(rand(B, H)) if delta else None
    state = rand(pool or B, H, d_k, d_v)
    slots = torch.randperm(pool, generator=gen, device=DEV)[:B].int() if pool else None
    before, places = state.clone(), list(range(B)) if slots is None else slots.tolist()
    if slots is not None and B > 1:  # two that are padding
        slots[0], slots[1] = -1, pool
        places[0] = places[1] = None
    o = tri.gdn_step(q, k, v, g, state, beta=beta, slots=slots, scale=0.4)
    left = torch.ones(state.shape[0], dtype=torch.bool)
    for b in list(range(min(B, 6))) + [B - 1]:
        if places[b] is None:
            assert not o[b].any()
            continue
        ro, rs = layer.step(exact(q[b]), exact(k[b]), exact(v[b]), None if g is None else exact(g[b]), None if beta is None else exact(beta[b]), exact(before[places[b]]), 0.4)
        # sums of d_k products in fp32, twice
        close(o[b], ro, U_OF[dtype] + 4 * d_k * 2.0 ** -24, f"o of {b}")
        close(state[places[b]].flatten(1), rs.reshape(H, -1), 4 * (d_k + 2) * 2.0 ** -24, f"state of {b}")
    for p in places:
        if p is not None:
            left[p] = False
    assert torch.equal(state[left.to(DEV)], before[left.to(DEV)])


def test_step_follows_the_chunks():
    """A prompt by chunks (keys, inverse applied, attention) and the same prompt token by token."""
    B, T, H, d, C = 1, 70, 2, 64, 64
    gen = torch.Generator(device=DEV).manual_seed(21)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    Q, K, V = rand(B, T, H, d).to(BF), torch.nn.functional.normalize(rand(B, T, H, d), dim=-1).to(BF), rand(B, T, H, d).to(BF)
    beta, rate = torch.sigmoid(rand(B, T, H)), -0.05 * torch.rand(B, T, H, generator=gen, device=DEV)
    g = torch.cat([r.cumsum(1) for r in rate.split(C, 1)], 1).contiguous()
    U, W = tri.gdn_chunk_tri_solve_multi(K, beta, g, [V, K], C, row_scales=[beta, (beta * torch.exp(g)).contiguous()])
    O, final = tri.gdn_chunk_attn(Q, K, U, g, C, W=W)
    state = torch.zeros(B, H, d, d, device=DEV)
    outs = [tri.gdn_step(Q[:, t].contiguous(), K[:, t].contiguous(), V[:, t].contiguous(), rate[:, t].contiguous(), state, beta=beta[:, t].contiguous()) for t in range(T)]
    # U and W come out of the inverse in bf16: the tolerance of the inverse with 16-bit operands
    for x, y in ((O.float(), torch.stack(outs, 1).float()), (final, state)):
        assert (x - y).norm() <= 2e-2 * y.norm()


@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("N,D", [(1, 8), (3, 72), (5, 512), (2, 520), (3, 2048), (4, 4104), (2, 8192), (3, 16384), (2050, 136), (2051, 2048), (2049, 1024)])
def test_norm(N, D, dtype):
    gen = torch.Generator(device=DEV).manual_seed(N + D)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    x, r, w = rand(N, D).to(dtype), (3 * rand(N, D)).to(dtype), (1 + 0.2 * rand(D)).to(dtype)
    x[-1], r[-1] = 0, 0  # a row of zeros
    rows = sorted({0, N // 2, N - 1})
    u = U_OF[dtype]
    for residual in (None, r):
        y, s = tri.add_rms_norm(x, w, residual=residual, eps=1e-5)
        assert (s is x) if residual is None else torch.equal(s, x + r)
        ref = layer.rms_norm(exact(s[rows]), exact(w), 1e-5)
        # one rounding to the type; the fp32 sum of squares (halved by the root) and three products
        bound = u * np.abs(ref) + (D / 2 ** 10 + 8) * 2.0 ** -24 * np.abs(ref)
        assert (np.abs(exact(y[rows]) - ref) <= bound + (2.0 ** -25 if dtype == HF else 1e-38)).all()
        for group in (0, 128) if D % 128 == 0 else (0,):
            q, scales, s2 = tri.add_rms_norm_fp8(x, w, residual=residual, eps=1e-5, group=group)
            assert torch.equal(s2, s) and scales.shape == (N, D // group if group else 1) and q.dtype == torch.float8_e4m3fn
            z = ref.reshape(len(rows), -1, group or D)
            want = np.abs(z).max(-1) / 448
            want[want == 0] = 1
            np.testing.assert_allclose(exact(scales[rows]), want, rtol=(D / 2 ** 10 + 16) * 2.0 ** -24)
            got = exact(q[rows].float()).reshape(z.shape) * exact(scales[rows])[..., None]
            # half a step of 8 bits: 2^-4 of the value, or of the smallest normal value's step below 2^-6
            assert (np.abs(got - z) <= (2.0 ** -4 + 1e-5) * np.maximum(np.abs(z), 2.0 ** -6 * want[..., None])).all()
            assert N == 1 or np.abs(exact(q[rows[:-1]].float())).max() == 448


def test_norm_of_rows_that_are_not_finite():
    x, w = torch.randn(4, 256, device=DEV).to(BF), torch.ones(256, device=DEV, dtype=BF)
    x[1, 3], x[2, 200] = float("nan"), float("inf")
    y, _ = tri.add_rms_norm(x, w)
    assert torch.isfinite(y[[0, 3]].float()).all() and torch.isnan(y[1].float()).all()
    assert torch.isnan(y[2, 200].float())  # inf / inf; the other elements are 0
    for group in (0, 128):
        q, scales, _ = tri.add_rms_norm_fp8(x, w, group=group)
        assert torch.isfinite(q[[0, 3]].float()).all() and torch.isfinite(scales[[0, 3]]).all()
        assert torch.isnan(q[1].float()).all() and torch.isnan(scales[1]).all() and torch.isnan(q[2, 200].float())


@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("N,D", [(1, 8), (3, 72), (700, 512), (2, 520), (513, 2048), (5, 4104), (2, 8192), (3, 16384)])
def test_norm_gradient(N, D, dtype):
    gen = torch.Generator(device=DEV).manual_seed(N + D)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    s, w, dy, more = rand(N, D).to(dtype), (1 + 0.2 * rand(D)).to(dtype), rand(N, D).to(dtype), rand(N, D).to(dtype)
    ds, dw = layer.rms_norm_bwd(exact(dy), exact(s), exact(w), 1e-5)
    for dsum in (None, more):
        dx, dweight = tri.add_rms_norm_bwd(dy, s, w, eps=1e-5, dsum=dsum)
        close(dx, ds if dsum is None else ds + exact(more), U_OF[dtype] + 16 * 2.0 ** -24, "dx")
        # per column a sum of N products in fp32
        size = np.abs(exact(dy) * exact(s)).sum(0)
        assert (np.abs(exact(dweight) - dw) <= (N + 32) * 2.0 ** -24 * size * 3).all()
        again = tri.add_rms_norm_bwd(dy, s, w, eps=1e-5, dsum=dsum)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dweight)


def test_state_pool_beyond_four_gigabytes():
    n, H, d = 20000, 4, 128
    state = torch.zeros(n, H, d, d, device=DEV)  # 5.2 GB
    gen = torch.Generator(device=DEV).manual_seed(2)
    rand = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    q, k, v = rand(2, H, d).to(BF), rand(2, H, d).to(BF), rand(2, H, d).to(BF)
    o = tri.gdn_step(q, k, v, None, state, slots=torch.tensor([n - 1, 0], dtype=torch.int32, device=DEV), scale=1.0)
    for b, slot in ((0, n - 1), (1, 0)):
        ro, rs = layer.step(exact(q[b]), exact(k[b]), exact(v[b]), None, None, np.zeros((H, d, d)), 1.0)
        close(o[b], ro, 2.0 ** -8 + 4 * d * 2.0 ** -24, "o")
        close(state[slot].flatten(1), rs.reshape(H, -1), 2.0 ** -23, "state")
    assert not state[1:n - 1].any()


@pytest.mark.parametrize("n_seq, H, Hk, delta", [(43, 4, 4, True), (43, 4, 2, False), (256, 1, 1, True), (257, 1, 1, True), (8, 17, 17, True)])
def test_many_packed_sequences_begin_with_the_longest_and_give_the_same(n_seq, H, Hk, delta):
    """More workgroups than compute units: sequences are taken by length, empty and equal ones among them.  Bit for bit what each gives alone."""
    lens = [(97 * i * i + 31 * (i % 5)) % 331 if i % 6 else (0 if i % 4 else 128) for i in range(n_seq)]
    x = make(lens, H, Hk, 128, 128, 64, BF, delta=delta, seed=5)
    o, fin = tri.gdn_chunk_attn_varlen(x["q"], x["k"], x["u"], x["g"], lens, 64, W=x["w"], state=x["state"])
    grads = tri.gdn_chunk_attn_bwd_varlen(x["q"], x["k"], x["u"], x["g"], x["do"], lens, 64, W=x["w"], state=x["state"], dstate=x["dstate"])
    at = 0
    for s, n in enumerate(lens):
        if s % max(1, n_seq // 24) == 0 or n == max(lens):
            part = lambda t: None if t is None else t[at:at + n].contiguous()
            own = lambda t: t[s:s + 1].contiguous()
            one, last = tri.gdn_chunk_attn_varlen(part(x["q"]), part(x["k"]), part(x["u"]), part(x["g"]), [n], 64, W=part(x["w"]), state=own(x["state"]))
            assert torch.equal(one, o[at:at + n]) and torch.equal(last, fin[s:s + 1]), (s, n)
            alone = tri.gdn_chunk_attn_bwd_varlen(part(x["q"]), part(x["k"]), part(x["u"]), part(x["g"]), part(x["do"]), [n], 64, W=part(x["w"]), state=own(x["state"]), dstate=own(x["dstate"]))
            for i, (got, want) in enumerate(zip(grads, alone)):
                if want is not None:
                    assert torch.equal(got[s:s + 1] if i == 5 else got[at:at + n], want), (s, n, i)
        at += n
