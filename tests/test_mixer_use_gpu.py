"""The head norms and the gated recurrence as programs use them: captured, on other streams, in long sequences cut into segments, on large buffers, the same call twice, in the example.
Tolerances as in test_mixer_gpu.py."""
import pytest
import torch

import paper_2605_21325_amd as tri
from examples import mixed_delta_layer as example
from tests.test_mixer_gpu import BF, DEV, F, HF, check_heads, check_heads_bwd, check_scan, check_scan_bwd, make_heads, make_scan

pytestmark = pytest.mark.gpu


def calls(seed=0):
    """One call of each entry point, by name: (function of nothing, tensors whose values may change between calls)."""
    x, up = make_heads(3000, 4, 2, 64, 32, True, BF, seed=seed)
    v, dv = make_scan([700, 0, 1300], 96, BF, BF, True, seed=seed)
    f, df = make_scan([500] * 3, 64, HF, F, False, packed=False, seed=seed)
    s, _ = make_scan([40], 128, BF, BF, True, seed=seed)
    pool, slots = torch.randn(50, 128, device=DEV), torch.arange(40, dtype=torch.int32, device=DEV)
    h, hf = tri.gated_scan_varlen(**v, seqlens=[700, 0, 1300], logit=True, mix=True)[0], tri.gated_scan(**f)[0]
    changing = [x["q"], up["dq_out"], v["x"], dv["dh"], f["x"], df["dh"], s["x"]]

    def step():
        held = pool.clone()
        return tri.gated_scan_step(s["x"], s["g"], held, slots, logit=True, mix=True), held

    return {
        "heads": lambda: tri.qk_norm_rope(**x), "heads_bwd": lambda: tri.qk_norm_rope_bwd(**up, **x),
        "scan_varlen": lambda: tri.gated_scan_varlen(**v, seqlens=[700, 0, 1300], logit=True, mix=True), "scan": lambda: tri.gated_scan(**f),
        "scan_bwd_varlen": lambda: tri.gated_scan_bwd_varlen(v["x"], v["g"], h, dv["dh"], [700, 0, 1300], v["state"], dv["dstate"], logit=True, mix=True),
        "scan_bwd": lambda: tri.gated_scan_bwd(None, f["g"], hf, df["dh"], f["state"], df["dstate"]), "scan_step": step}, changing


NAMES = ["heads", "heads_bwd", "scan_varlen", "scan", "scan_bwd_varlen", "scan_bwd", "scan_step"]


@pytest.mark.parametrize("name", NAMES)
def test_captured_and_replayed(name):
    """Two graphs of one pool, replayed in turn with other values and with the program's own calls between them."""
    fs, changing = calls()
    f = fs[name]
    f()
    torch.cuda.synchronize()
    pool = torch.cuda.graph_pool_handle()
    graphs, outs = [], []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=pool):
            outs.append(f())
        graphs.append(g)
    gen = torch.Generator(device=DEV).manual_seed(9)
    for _ in range(3):
        for t in changing:
            t.copy_(torch.randn(t.shape, generator=gen, device=DEV))
        want = f()
        for g, out in zip(graphs, outs):
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(out, want) if b is not None)


@pytest.mark.parametrize("name", NAMES)
def test_on_another_stream_and_twice(name):
    fs, _ = calls()
    want = fs[name]()
    again = fs[name]()
    side = [torch.cuda.Stream(), torch.cuda.Stream()]
    got = []
    torch.cuda.synchronize()
    for s in side:
        with torch.cuda.stream(s):
            got.append(fs[name]())
    torch.cuda.synchronize()
    for r in [again, *got]:
        assert all(torch.equal(a, b) for a, b in zip(r, want) if b is not None)


def test_a_stream_as_an_argument():
    s = torch.cuda.Stream()
    x, _ = make_heads(100, 4, 2, 64, 64, True, BF)
    v, _ = make_scan([300, 200], 64, BF, BF, True)
    want, kept = tri.qk_norm_rope(**x), tri.gated_scan_varlen(**v, seqlens=[300, 200], logit=True)
    torch.cuda.synchronize()
    got, more = tri.qk_norm_rope(**x, stream=s), tri.gated_scan_varlen(**v, seqlens=[300, 200], logit=True, stream=s)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip((*got, *more), (*want, *kept)))


@pytest.mark.parametrize("lens,D,dtype,gtype,logit,mix", [
    ([1500], 4480, F, F, True, True), ([3000, 5, 0, 700], 1000, BF, BF, True, False), ([2600, 2600], 320, BF, F, False, True), ([1100] * 4, 2048, HF, HF, False, False), ([385], 64, F, F, False, False),
    ([769, 0, 0, 1], 128, BF, BF, True, True), ([5000], 33, HF, F, False, True), ([70000, 3], 16, BF, BF, True, True)])
def test_sequences_in_segments(lens, D, dtype, gtype, logit, mix):
    v, up = make_scan(lens, D, dtype, gtype, logit)
    got = tri.gated_scan_varlen(**v, seqlens=lens, logit=logit, mix=mix)
    check_scan(lens, v, got, logit, mix)
    check_scan_bwd(lens, v, got[0], up, tri.gated_scan_bwd_varlen(v["x"], v["g"], got[0], up["dh"], lens, v["state"], up["dstate"], logit=logit, mix=mix), logit, mix)
    state = v["state"].clone()
    again, same = tri.gated_scan_varlen(v["x"], v["g"], lens, state, logit=logit, mix=mix, final_state=state)
    assert torch.equal(again, got[0]) and torch.equal(state, got[1])


@pytest.mark.parametrize("lens,D,dtype,gtype,logit,mix", [
    ([(37 * i) % 50 * 7 for i in range(24)], 1000, BF, BF, True, True), ([(11 * i) % 17 for i in range(100)], 256, HF, F, False, False), ([5] * 127 + [300], 320, F, F, True, False),
    ([i % 3 for i in range(1000)], 64, BF, F, False, True), ([0] * 20 + [130] + [0] * 20 + [1], 1024, BF, BF, True, True),
    ([(29 * i) % 300 for i in range(50)], 510, F, F, True, True), ([(29 * i) % 270 for i in range(52)], 512, HF, F, False, True), ([257] * 260, 66, HF, HF, True, False),
    ([256, 255] * 130, 128, BF, BF, True, True), ([1] * 30 + [700] + [0] * 10 + [3], 512, BF, BF, True, True), ([1] * 30 + [700] + [0] * 10 + [3], 130, F, F, False, False)])
def test_many_packed_sequences(lens, D, dtype, gtype, logit, mix):
    """Where the longest begin, and beyond."""
    v, up = make_scan(lens, D, dtype, gtype, logit)
    got = tri.gated_scan_varlen(**v, seqlens=lens, logit=logit, mix=mix)
    check_scan(lens, v, got, logit, mix)
    check_scan_bwd(lens, v, got[0], up, tri.gated_scan_bwd_varlen(v["x"], v["g"], got[0], up["dh"], lens, v["state"], up["dstate"], logit=logit, mix=mix), logit, mix)


@pytest.mark.parametrize("N,H,Hk,d,rot,inter,dtype", [(4200, 2, 1, 64, 16, False, BF), (6001, 1, 1, 32, 8, True, HF), (4100, 3, 2, 128, 0, False, F), (9000, 1, 0, 16, 0, False, BF), (2100, 5, 1, 96, 0, True, BF),
                                                      (3154, 4, 2, 80, 0, True, BF), (30011, 1, 1, 32, 0, False, HF), (333, 3, 1, 48, 16, False, F), (40, 1, 1, 64, 64, True, BF), (700, 7, 3, 512, 512, True, BF)])
def test_several_tokens_to_a_wavefront(N, H, Hk, d, rot, inter, dtype):
    x, up = make_heads(N, H, Hk, d, rot, True, dtype)
    check_heads(x, tri.qk_norm_rope(**x, interleaved=inter), False, inter)
    check_heads_bwd(x, up, tri.qk_norm_rope_bwd(**up, **x, interleaved=inter), False, inter)


def test_offsets_beyond_4_gb():
    """Columns of rows that lie 2^18 elements apart: 10000 tokens of 5 GB, and a pool of states of 5 GB."""
    N = 10000
    wide = torch.zeros(N, 1 << 18, dtype=BF, device=DEV)
    x, _ = make_heads(N, 2, 1, 64, 16, True, BF)
    q, k = wide[:, -192:-64].view(N, 2, 64), wide[:, -64:].view(N, 1, 64)
    q.copy_(x["q"]), k.copy_(x["k"])
    want = tri.qk_norm_rope(**x)
    assert all(torch.equal(a, b) for a, b in zip(tri.qk_norm_rope(**dict(x, q=q, k=k)), want))
    tri.qk_norm_rope(**x, q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    v, up = make_scan([N - 100, 100], 64, BF, BF, True)
    a, b = wide[:, -320:-256], wide[:, -256:-192]
    a.copy_(v["x"]), b.copy_(v["g"])
    h, final = tri.gated_scan_varlen(**v, seqlens=[N - 100, 100], logit=True, mix=True)
    got, last = tri.gated_scan_varlen(a, b, [N - 100, 100], v["state"], logit=True, mix=True, h=wide[:, -384:-320])
    assert torch.equal(got, h) and torch.equal(last, final)
    dx, dg, d0 = tri.gated_scan_bwd_varlen(v["x"], v["g"], h, up["dh"], [N - 100, 100], v["state"], logit=True, mix=True)
    ox, og, o0 = tri.gated_scan_bwd_varlen(a, b, got, up["dh"], [N - 100, 100], v["state"], logit=True, mix=True, dx=wide[:, -448:-384], dg=wide[:, -512:-448])
    assert torch.equal(ox, dx) and torch.equal(og, dg) and torch.equal(o0, d0)
    del wide, q, k, a, b, got, ox, og
    pool = torch.zeros(20000, 1 << 16, device=DEV)
    one, _ = make_scan([2], 1 << 16, BF, BF, True)
    h = tri.gated_scan_step(one["x"], one["g"], pool, torch.tensor([19999, 1], dtype=torch.int32, device=DEV), logit=True, mix=True)
    assert torch.equal(pool[[19999, 1]].to(BF), h) and (h[0] != 0).any() and int(torch.count_nonzero(pool[2:19999])) == 0


def test_one_token_of_each_of_long_sequences():
    """Rows further apart than a recurrence's may be."""
    B, row = 5, (1 << 24) + 8192
    wide = torch.zeros(B, row, dtype=BF, device=DEV)
    v, _ = make_scan([B], 320, BF, BF, True)
    x, up = make_heads(B, 3, 2, 64, 32, True, BF)
    p = [wide[:, i * 320:(i + 1) * 320] for i in range(6)]
    p[0].copy_(v["x"]), p[1].copy_(v["g"])
    pools = torch.ones(2, B, 320, device=DEV)
    want = tri.gated_scan_step(v["x"], v["g"], pools[0], logit=True, mix=True)
    tri.gated_scan_step(p[0], p[1], pools[1], logit=True, mix=True, h=p[2])
    assert torch.equal(p[2], want) and torch.equal(pools[0], pools[1])
    q, k = p[3][:, :192].view(B, 3, 64), p[3][:, 192:].view(B, 2, 64)
    q.copy_(x["q"]), k.copy_(x["k"])
    want = tri.qk_norm_rope(**x)
    got = tri.qk_norm_rope(**dict(x, q=q, k=k), q_out=p[4][:, :192].view(B, 3, 64), k_out=p[4][:, 192:].view(B, 2, 64))
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    back = tri.qk_norm_rope_bwd(**up, **x)
    got = tri.qk_norm_rope_bwd(**up, **dict(x, q=q, k=k), dq=p[5][:, :192].view(B, 3, 64), dk=p[5][:, 192:].view(B, 2, 64))
    assert all(torch.equal(a, b) for a, b in zip(got, back))


def test_rows_behind_the_last_sequence_stay_as_they_are():
    v, up = make_scan([70, 58], 64, BF, BF, True)
    h = torch.full((140, 64), 7.0, dtype=BF, device=DEV)
    tri.gated_scan_varlen(**v, seqlens=[70, 58], logit=True, h=h[:128])
    assert (h[128:] == 7).all() and not (h[:128] == 7).all()
    dx, dg = torch.full_like(h, 7.0), torch.full_like(h, 7.0)
    tri.gated_scan_bwd_varlen(v["x"], v["g"], h[:128], up["dh"], [70, 58], v["state"], logit=True, dx=dx[6:134], dg=dg[6:134])
    assert all((t[:6] == 7).all() and (t[134:] == 7).all() for t in (dx, dg))


@pytest.mark.parametrize("T", [100, 1000])
def test_a_nan_of_any_bits_goes_on(T):
    x = torch.zeros(1, T, 64, device=DEV)
    x.view(torch.int32)[0, 3, 5] = -1
    h, final = tri.gated_scan(x, torch.zeros_like(x), logit=True, mix=True)
    assert h[0, 3:, 5].isnan().all() and final[0, 5].isnan() and (h[..., 6] == 0).all()


# ---------------------------------------------------------------- the example

def test_gradients_of_the_example():
    """Against autograd through the recurrence and the norm in 64 bits: outputs and gradients end in bf16, 2^-9 of a value each, gradients of the mixed stream too behind h as it was
    written (2^-9 of its size); 2^-7 of the whole bounds them."""
    gen = torch.Generator(device=DEV).manual_seed(3)
    B, T, H, d = 2, 70, 2, 32
    W = 3 * H * d
    both = torch.randn(B, T, 2 * W, generator=gen, device=DEV).to(BF)
    ups = [torch.randn(B, T, H, d, generator=gen, device=DEV).to(BF) for _ in range(3)]
    mine = both.clone().requires_grad_()
    got = example.UnitHeads.apply(example.Mix.apply(mine), H)
    torch.autograd.backward(got, ups)
    ref = both.double().cpu().requires_grad_()
    x, a = ref[..., :W], torch.sigmoid(ref[..., W:])
    s, ys = torch.zeros(B, W, dtype=torch.float64), []
    for t in range(T):
        s = a[:, t] * s + (1 - a[:, t]) * x[:, t]
        ys.append(s)
    q, k, v = torch.stack(ys, 1).unflatten(-1, (3, H, d)).unbind(-3)
    unit = lambda z: z / (z.square().sum(-1, keepdim=True) + 1e-6).sqrt()
    want = unit(q), unit(k), v
    torch.autograd.backward(want, [u.double().cpu() for u in ups])
    for g, w in zip((*got, mine.grad), (*want, ref.grad)):
        assert (g.detach().double().cpu() - w.detach()).norm() <= 2.0 ** -7 * w.norm()


def test_the_example_runs():
    """Training goes on without anything that is not finite; tokens one by one are the prompt: 2^-6 as in gated_delta_layer.py, and the mixed stream's roundings, which may fall to the
    other side (2^-8 of some of the queries, keys and values each)."""
    torch.manual_seed(0)
    layer = example.MixedLayer(256, 4)
    losses = example.train(layer, steps=5)
    assert all(x == x and x < float("inf") for x in losses) and all(p.grad.isfinite().all() for p in layer.parameters())
    assert example.answer(layer) <= 2.0 ** -5
