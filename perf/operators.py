"""What a gated linear-attention layer runs beside the chunk inverse, as cases that can be timed and checked one by one.

Operators (key "op"):
  chunk      attention over chunks of C tokens with one decay per head: a layer's output for prompts, and the state after them.
             With delta = True the chunk's values are the delta rule's, U - W S, from the two solved right-hand sides U and W
  chunk_bwd  its gradient: of queries, keys, values (and W), decay and initial state
  step       the same layer's single token: the state is updated in place, in a pool of slots
  norm       root-mean-square norm with the residual's addition in front; the result in x's type or in 8 bits with scales
  norm_bwd   its gradient

A case is a dict of plain values:
  B, T, lens   sequences and tokens per sequence; lens = True: packed sequences of different lengths, T the mean
  H, Hk        heads of values, decay and state / of queries and keys (Hk divides H: consecutive heads share one)
  dk, dv, C    key channels, value columns, chunk size
  type         element type of the tokens' tensors; states, decays and scales are fp32
  gate         False: no decay;   delta: the delta rule;   state: an initial state is given (chunk_bwd: a final state's gradient too)
  slots        step: slots of the state pool, of which B are used
  N, D         norm: rows and columns;   residual: one is added;   out: "same" or "fp8";   group: columns a scale (0: the row)
"""
import math

import torch

own = False

_TYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_EPS = 1e-6
_FP8_MAX = 448.0  # the largest finite value of the 8-bit type (4 exponent, 3 mantissa bits)


def _attn(name, op="chunk", **kw):
    c = dict(op=op, B=1, T=4096, lens=False, H=16, Hk=16, dk=128, dv=128, C=64, type="bf16", gate=True, delta=True, state=False)
    c.update(kw)
    return dict(c, name=name)


def _step(name, **kw):
    c = dict(op="step", B=1, H=16, Hk=16, dk=128, dv=128, type="bf16", gate=True, delta=True, slots=4)
    c.update(kw)
    return dict(c, name=name)


def _norm(name, op="norm", **kw):
    c = dict(op=op, N=4096, D=2048, type="bf16", residual=True, out="fp8", group=0)
    c.update(kw)
    return dict(c, name=name)


def listed():
    return [
        # A short prompt of the smallest layer: four chunks of two heads, where launches count.
        _attn("prompt_tiny", T=256, H=2, Hk=2, dk=64, dv=64),
        # One layer's prefill of one 4096-token prompt: few heads for the card, many chunks one after another.
        _attn("prompt_1x4096"),
        # The same layer on a batch of long prompts: the throughput case.
        _attn("prompt_8x8192", B=8, T=8192),
        # Continuous batching of a layer without the delta rule on one shard (4 heads): packed prompts that end inside chunks
        # and continue from earlier states.
        _attn("packed_48x1100", B=48, T=1100, lens=True, H=4, Hk=4, type="f16", delta=False, state=True),
        # Large chunks, no decay, one very long prompt, two value heads to a key head.
        _attn("long_32768_c128", T=32768, H=32, Hk=16, C=128, gate=False),
        # Training on short odd-length sequences, plain decay, shared key heads, fp16.
        _attn("train_2x1000", op="chunk_bwd", B=2, T=1000, H=8, Hk=4, dk=64, type="f16", delta=False, state=True),
        # Training of the delta-rule layer at the single-layer size, four sequences.
        _attn("train_4x4096", op="chunk_bwd", B=4),
        # One user's next token.
        _step("step_1"),
        # The next token of a full server: 256 sequences in a pool of 300 slots.
        _step("step_256", B=256, H=32, Hk=16, slots=300),
        # The layer's entry in decoding: three rows, 8 bits for the projection behind it.
        _norm("norm_3rows", N=3),
        # The same for a batch of prompts, a scale for every 128 columns.
        _norm("norm_65536rows", N=65536, group=128),
        # Its training pass, an odd number of rows.
        _norm("norm_train", op="norm_bwd", N=16381, D=4096, out="same"),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), work(c)["bytes"])
    while True:
        op = rng.choice(["chunk", "chunk", "chunk", "chunk_bwd", "chunk_bwd", "step", "step", "norm", "norm", "norm_bwd"])
        if op in ("norm", "norm_bwd"):
            out = rng.choice(["fp8", "fp8", "same"]) if op == "norm" else "same"
            group = rng.choice([0, 128]) if out == "fp8" else 0
            c = _norm("", op=op, N=_log(rng, 1, 65536), D=128 * _log(rng, 1, 64) if group else 8 * _log(rng, 8, 1024), type=rng.choice(["bf16", "bf16", "f16", "f32"]),
                      residual=op == "norm" and rng.random() < 0.75, out=out, group=group)
        elif op == "step":
            H, B = rng.choice([2, 4, 8, 16, 32]), _log(rng, 1, 256)
            c = _step("", B=B, H=H, Hk=max(1, H // rng.choice([1, 1, 2])), dk=rng.choice([64, 128]), dv=rng.choice([64, 128]),
                      type=rng.choice(["bf16", "f16"]), gate=rng.random() < 0.8, delta=rng.random() < 0.7, slots=B + rng.randint(0, 64))
            c["gate"] = c["gate"] or not c["delta"]  # (a sum without decay or correction grows without end when called again and again)
        else:
            H = rng.choice([2, 4, 8, 16, 32])
            c = _attn("", op=op, B=_log(rng, 1, 32), T=_log(rng, 1, 32768 if op == "chunk" else 8192), lens=rng.random() < 0.3, H=H, Hk=max(1, H // rng.choice([1, 1, 2])),
                      dk=rng.choice([64, 128, 128]), dv=rng.choice([64, 128, 128]), C=rng.choice([64, 64, 128]), type=rng.choice(["bf16", "bf16", "f16"]),
                      gate=rng.random() < 0.8, delta=rng.random() < 0.6, state=rng.random() < 0.5)
        if work(c)["bytes"] <= most[op]:
            del c["name"]
            return c


def _lengths(c):
    """Tokens of each sequence; those of packed sequences follow from the case alone, mean T, from one token up."""
    if not c["lens"] or c["B"] == 1:
        return [c["T"]] * c["B"]
    return [1 + (c["T"] - 1) * 2 * ((i * 7 + 3) % c["B"]) // (c["B"] - 1) for i in range(c["B"])]


def work(c):
    e = 4 if c["type"] == "f32" else 2
    if c["op"] in ("norm", "norm_bwd"):
        x = c["N"] * c["D"]
        if c["op"] == "norm_bwd":
            return {"bytes": 3 * e * x + (e + 4) * c["D"], "flops": 10 * x}
        scales = 4 * c["N"] * (c["D"] // c["group"] if c["group"] else 1) if c["out"] == "fp8" else 0
        return {"bytes": (e + (2 * e if c["residual"] else 0) + (1 if c["out"] == "fp8" else e)) * x + scales + e * c["D"], "flops": 6 * x}
    H, Hk, dk, dv, d = c["H"], c["Hk"], c["dk"], c["dv"], int(c["delta"])
    if c["op"] == "step":
        return {"bytes": c["B"] * (8 * H * dk * dv + e * (2 * Hk * dk + 2 * H * dv) + 4 * H * (d + int(c["gate"])) + 4), "flops": c["B"] * H * dk * dv * (4 + 2 * d + int(c["gate"]))}
    n, C = sum(_lengths(c)), c["C"]
    tokens = e * (2 * Hk * dk + 2 * H * dv + d * H * dk) + 4 * H * int(c["gate"])  # q, k, u, o, w; g
    states = 4 * c["B"] * H * dk * dv
    products = H * (2 * dk * dv * (2 + d) + (C + 1) * (dk + dv))
    if c["op"] == "chunk":
        return {"bytes": n * tokens + states * (1 + int(c["state"])), "flops": n * products}
    return {"bytes": n * (2 * tokens - e * H * dv) + states * 3 * int(c["state"]), "flops": n * 2 * products + n * H * 2 * dk * dv}


def _rand(gen, shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _unit(gen, shape, dtype):
    x = torch.randn(shape, generator=gen, device="cuda")
    return (x / x.norm(dim=-1, keepdim=True)).to(dtype)


def _solved(K, beta, g, V, lens, C):
    """The delta rule's solved right-hand sides U = (I + A)^-1 diag(beta) V and W = (I + A)^-1 diag(beta e^g) K, chunk by chunk."""
    total, H, dk = K.shape
    starts = torch.tensor([a + t for a, n in zip(_offsets(lens), lens) for t in range(0, n, C)], device=K.device)
    ends = torch.tensor([a + min(t + C, n) for a, n in zip(_offsets(lens), lens) for t in range(0, n, C)], device=K.device)
    U, W = torch.empty_like(V), torch.empty_like(K)
    eye = torch.eye(C, device=K.device)
    for at in range(0, len(starts), 512):
        rows = starts[at:at + 512, None] + torch.arange(C, device=K.device)
        there = rows < ends[at:at + 512, None]
        rows = torch.minimum(rows, ends[at:at + 512, None] - 1)
        k, v = (x[rows].float().transpose(1, 2) for x in (K, V))                                   # [chunk, H, C, d]
        b, gg = ((x[rows] * there[:, :, None]).transpose(1, 2).unsqueeze(-1) for x in (beta, g))
        A = torch.tril(torch.exp(torch.tril(gg - gg.transpose(-1, -2))) * torch.matmul(k, k.transpose(-1, -2).contiguous()) * b, -1)
        X, Y = eye - A, A
        for _ in range(int(math.log2(C)) - 1):
            Y = torch.matmul(Y, Y)
            X = X + torch.matmul(X, Y)
        u, w = torch.matmul(X, b * v).transpose(1, 2), torch.matmul(X, b * torch.exp(gg) * k).transpose(1, 2)
        U[rows[there]], W[rows[there]] = u[there].to(U.dtype), w[there].to(W.dtype)
    return U, W


def _offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _local_cumsum(rate, lens, C):
    """The running sum of a token's log-decays [total, H], beginning again at every chunk."""
    total = rate.shape[0]
    first = torch.cat([torch.arange(n) // C * C + a for a, n in zip(_offsets(lens), lens)]).to(rate.device)
    s = rate.double().cumsum(0)
    before = torch.cat([torch.zeros_like(s[:1]), s])[first]
    return (s - before).float() if total else rate


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 17)
    t = _TYPE[c["type"]]
    s = {"case": c}
    if c["op"] in ("norm", "norm_bwd"):
        s["x"] = _rand(gen, (c["N"], c["D"]), t)
        s["weight"] = (1 + 0.1 * _rand(gen, (c["D"],))).to(t)
        if c["op"] == "norm_bwd":
            s["dy"] = _rand(gen, (c["N"], c["D"]), t)
        elif c["residual"]:
            s["residual"] = (2 * _rand(gen, (c["N"], c["D"]))).to(t)
        return s
    H, Hk, dk, dv = c["H"], c["Hk"], c["dk"], c["dv"]
    s["scale"] = dk ** -0.5
    if c["op"] == "step":
        B = c["B"]
        s["q"], s["k"], s["v"] = _unit(gen, (B, Hk, dk), t), _unit(gen, (B, Hk, dk), t), _rand(gen, (B, H, dv), t)
        s["g"] = -0.05 * torch.nn.functional.softplus(_rand(gen, (B, H))) if c["gate"] else None
        s["beta"] = torch.sigmoid(_rand(gen, (B, H))) if c["delta"] else None
        s["pool"] = _rand(gen, (c["slots"], H, dk, dv))
        s["slots"] = torch.randperm(c["slots"], generator=gen, device="cuda")[:B].int()
        return s
    lens = _lengths(c)
    total = sum(lens)
    q, k, v = _unit(gen, (total, Hk, dk), t), _unit(gen, (total, Hk, dk), t), _rand(gen, (total, H, dv), t)
    rate = -0.05 * torch.nn.functional.softplus(_rand(gen, (total, H)))
    g = _local_cumsum(rate, lens, c["C"]) if c["gate"] else None
    w = None
    if c["delta"]:
        beta = torch.sigmoid(_rand(gen, (total, H)))
        v, w = _solved(k.repeat_interleave(H // Hk, 1), beta, torch.zeros_like(beta) if g is None else g, v, lens, c["C"])
    s["lens"] = lens
    s["q"], s["k"], s["u"], s["w"], s["g"] = (x if x is None or c["lens"] else x.view(c["B"], c["T"], *x.shape[1:]) for x in (q, k, v, w, g))
    s["state"] = _rand(gen, (c["B"], H, dk, dv)) if c["state"] else None
    if c["op"] == "chunk_bwd":
        s["do"] = _rand(gen, s["u"].shape, t)
        s["dstate"] = _rand(gen, (c["B"], H, dk, dv)) if c["state"] else None
    return s


def _chunked(s, q, k, u, w, g):
    """Tokens' tensors (fp32) as [sequence, H, chunk, C, d], what is not there 0; g without decay behind a sequence's end."""
    c, lens = s["case"], s["lens"]
    C, H = c["C"], c["H"]
    chunks = max(1, -(-max(lens) // C))
    n = torch.tensor(lens, device=q.device)[:, None]
    at = torch.tensor(_offsets(lens)[:-1], device=q.device)[:, None]
    token = torch.arange(chunks * C, device=q.device)[None]
    there = token < n
    rows = at + torch.minimum(token, n - 1).clamp_min(0)

    def cut(x, mask):
        x = x.reshape(-1, *x.shape[-2:])[rows] * mask[..., None, None]
        x = x.repeat_interleave(H // x.shape[2], 2)
        return x.view(len(lens), chunks, C, H, x.shape[-1]).permute(0, 3, 1, 2, 4)

    gate = torch.zeros(len(lens), H, chunks, C, device=q.device) if g is None else cut(g.reshape(-1, H, 1), token // C * C < n)[..., 0]
    return cut(q, there), cut(k, there), cut(u, there), None if w is None else cut(w, there), gate, there


def _attend(s, q, k, u, w, g, state):
    """Plain form, 32 bits: (output, final state).  With G = e^g, D_ij = e^(g_i - g_j) for i >= j and S the state before a chunk,
        V' = U - W S,   O = scale (diag(G) Q S + (Q K^T . D) V'),   S <- G_C S + (diag(e^(g_C - g)) K)^T V'."""
    c = s["case"]
    Q, K, U, W, G, there = _chunked(s, q, k, u, w, g)
    seqs, H, chunks, C, dk = Q.shape
    if state is None:
        state = torch.zeros(seqs, H, dk, U.shape[-1], device=Q.device)
    causal = torch.ones(C, C, dtype=torch.bool, device=Q.device).tril()
    P = torch.matmul(Q, K.transpose(-1, -2)) * torch.exp((G[..., :, None] - G[..., None, :]).masked_fill(~causal, -math.inf))
    Kt = (K * torch.exp(G[..., -1:] - G)[..., None]).transpose(-1, -2)
    last = G[..., -1]
    if W is None:  # states before every chunk, all at once: those of the chunks before, decayed
        total = torch.cat([torch.zeros_like(last[..., :1]), last.cumsum(-1)], -1)
        E = torch.exp((total[..., :, None] - total[..., None, 1:]).masked_fill(~torch.ones(chunks + 1, chunks, dtype=torch.bool, device=Q.device).tril(-1), -math.inf))
        new = torch.matmul(Kt, U).flatten(-2)
        S = (torch.matmul(E, new) + torch.exp(total)[..., None] * state.flatten(-2)[:, :, None]).view(seqs, H, chunks + 1, dk, -1)
        state, S, V = S[:, :, -1], S[:, :, :-1], U
    else:  # each chunk's values depend on the state before it
        before, values = [], []
        for j in range(chunks):
            before.append(state)
            values.append(U[:, :, j] - torch.matmul(W[:, :, j], state))
            state = torch.exp(last[:, :, j])[..., None, None] * state + torch.matmul(Kt[:, :, j], values[-1])
        S, V = torch.stack(before, 2), torch.stack(values, 2)
    O = s["scale"] * (torch.exp(G)[..., None] * torch.matmul(Q, S) + torch.matmul(P, V))
    O = O.permute(0, 2, 3, 1, 4).reshape(seqs, chunks * C, H, -1)[there]
    return O.reshape(u.shape), state


def _float8(y, group):
    """y as 8-bit values and their scales: a scale is the largest magnitude of its columns over the type's largest value."""
    z = y.view(y.shape[0], -1, group or y.shape[1])
    scale = z.abs().amax(-1) / _FP8_MAX
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    return (z / scale[..., None]).view_as(y).clamp(-_FP8_MAX, _FP8_MAX).to(torch.float8_e4m3fn), scale


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s, c)
    t = _TYPE[c["type"]]
    if c["op"] == "norm":
        x = s["x"].float()
        if c["residual"]:
            r = (x + s["residual"].float()).to(t)
            x = r.float()
        y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS) * s["weight"].float()
        y = _float8(y, c["group"]) if c["out"] == "fp8" else (y.to(t),)
        return y + ((r,) if c["residual"] else ())
    if c["op"] == "norm_bwd":
        x, dy = s["x"].float(), s["dy"].float()
        rstd = torch.rsqrt((x * x).mean(-1, keepdim=True) + _EPS)
        xhat, d = x * rstd, dy * s["weight"].float()
        return (rstd * (d - xhat * (d * xhat).mean(-1, keepdim=True))).to(t), (dy * xhat).sum(0)
    if c["op"] == "step":
        at = s["slots"].long()
        S, rep = s["pool"][at], c["H"] // c["Hk"]
        q, k, v = s["q"].float().repeat_interleave(rep, 1), s["k"].float().repeat_interleave(rep, 1), s["v"].float()
        if c["gate"]:
            S = S * torch.exp(s["g"])[..., None, None]
        if c["delta"]:
            v = s["beta"][..., None] * (v - (k[..., None] * S).sum(-2))
        S = S + k[..., None] * v[..., None, :]
        s["pool"][at] = S
        return (s["scale"] * (q[..., None] * S).sum(-2)).to(t), s["pool"]
    x = [None if s[n] is None else s[n].float() for n in ("q", "k", "u", "w", "g", "state")]
    if c["op"] == "chunk":
        O, final = _attend(s, *x)
        return O.to(t), final
    with torch.enable_grad():
        x = [None if y is None else y.detach().requires_grad_() for y in x]
        O, final = _attend(s, *x)
        out, grad = ([O, final], [s["do"].float(), s["dstate"]]) if c["state"] else ([O], [s["do"].float()])
        got = iter(torch.autograd.grad(out, [y for y in x if y is not None], grad))
    return tuple(next(got).to(t if i < 4 else torch.float32) for i, y in enumerate(x) if y is not None)


def _run_own(s, c):
    import paper_2605_21325_amd as tri
    if c["op"] == "norm":
        r = s.get("residual")
        if c["out"] == "fp8":
            q, scale, total = tri.add_rms_norm_fp8(s["x"], s["weight"], residual=r, eps=_EPS, group=c["group"])
            return (q, scale) + ((total,) if c["residual"] else ())
        y, total = tri.add_rms_norm(s["x"], s["weight"], residual=r, eps=_EPS)
        return (y,) + ((total,) if c["residual"] else ())
    if c["op"] == "norm_bwd":
        return tri.add_rms_norm_bwd(s["dy"], s["x"], s["weight"], eps=_EPS)
    if c["op"] == "step":
        return tri.gdn_step(s["q"], s["k"], s["v"], s["g"], s["pool"], beta=s["beta"], slots=s["slots"], scale=s["scale"]), s["pool"]
    packed = (s["lens"],) if c["lens"] else ()
    if c["op"] == "chunk":
        f = tri.gdn_chunk_attn_varlen if c["lens"] else tri.gdn_chunk_attn
        return f(s["q"], s["k"], s["u"], s["g"], *packed, c["C"], W=s["w"], state=s["state"], scale=s["scale"])
    f = tri.gdn_chunk_attn_bwd_varlen if c["lens"] else tri.gdn_chunk_attn_bwd
    got = f(s["q"], s["k"], s["u"], s["g"], s["do"], *packed, c["C"], W=s["w"], state=s["state"], dstate=s["dstate"], scale=s["scale"])
    return tuple(x for x in got if x is not None)


def exact(case, seed):
    """From the definitions, in 64 bits: the recurrence token by token, with gradients taken through it a chunk at a time."""
    s, c = prepare(case, seed), case
    if c["op"] in ("norm", "norm_bwd"):
        x = s["x"].double()
        r = x + s["residual"].double() if c["op"] == "norm" and c["residual"] else None
        if r is not None:
            x = r.to(s["x"].dtype).double()  # the norm is that of the sum as it is stored
        rms = (x.square().sum(-1, keepdim=True) / c["D"] + _EPS).sqrt()
        w = s["weight"].double()
        if c["op"] == "norm_bwd":
            dy = s["dy"].double()
            dot = (dy * w * x).sum(-1, keepdim=True) / c["D"]
            return dy * w / rms - x * dot / rms ** 3, (dy * x / rms).sum(0)
        y = x / rms * w
        if c["out"] == "fp8":
            z = y.view(c["N"], -1, c["group"] or c["D"])
            scale = z.abs().amax(-1) / _FP8_MAX
            y = ((z / scale[..., None]).view_as(y), scale)
        else:
            y = (y,)
        return y + ((r,) if r is not None else ())
    rep = c["H"] // c["Hk"]
    if c["op"] == "step":
        at = s["slots"].long()
        pool = s["pool"].double()
        q, k, v = s["q"].double().repeat_interleave(rep, 1), s["k"].double().repeat_interleave(rep, 1), s["v"].double()
        S = pool[at]
        if c["gate"]:
            S *= s["g"].double().exp()[..., None, None]
        if c["delta"]:
            v = s["beta"].double()[..., None] * (v - torch.matmul(k[..., None, :], S)[..., 0, :])
        S += k[..., None] * v[..., None, :]
        pool[at] = S
        return s["scale"] * torch.matmul(q[..., None, :], S)[..., 0, :], pool
    lens, C, H = s["lens"], c["C"], c["H"]
    if max(lens) * (1 if c["op"] == "chunk" else 4) > 100000 or sum(lens) * H * c["dk"] > 2 ** 29:
        return None  # (takes too long)
    at, n = torch.tensor(_offsets(lens)[:-1], device="cuda"), torch.tensor(lens, device="cuda")

    def tokens(x, a, b):
        """Tokens a to b - 1 of every sequence [sequence, b - a, ...] in 64 bits; zeros behind its end."""
        x = x.reshape(sum(lens), *((H,) if x is s["g"] else x.shape[-2:]))
        i = torch.arange(a, b, device="cuda")[None] + at[:, None]
        ok = torch.arange(a, b, device="cuda")[None] < n[:, None]
        y = x[i.clamp(max=max(0, sum(lens) - 1))].double()
        return y.masked_fill(~ok.view(*ok.shape, *[1] * (y.dim() - 2)), 0)

    def chunk(S, q, k, u, w, g, live):
        """One chunk of every sequence, a token at a time: (outputs, state after it)."""
        q, k = (x.repeat_interleave(rep, 2) for x in (q, k))
        S0, out, prev = S, [], None
        for i in range(q.shape[1]):
            if g is not None:
                step = g[:, i] if i == 0 else g[:, i] - g[:, i - 1]
                S = S * torch.where(live[:, i, None], step, torch.zeros_like(step)).exp()[..., None, None]
            v = u[:, i] if w is None else u[:, i] - torch.matmul(w[:, i, :, None], S0)[..., 0, :]
            S = S + k[:, i, :, :, None] * v[..., None, :]
            out.append(s["scale"] * torch.matmul(q[:, i, :, None], S)[..., 0, :])
        return torch.stack(out, 1), S

    S = torch.zeros(len(lens), H, c["dk"], c["dv"], device="cuda", dtype=torch.float64) if s["state"] is None else s["state"].double()
    names = [x for x in ("q", "k", "u", "w", "g") if s[x] is not None]
    spans = [(a, min(a + C, max(lens))) for a in range(0, max(lens), C)]
    live = [torch.arange(a, b, device="cuda")[None] < n[:, None] for a, b in spans]
    shape = lambda x, like: x.reshape(like.shape)  # noqa: E731

    def gather(parts):
        """Parts [sequence, span, ...] of the spans put together in the order of the tokens."""
        return torch.cat(parts, 1)[torch.cat(live, 1)]

    before, outs = [], []
    for (a, b), ok in zip(spans, live):
        before.append(S)
        have = {x: tokens(s[x], a, b) for x in names}
        o, S = chunk(S, have["q"], have["k"], have["u"], have.get("w"), have.get("g"), ok)
        outs.append(o)
    if c["op"] == "chunk":
        return shape(gather(outs), s["u"]), S
    dS = torch.zeros_like(S) if s["dstate"] is None else s["dstate"].double()
    grads = {x: [] for x in names}
    for j in reversed(range(len(spans))):
        (a, b), ok = spans[j], live[j]
        with torch.enable_grad():
            have = {x: tokens(s[x], a, b).requires_grad_() for x in names}
            S0 = before[j].detach().requires_grad_()
            o, S1 = chunk(S0, have["q"], have["k"], have["u"], have.get("w"), have.get("g"), ok)
            got = torch.autograd.grad([o, S1], [have[x] for x in names] + [S0], [tokens(s["do"], a, b), dS])
        for x, y in zip(names, got):
            grads[x].insert(0, y)
        dS = got[-1]
    got = [shape(gather(grads[x]), s[x]) for x in names]
    return tuple(got + ([dS] if c["state"] else []))
