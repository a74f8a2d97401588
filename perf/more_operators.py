"""What stands between a projection and a linear-attention layer's operators, as cases that can be timed and checked one by one.

Operators (key "op"):
  heads      norms of queries and keys for each head (root mean square, or to unit length), rotated by position in the same pass
  heads_bwd  its gradient: of queries, keys and the weights
  scan       the gated recurrence channel by channel, h_t = a_t h_(t-1) + b_t, over whole sequences, and the state after them
  scan_bwd   its gradient: of inputs, gates and initial state
  scan_step  one token of it: the state is updated in place, in a pool of slots

A case is a dict of plain values:
  N, H, Hk, d  tokens, heads of queries, heads of keys, elements of a head
  rot          columns of a head that are rotated (0: none);   interleaved: pairs (2i, 2i + 1), otherwise (i, i + rot / 2)
  unit         to unit length, otherwise root mean square;   weight: one for queries and one for keys
  joint        queries and keys are columns of one projection of queries, keys and values;   far: positions near a million
  B, T, lens   sequences and tokens per sequence; lens = True: packed sequences of different lengths, T the mean
  D            channels;   logit: a = sigmoid(g), otherwise a = e^g;   mix: b = (1 - a) x, otherwise b = x
  joint        x and g are columns of one projection;   state: an initial state is given (scan_bwd: a final state's gradient too)
  slots        scan_step: slots of the state pool, of which B are used
  type, gtype  element type of the tokens' tensors / of g; states and weights' gradients are fp32
"""
import math

import torch

own = False

_TYPE = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
_EPS = 1e-6


def _heads(name, op="heads", **kw):
    c = dict(op=op, N=4096, H=16, Hk=8, d=128, rot=128, interleaved=False, unit=False, weight=True, joint=False, far=False, type="bf16")
    c.update(kw)
    return dict(c, name=name)


def _scan(name, op="scan", **kw):
    c = dict(op=op, B=1, T=4096, lens=False, D=2048, logit=True, mix=True, joint=False, state=False, type="bf16", gtype="bf16")
    c.update(kw)
    return dict(c, name=name)


def _step(name, **kw):
    c = dict(op="scan_step", B=1, D=2048, logit=True, mix=True, joint=False, slots=4, type="bf16", gtype="bf16")
    c.update(kw)
    return dict(c, name=name)


def listed():
    return [
        # One user's next token, straight from the projection, at a far position: a launch's latency.
        _heads("heads_1token", N=1, joint=True, far=True),
        # Heads of 80 with 32 rotated columns in pairs side by side, a ragged number of tokens, fp16.
        _heads("heads_1001_odd", N=1001, H=10, Hk=10, d=80, rot=32, interleaved=True, type="f16"),
        # The delta-rule layer's queries and keys for eight prompts of 8192 tokens, to unit length: the throughput case.
        _heads("heads_65536_unit", N=65536, H=16, Hk=16, rot=0, unit=True, weight=False),
        # Training: queries and keys of 16384 tokens, weights' gradients with them.
        _heads("heads_train", op="heads_bwd", N=16384, H=32, Hk=8),
        # Training of the delta-rule layer on short odd-length sequences, fp16.
        _heads("heads_train_unit", op="heads_bwd", N=2002, H=8, Hk=4, d=64, rot=0, unit=True, weight=False, type="f16"),
        # One prompt of 4096 tokens: few channels for the card, a long way through time.
        _scan("scan_1x4096"),
        # A batch of long prompts, inputs and gates from one projection: the throughput case.
        _scan("scan_8x8192", B=8, T=8192, joint=True),
        # Continuous batching: packed prompts that continue from earlier states, fp32 log-decays, fp16.
        _scan("scan_packed_48x1100", B=48, T=1100, lens=True, D=1000, logit=False, mix=False, state=True, type="f16", gtype="f32"),
        # Training on four sequences.
        _scan("scan_train_4x4096", op="scan_bwd", B=4),
        # Training on two short odd-length sequences with log-decays, fp32.
        _scan("scan_train_2x333", op="scan_bwd", B=2, T=333, D=510, logit=False, mix=False, state=True, type="f32", gtype="f32"),
        # One user's next token.
        _step("scan_step_1"),
        # The next token of a full server: 256 sequences in a pool of 300 slots.
        _step("scan_step_256", B=256, D=8192, joint=True, slots=300),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    most = {}
    for c in listed():
        most[c["op"]] = max(most.get(c["op"], 0), work(c)["bytes"])
    while True:
        op = rng.choice(["heads", "heads", "heads_bwd", "scan", "scan", "scan", "scan_bwd", "scan_bwd", "scan_step"])
        t = rng.choice(["bf16", "bf16", "f16", "f32"])
        if op in ("heads", "heads_bwd"):
            Hk, d = rng.choice([1, 2, 4, 8, 16]), rng.choice([32, 64, 64, 80, 96, 128, 128, 128, 192, 256, 2 * rng.randint(8, 128)])
            unit = rng.random() < 0.4
            rot = rng.choice([0, d // 4 * 2, d]) if unit else rng.choice([d, d, d // 4 * 2, 0])
            c = _heads("", op=op, N=_log(rng, 1, 65536), H=Hk * rng.choice([1, 1, 2, 4, 5]), Hk=Hk, d=d, rot=rot, interleaved=rng.random() < 0.4,
                       unit=unit, weight=rng.random() < (0.3 if unit else 0.9), joint=rng.random() < 0.5, far=rng.random() < 0.3, type=t)
        else:
            gtype = rng.choice([t, t, "f32"])
            D = rng.choice([8 * _log(rng, 2, 1024), 128 * _log(rng, 1, 64), _log(rng, 16, 8192)])
            logit = rng.random() < 0.6
            kw = dict(D=D, logit=logit, mix=rng.random() < 0.6, joint=gtype == t and rng.random() < 0.4, type=t, gtype=gtype)
            if op == "scan_step":
                B = _log(rng, 1, 256)
                c = _step("", B=B, slots=B + rng.randint(0, 64), **kw)
            else:
                c = _scan("", op=op, B=_log(rng, 1, 64), T=_log(rng, 1, 32768), lens=rng.random() < 0.35, state=rng.random() < 0.5, **kw)
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
    if c["op"] in ("heads", "heads_bwd"):
        x, back = c["N"] * (c["H"] + c["Hk"]) * c["d"], c["op"] == "heads_bwd"
        small = c["N"] * 4 * (c["rot"] > 0) + 2 * c["rot"] + 2 * c["d"] * c["weight"] * (e + 4 * back)
        turned = c["N"] * (c["H"] + c["Hk"]) * c["rot"]
        return {"bytes": (3 if back else 2) * e * x + small, "flops": (9 if back else 4) * x + 3 * turned}
    eg = 4 if c["gtype"] == "f32" else 2
    if c["op"] == "scan_step":
        return {"bytes": c["B"] * (c["D"] * (8 + 2 * e + eg) + 4), "flops": c["B"] * c["D"] * 6}
    n, states = sum(_lengths(c)), 4 * c["B"] * c["D"]
    if c["op"] == "scan":
        return {"bytes": n * c["D"] * (2 * e + eg) + states * (1 + int(c["state"])), "flops": n * c["D"] * 6}
    return {"bytes": n * c["D"] * ((3 + int(c["mix"])) * e + 2 * eg) + states * 3 * int(c["state"]), "flops": n * c["D"] * 10}


def _rand(gen, shape, dtype=torch.float32):
    return torch.randn(shape, generator=gen, device="cuda", dtype=torch.float32).to(dtype)


def _offsets(lens):
    at = [0]
    for n in lens:
        at.append(at[-1] + n)
    return at


def _gates(gen, c, shape):
    """Gates as layers have them: channels that forget within a few tokens beside channels that hold for thousands."""
    slow = 7 * torch.rand(c["D"], generator=gen, device="cuda")
    if c["logit"]:
        return _rand(gen, shape) + slow
    return -torch.nn.functional.softplus(_rand(gen, shape)) * torch.exp(-slow)


def _pair(gen, c, shape):
    """x and g of a recurrence; columns of one tensor where they come from one projection."""
    t, x, g = _TYPE[c["type"]], _rand(gen, shape), _gates(gen, c, shape)
    if c["joint"]:
        both = torch.cat([x.to(t), g.to(t)], -1)
        return both[..., :c["D"]], both[..., c["D"]:]
    return x.to(t), g.to(_TYPE[c["gtype"]])


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed * 1000003 + 29)
    t = _TYPE[c["type"]]
    s = {"case": c}
    if c["op"] in ("heads", "heads_bwd"):
        N, H, Hk, d, r = c["N"], c["H"], c["Hk"], c["d"], c["rot"]
        if c["joint"]:
            all3 = _rand(gen, (N, (H + 2 * Hk) * d), t)
            s["q"], s["k"] = all3[:, :H * d].view(N, H, d), all3[:, H * d:(H + Hk) * d].view(N, Hk, d)
        else:
            s["q"], s["k"] = _rand(gen, (N, H, d), t), _rand(gen, (N, Hk, d), t)
        s["qw"], s["kw"] = ((1 + 0.1 * _rand(gen, (d,))).to(t) if c["weight"] else None for _ in range(2))
        s["pos"] = s["freq"] = None
        if r:
            first = torch.randint(1000000, (1,), generator=gen, device="cuda") if c["far"] else torch.randint(1000, (1,), generator=gen, device="cuda")
            s["pos"] = (first + torch.arange(N, device="cuda") % 4096).int()
            s["freq"] = (10000.0 ** (-torch.arange(r // 2, device="cuda", dtype=torch.float64) * 2 / r)).float()
        if c["op"] == "heads_bwd":
            s["dq"], s["dk"] = _rand(gen, (N, H, d), t), _rand(gen, (N, Hk, d), t)
        return s
    if c["op"] == "scan_step":
        s["x"], s["g"] = _pair(gen, c, (c["B"], c["D"]))
        s["pool"] = _rand(gen, (c["slots"], c["D"]))
        s["slots"] = torch.randperm(c["slots"], generator=gen, device="cuda")[:c["B"]].int()
        return s
    lens = s["lens"] = _lengths(c)
    lead = (sum(lens),) if c["lens"] else (c["B"], c["T"])
    s["x"], s["g"] = _pair(gen, c, (*lead, c["D"]))
    s["state"] = _rand(gen, (c["B"], c["D"])) if c["state"] else None
    if c["op"] == "scan_bwd":
        s["h"] = _forward(s)[0]
        s["dh"] = _rand(gen, (*lead, c["D"]), t)
        s["dstate"] = _rand(gen, (c["B"], c["D"])) if c["state"] else None
    return s


def _decay(s, g):
    """(a, what x is multiplied by or None) in 32 bits."""
    c, g = s["case"], g.float()
    a = torch.sigmoid(g) if c["logit"] else torch.exp(g)
    if not c["mix"]:
        return a, None
    return a, torch.sigmoid(-g) if c["logit"] else -torch.expm1(g)


def _linear(a, b, longest):
    """y_t = a_t y_(t-1) + b_t along the first dimension, a = 0 where a sequence begins: spans of 1, 2, 4, ... tokens put together."""
    d = 1
    while d < longest:
        b = torch.cat([b[:d], b[d:] + a[d:] * b[:-d]])
        a = torch.cat([a[:d], a[d:] * a[:-d]])
        d *= 2
    return b


def _ends(s, device):
    """First tokens of the sequences and, last, how many tokens there are."""
    return torch.tensor(_offsets(s["lens"]), device=device)


def _forward(s):
    """Plain form, 32 bits: (h, final state)."""
    c, t = s["case"], _TYPE[s["case"]["type"]]
    D, at = c["D"], _ends(s, s["x"].device)
    x = s["x"].reshape(-1, D).float()
    a, share = _decay(s, s["g"].reshape(-1, D))
    b = x if share is None else share * x
    if s["state"] is not None:
        b = b.index_add(0, at[:-1], a[at[:-1]] * s["state"])
    h = _linear(a.index_fill(0, at[:-1], 0.0), b, max(s["lens"]))
    return h.to(t).view(s["x"].shape), h[at[1:] - 1]


def _backward(s):
    """Plain form, 32 bits: r_t = dh_t + a_(t+1) r_(t+1), and from it the gradients of x, g and the initial state."""
    c, t = s["case"], _TYPE[s["case"]["type"]]
    D, at = c["D"], _ends(s, s["x"].device)
    first, last = at[:-1], at[1:] - 1
    x, g, h = (s[n].reshape(-1, D).float() for n in ("x", "g", "h"))
    a, share = _decay(s, g)
    dh = s["dh"].reshape(-1, D).float()
    if s["dstate"] is not None:
        dh = dh.index_add(0, last, s["dstate"])
    after = torch.cat([a[1:], a[:1]]).index_fill(0, last, 0.0)
    r = _linear(after.flip(0), dh.flip(0), max(s["lens"])).flip(0)
    before = torch.cat([h[:1], h[:-1]])
    before[first] = torch.zeros_like(before[first]) if s["state"] is None else s["state"]
    dg = r * (before if share is None else before - x) * a
    if c["logit"]:
        dg = dg * torch.sigmoid(-g)
    dx = r if share is None else r * share
    grads = (dx.to(t).view(s["x"].shape), dg.to(s["g"].dtype).view(s["g"].shape))
    return grads if s["state"] is None else (*grads, (a * r)[first])


def _angles(s):
    """cos and sin of the tokens' rotations [N, 1, rot / 2]; the angle in 64 bits."""
    t = s["pos"].double()[:, None] * s["freq"].double()
    return torch.cos(t).float()[:, None], torch.sin(t).float()[:, None]


def _turn(s, y, back=False):
    c, r = s["case"], s["case"]["rot"]
    if not r:
        return y
    cos, sin = _angles(s)
    if back:
        sin = -sin
    a, b = (y[..., 0:r:2], y[..., 1:r:2]) if c["interleaved"] else (y[..., :r // 2], y[..., r // 2:r])
    a, b = a * cos - b * sin, b * cos + a * sin
    turned = torch.stack([a, b], -1).flatten(-2) if c["interleaved"] else torch.cat([a, b], -1)
    return torch.cat([turned, y[..., r:]], -1)


def _head_norm(s, x):
    sq = (x * x).sum(-1, keepdim=True)
    return torch.rsqrt((sq if s["case"]["unit"] else sq / s["case"]["d"]) + _EPS)


def run(state):
    s, c = state, state["case"]
    if own:
        return _run_own(s, c)
    t = _TYPE[c["type"]]
    if c["op"] == "heads":
        out = []
        for x, w in ((s["q"].float(), s["qw"]), (s["k"].float(), s["kw"])):
            y = x * _head_norm(s, x)
            out.append(_turn(s, y if w is None else y * w.float()).to(t))
        return tuple(out)
    if c["op"] == "heads_bwd":
        out, weights = [], []
        for x, w, dy in ((s["q"].float(), s["qw"], s["dq"].float()), (s["k"].float(), s["kw"], s["dk"].float())):
            n = _head_norm(s, x)
            dy, hat = _turn(s, dy, back=True), x * n
            if w is not None:
                weights.append((dy * hat).sum((0, 1)))
                dy = dy * w.float()
            dot = (dy * hat).sum(-1, keepdim=True)
            out.append((n * (dy - hat * (dot if c["unit"] else dot / c["d"]))).to(t))
        return tuple(out + weights)
    if c["op"] == "scan":
        return _forward(s)
    if c["op"] == "scan_bwd":
        return _backward(s)
    at = s["slots"].long()
    a, share = _decay(s, s["g"])
    x = s["x"].float()
    h = a * s["pool"][at] + (x if share is None else share * x)
    s["pool"][at] = h
    return h.to(t), s["pool"]


def _run_own(s, c):
    import paper_2605_21325_amd as tri
    if c["op"] == "heads":
        return tri.qk_norm_rope(s["q"], s["k"], s["qw"], s["kw"], s["pos"], s["freq"], unit=c["unit"], interleaved=c["interleaved"], eps=_EPS)
    if c["op"] == "heads_bwd":
        got = tri.qk_norm_rope_bwd(s["dq"], s["dk"], s["q"], s["k"], s["qw"], s["kw"], s["pos"], s["freq"], unit=c["unit"], interleaved=c["interleaved"], eps=_EPS)
        return tuple(x for x in got if x is not None)
    kind = dict(logit=c["logit"], mix=c["mix"])
    if c["op"] == "scan_step":
        return tri.gated_scan_step(s["x"], s["g"], s["pool"], slots=s["slots"], **kind), s["pool"]
    packed = (s["lens"],) if c["lens"] else ()
    if c["op"] == "scan":
        return (tri.gated_scan_varlen if packed else tri.gated_scan)(s["x"], s["g"], *packed, state=s["state"], **kind)
    got = (tri.gated_scan_bwd_varlen if packed else tri.gated_scan_bwd)(s["x"], s["g"], s["h"], s["dh"], *packed, state=s["state"], dstate=s["dstate"], **kind)
    return tuple(x for x in got if x is not None)


def exact(case, seed):
    """From the definitions, in 64 bits: rotations as products of complex numbers, the recurrence and its gradient token by token."""
    s, c = prepare(case, seed), case
    if c["op"] in ("heads", "heads_bwd"):
        if c["N"] * (c["H"] + c["Hk"]) * c["d"] > 2 ** 30:
            return None  # (takes too much memory)
        if c["rot"]:
            phase = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), torch.outer(s["pos"].double(), s["freq"].double()))[:, None]

        def rotated(y, phase):
            r, y = c["rot"], y.clone()
            pairs = y[..., :r].unflatten(-1, (-1, 2)) if c["interleaved"] else y[..., :r].unflatten(-1, (2, -1)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * phase)
            y[..., :r] = (z if c["interleaved"] else z.transpose(-1, -2)).flatten(-2)
            return y

        out, weights = [], []
        for n, w in (("q", s["qw"]), ("k", s["kw"])):
            x = s[n].double()
            w = torch.ones(c["d"], dtype=torch.float64, device="cuda") if w is None else w.double()
            length = (x.square().sum(-1, keepdim=True) / (1 if c["unit"] else c["d"]) + _EPS).sqrt()
            if c["op"] == "heads":
                y = x / length * w
                out.append(rotated(y, phase) if c["rot"] else y)
                continue
            dy = s["d" + n].double()
            dy = rotated(dy, phase.conj().resolve_conj()) if c["rot"] else dy
            if c["weight"]:
                weights.append((dy * x / length).sum((0, 1)))
            dy = dy * w
            out.append(dy / length - x * (dy * x).sum(-1, keepdim=True) / (length ** 3 * (1 if c["unit"] else c["d"])))
        return tuple(out + weights)

    def gates(g):
        """(a, 1 - a) of log-decays or logits."""
        g = g.double()
        return (1 / (1 + torch.exp(-g)), 1 / (1 + torch.exp(g))) if c["logit"] else (torch.exp(g), -torch.expm1(g))

    if c["op"] == "scan_step":
        at, pool = s["slots"].long(), s["pool"].double()
        a, rest = gates(s["g"])
        h = a * pool[at] + (rest if c["mix"] else 1) * s["x"].double()
        pool[at] = h
        return h, pool
    lens, D = s["lens"], c["D"]
    if max(lens) > 100000 or sum(lens) * D > 2 ** 28:
        return None  # (takes too long)
    # The sequences stand in the order of their lengths: those that are there at a time are the first ones.
    order = sorted(range(len(lens)), key=lambda i: -lens[i])
    at = torch.tensor([_offsets(lens)[i] for i in order], device="cuda")
    alive, m = [], len(lens)
    for i in range(max(lens)):
        while lens[order[m - 1]] <= i:
            m -= 1
        alive.append(m)
    order = torch.tensor(order, device="cuda")
    x, g = s["x"].reshape(-1, D), s["g"].reshape(-1, D)
    S = torch.zeros(len(lens), D, dtype=torch.float64, device="cuda") if s["state"] is None else s["state"].double()[order]
    if c["op"] == "scan":
        out = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for i, m in enumerate(alive):
            now = at[:m] + i
            a, rest = gates(g[now])
            S[:m] = a * S[:m] + (rest if c["mix"] else 1) * x[now].double()
            out[now] = S[:m]
        return out.view(s["x"].shape), torch.empty_like(S).index_copy_(0, order, S)
    h, dh = s["h"].reshape(-1, D), s["dh"].reshape(-1, D)
    dx, dg = torch.empty(x.shape, dtype=torch.float64, device="cuda"), torch.empty(x.shape, dtype=torch.float64, device="cuda")
    R = torch.zeros_like(S) if s["dstate"] is None else s["dstate"].double()[order]  # the gradient of the state after a token
    for i in reversed(range(len(alive))):
        m = alive[i]
        now = at[:m] + i
        a, rest = gates(g[now])
        r = R[:m] + dh[now].double()
        past = h[now - 1].double() if i else S[:m]
        dx[now] = r * rest if c["mix"] else r
        dg[now] = r * (past - x[now].double() if c["mix"] else past) * a * (rest if c["logit"] else 1)
        R[:m] = r * a
    grads = (dx.view(s["x"].shape), dg.view(s["x"].shape))
    return grads if s["state"] is None else (*grads, torch.empty_like(R).index_copy_(0, order, R))
