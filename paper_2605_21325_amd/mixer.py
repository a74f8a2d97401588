"""ctypes binding of what stands between a projection and the layer's operators -- argument marshalling only, as in binding.py: norms of queries and keys for
each head with the rotation by position, the gated recurrence channel by channel with its gradient and its single token.

A call uses the current stream (or `stream`); tensors it makes itself are allocated on it.  Tokens' tensors may be columns of a wider one (a projection
as it is): the elements of a token stand side by side and tokens one stride apart; everything else must be contiguous.  Autograd records none of them: a gradient
is the call of its own beside each.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import binding
from .binding import OK, TriInvError, _chunk_offsets, _dev, _stream_ptr, dtype_code
from .layer import _has, _on, _opt

HEADS_UNIT, HEADS_INTERLEAVED, HEADS_POS64 = 1, 2, 4
SCAN_LOGIT, SCAN_MIX = 1, 2


_connected = None  # the native argument handling that knows these entry points


def _fast(t: torch.Tensor, stream):
    """(native argument handling, device, stream) for a plain call on the current stream, or None (see binding.py)."""
    global _connected
    if binding._lib is not binding._fast_lib or stream is not None or not t.is_cuda:
        return None
    if binding._fast is not _connected:
        L = binding.lib()
        binding._fast.connect_mixer(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
            L.qk_norm_rope, L.qk_norm_rope_bwd, L.qk_norm_rope_bwd_workspace, L.gated_scan, L.gated_scan_varlen, L.gated_scan_workspace, L.gated_scan_bwd, L.gated_scan_bwd_varlen,
            L.gated_scan_step)))
        _connected = binding._fast
    dev = binding._device_index()
    return binding._fast, dev, binding._raw_stream(dev)


def _address(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise ValueError(f"{name} must live in device memory")
    return t.data_ptr()


def _rows(t: Optional[torch.Tensor], name: str, inner: int, shape=None, dtype=None):
    """(address, elements from a token to the next) of a tensor whose last `inner` dimensions are a token's."""
    if t is None:
        return None, 0
    if shape is not None:
        _has(t, name, shape, dtype)
    address = _address(t, name)
    sizes, strides = t.shape, t.stride()
    width = 1
    for n, s in zip(reversed(sizes[len(sizes) - inner:]), reversed(strides[len(sizes) - inner:])):
        if n != 1 and s != width and t.numel():
            raise ValueError(f"{name}: a token's elements must be contiguous")
        width *= n
    step, span = width, None  # of a token; of all tokens of the dimensions seen
    for n, s in zip(reversed(sizes[:len(sizes) - inner]), reversed(strides[:len(sizes) - inner])):
        if n == 1 or not t.numel():
            continue
        if span is None:
            step = s
        elif s != span:
            raise ValueError(f"{name}: tokens must stand one stride apart")
        span = s * n
    return address, step


def _one_device(*tensors) -> None:
    """Refuses tensors of several devices, or of another than the current one, whose streams and kernels would not be theirs."""
    at = {t.device for t in tensors if t is not None}
    if len(at) > 1:
        raise ValueError(f"tensors of several devices: {sorted(str(d) for d in at)}")
    d = next(iter(at))
    if d.type == "cuda" and d.index != torch.cuda.current_device():
        raise ValueError(f"tensors of {d}, the current device is cuda:{torch.cuda.current_device()}")


def _heads_flags(unit, interleaved, positions):
    return HEADS_UNIT * bool(unit) | HEADS_INTERLEAVED * bool(interleaved) | HEADS_POS64 * (positions is not None and positions.dtype == torch.int64)


def _heads_checked(q, k, q_weight, k_weight, positions, inv_freq):
    """(leading dimensions, tokens, H, H_k, d, rot)."""
    if q.dim() < 2:
        raise ValueError(f"q must be [..., H, d], not {list(q.shape)}")
    lead, (H, d) = q.shape[:-2], q.shape[-2:]
    H_k = 0 if k is None else k.shape[-2] if k.dim() >= 2 else -1
    _has(k, "k", (*lead, H_k, d), q.dtype)
    _has(q_weight, "q_weight", (d,), q.dtype)
    _has(k_weight, "k_weight", (d,), q.dtype)
    if k is None and k_weight is not None:
        raise ValueError("k_weight without k")
    if (positions is None) != (inv_freq is None):
        raise ValueError("positions and inv_freq belong together")
    rot = 0
    if positions is not None:
        if positions.dtype not in (torch.int32, torch.int64):
            raise TypeError(f"positions is {positions.dtype}, not torch.int32 or torch.int64")
        _has(positions, "positions", lead, positions.dtype)
        rot = 2 * inv_freq.numel()
        _has(inv_freq, "inv_freq", (rot // 2,), torch.float32)
        if rot > d:
            raise ValueError(f"inv_freq rotates {rot} elements, a head has {d}")
    return lead, lead.numel(), H, H_k, d, rot


def qk_norm_rope(q: torch.Tensor, k: Optional[torch.Tensor], q_weight: Optional[torch.Tensor] = None, k_weight: Optional[torch.Tensor] = None,
                 positions: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None, unit: bool = False, interleaved: bool = False, eps: float = 1e-6,
                 q_out: Optional[torch.Tensor] = None, k_out: Optional[torch.Tensor] = None, stream=None):
    """(q_out, k_out): the heads of q [..., H, d] and k [..., H_k, d] (or None) over sqrt(mean(x^2) + eps), or with unit over sqrt(sum(x^2) + eps), times their
    weight [d], their first 2 len(inv_freq) elements rotated by the angles positions [...] (int32 or int64) times inv_freq (fp32): pairs (i, i + rot / 2), or
    interleaved (2 i, 2 i + 1).  q and k may be columns of a projection; q_out and k_out (q and k themselves too) likewise."""
    f = _fast(q, stream)
    if f:
        r = f[0].heads(f[1], f[2], q, k, q_weight, k_weight, positions, inv_freq, unit, interleaved, eps, q_out, k_out)
        if r is not None:
            return r
    _one_device(q, k, q_weight, k_weight, positions, inv_freq, q_out, k_out)
    lead, N, H, H_k, d, rot = _heads_checked(q, k, q_weight, k_weight, positions, inv_freq)
    if k is None and k_out is not None:
        raise ValueError("k_out without k")
    (pq, sq), (pk, sk) = _rows(q, "q", 2), _rows(k, "k", 2)
    with _on(stream, q.device):
        q_out = torch.empty(q.shape, dtype=q.dtype, device=q.device) if q_out is None else q_out
        k_out = None if k is None else torch.empty(k.shape, dtype=k.dtype, device=k.device) if k_out is None else k_out
    (oq, soq), (ok, sok) = _rows(q_out, "q_out", 2, q.shape, q.dtype), _rows(k_out, "k_out", 2, None if k is None else k.shape, q.dtype)
    st = binding.lib().qk_norm_rope(pq, pk, _opt(q_weight, "q_weight"), _opt(k_weight, "k_weight"), _opt(positions, "positions"), _opt(inv_freq, "inv_freq"), oq, ok, N, sq, sk, soq, sok,
                                    H, H_k, d, rot, dtype_code(q.dtype), _heads_flags(unit, interleaved, positions), eps, _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, "qk_norm_rope")
    return q_out, k_out


def qk_norm_rope_bwd(dq_out: torch.Tensor, dk_out: Optional[torch.Tensor], q: torch.Tensor, k: Optional[torch.Tensor], q_weight: Optional[torch.Tensor] = None,
                     k_weight: Optional[torch.Tensor] = None, positions: Optional[torch.Tensor] = None, inv_freq: Optional[torch.Tensor] = None, unit: bool = False,
                     interleaved: bool = False, eps: float = 1e-6, dq: Optional[torch.Tensor] = None, dk: Optional[torch.Tensor] = None, stream=None):
    """(dq, dk, dq_weight, dk_weight) of qk_norm_rope, from its inputs and the gradients of its results; the weights' are fp32, None in the place of the gradient of
    what was not given.  dq and dk may be columns of a wider tensor (a projection's gradient), or dq_out and dk_out themselves."""
    f = _fast(q, stream)
    if f:
        r = f[0].heads_bwd(f[1], f[2], dq_out, dk_out, q, k, q_weight, k_weight, positions, inv_freq, unit, interleaved, eps, dq, dk)
        if r is not None:
            return r
    _one_device(q, k, q_weight, k_weight, positions, inv_freq, dq_out, dk_out, dq, dk)
    lead, N, H, H_k, d, rot = _heads_checked(q, k, q_weight, k_weight, positions, inv_freq)
    if (k is None) != (dk_out is None):
        raise ValueError("k and dk_out belong together")
    if k is None and dk is not None:
        raise ValueError("dk without k")
    k_shape = None if k is None else k.shape
    (pq, sq), (pk, sk) = _rows(q, "q", 2), _rows(k, "k", 2)
    (uq, suq), (uk, suk) = _rows(dq_out, "dq_out", 2, q.shape, q.dtype), _rows(dk_out, "dk_out", 2, k_shape, q.dtype)
    size = ctypes.c_int64()
    st = binding.lib().qk_norm_rope_bwd_workspace(N, H, H_k, d, ctypes.byref(size))
    if st != OK:
        raise TriInvError(st, "qk_norm_rope_bwd")
    weights = q_weight is not None or k_weight is not None
    with _on(stream, q.device):
        dq = torch.empty(q.shape, dtype=q.dtype, device=q.device) if dq is None else dq
        dk = None if k is None else torch.empty(k.shape, dtype=k.dtype, device=k.device) if dk is None else dk
        dqw = None if q_weight is None else torch.empty(d, dtype=torch.float32, device=q.device)
        dkw = None if k_weight is None else torch.empty(d, dtype=torch.float32, device=q.device)
        ws = torch.empty(max(16, size.value), dtype=torch.uint8, device=q.device) if weights else None
    (oq, soq), (ok, sok) = _rows(dq, "dq", 2, q.shape, q.dtype), _rows(dk, "dk", 2, k_shape, q.dtype)
    st = binding.lib().qk_norm_rope_bwd(uq, uk, pq, pk, _opt(q_weight, "q_weight"), _opt(k_weight, "k_weight"), _opt(positions, "positions"), _opt(inv_freq, "inv_freq"), oq, ok,
                                        _opt(dqw, "dq_weight"), _opt(dkw, "dk_weight"), _opt(ws, "workspace"), ws.numel() if weights else 0, N, suq, suk, sq, sk, soq, sok,
                                        H, H_k, d, rot, dtype_code(q.dtype), _heads_flags(unit, interleaved, positions), eps, _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, "qk_norm_rope_bwd")
    return dq, dk, dqw, dkw


def _gate_type(g, x_dtype):
    if g.dtype not in (x_dtype, torch.float32):
        raise TypeError(f"g is {g.dtype}, not {x_dtype} or torch.float32")
    return dtype_code(g.dtype)


def _scan_workspace(where, N, n_seq, D, device):
    n = ctypes.c_int64()
    st = binding.lib().gated_scan_workspace(N, n_seq, D, ctypes.byref(n))
    if st != OK:
        raise TriInvError(st, where)
    return (torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None), n.value


def _flags(logit, mix):
    return SCAN_LOGIT * bool(logit) | SCAN_MIX * bool(mix)


def _scan(where, x, g, n_seq, N, where_args, state, logit, mix, h, final_state, stream):
    D = x.shape[-1]
    _has(g, "g", x.shape, g.dtype)
    g_code = _gate_type(g, x.dtype)
    _has(state, "state", (n_seq, D), torch.float32)
    _has(final_state, "final_state", (n_seq, D), torch.float32)
    (px, sx), (pg, sg) = _rows(x, "x", 1), _rows(g, "g", 1)
    with _on(stream, x.device):
        h = torch.empty(x.shape, dtype=x.dtype, device=x.device) if h is None else h
        final_state = torch.empty((n_seq, D), dtype=torch.float32, device=x.device) if final_state is None else final_state
        ws, n = _scan_workspace(where, N, n_seq, D, x.device)
    ph, sh = _rows(h, "h", 1, x.shape, x.dtype)
    st = getattr(binding.lib(), where)(px, pg, _opt(state, "state"), ph, _dev(final_state, "final_state"), _opt(ws, "workspace"), n, *where_args, D, sx, sg, sh, dtype_code(x.dtype), g_code,
                                       _flags(logit, mix), _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, where)
    return h, final_state


def gated_scan(x: torch.Tensor, g: torch.Tensor, state: Optional[torch.Tensor] = None, logit: bool = False, mix: bool = False, h: Optional[torch.Tensor] = None,
               final_state: Optional[torch.Tensor] = None, stream=None):
    """(h, final_state) of the gated recurrence h_t = a_t h_(t-1) + b_t over x, g [B, Tlen, D] (one sequence at least, tokens may be none): a = e^g, or with logit sigmoid(g); b = x, or with mix (1 - a) x.
    g is of x's type or fp32.  state: [B, D] fp32, the state before the first token (None: zeros)."""
    f = _fast(x, stream)
    if f:
        r = f[0].scan(f[1], f[2], x, g, state, logit, mix, h, final_state)
        if r is not None:
            return r
    _one_device(x, g, state, h, final_state)
    if x.dim() != 3:
        raise ValueError(f"x must be [B, Tlen, D], not {list(x.shape)}")
    B, T = x.shape[:2]
    return _scan("gated_scan", x, g, B, B * T, (B, T), state, logit, mix, h, final_state, stream)


def gated_scan_varlen(x: torch.Tensor, g: torch.Tensor, seqlens, state: Optional[torch.Tensor] = None, logit: bool = False, mix: bool = False,
                      h: Optional[torch.Tensor] = None, final_state: Optional[torch.Tensor] = None, stream=None):
    """gated_scan on packed sequences: x, g [total, D]; seqlens = host sequence of lengths (one at least; lengths of 0 are sequences too); states [len(seqlens), D]."""
    f = _fast(x, stream)
    if f:
        r = f[0].scan_varlen(f[1], f[2], x, g, seqlens, state, logit, mix, h, final_state)
        if r is not None:
            return r
    _one_device(x, g, state, h, final_state)
    if x.dim() != 2:
        raise ValueError(f"x must be [total, D], not {list(x.shape)}")
    total = x.shape[0]
    with _on(stream, x.device):
        cu, _, n_seq, _, keep = _chunk_offsets(x, seqlens if isinstance(seqlens, (list, tuple)) else list(seqlens), 128, stream)
    r = _scan("gated_scan_varlen", x, g, n_seq, total, (cu, n_seq, total), state, logit, mix, h, final_state, stream)
    r[0]._triinv_keepalive = r[1]._triinv_keepalive = keep  # the launch is asynchronous: the offsets live as long as a result
    return r


def _scan_bwd(where, x, g, h, dh, n_seq, N, where_args, state, dstate, logit, mix, dx, dg, stream):
    D = h.shape[-1]
    if x is None and mix:
        raise ValueError("the gradient with mix needs x")
    _has(x, "x", h.shape, h.dtype)
    _has(g, "g", h.shape, g.dtype)
    g_code = _gate_type(g, h.dtype)
    _has(state, "state", (n_seq, D), torch.float32)
    _has(dstate, "dstate", (n_seq, D), torch.float32)
    (px, sx), (pg, sg), (ph, sh), (pd, sd) = _rows(x if mix else None, "x", 1), _rows(g, "g", 1), _rows(h, "h", 1), _rows(dh, "dh", 1, h.shape, h.dtype)
    with _on(stream, h.device):
        dx = torch.empty(h.shape, dtype=h.dtype, device=h.device) if dx is None else dx
        dg = torch.empty(h.shape, dtype=g.dtype, device=h.device) if dg is None else dg
        dstate0 = None if state is None else torch.empty_like(state)
        ws, n = _scan_workspace(where, N, n_seq, D, h.device)
    (ox, sox), (og, sog) = _rows(dx, "dx", 1, h.shape, h.dtype), _rows(dg, "dg", 1, h.shape, g.dtype)
    st = getattr(binding.lib(), where)(px, pg, ph, _opt(state, "state"), pd, _opt(dstate, "dstate"), ox, og, _opt(dstate0, "dstate0"), _opt(ws, "workspace"), n, *where_args, D,
                                       sx, sg, sh, sd, sox, sog, dtype_code(h.dtype), g_code, _flags(logit, mix), _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, where)
    return dx, dg, dstate0


def gated_scan_bwd(x: Optional[torch.Tensor], g: torch.Tensor, h: torch.Tensor, dh: torch.Tensor, state: Optional[torch.Tensor] = None, dstate: Optional[torch.Tensor] = None,
                   logit: bool = False, mix: bool = False, dx: Optional[torch.Tensor] = None, dg: Optional[torch.Tensor] = None, stream=None):
    """(dx, dg, dstate0) of gated_scan, from its inputs, h as it returned it and the gradients dh of h and dstate (or None) of final_state; dstate0 is None where no
    state was given.  x may be None without mix.  dx and dg may be columns of a wider tensor (a projection's gradient)."""
    f = _fast(h, stream)
    if f:
        r = f[0].scan_bwd(f[1], f[2], x, g, h, dh, state, dstate, logit, mix, dx, dg)
        if r is not None:
            return r
    _one_device(x, g, h, dh, state, dstate, dx, dg)
    if h.dim() != 3:
        raise ValueError(f"h must be [B, Tlen, D], not {list(h.shape)}")
    B, T = h.shape[:2]
    return _scan_bwd("gated_scan_bwd", x, g, h, dh, B, B * T, (B, T), state, dstate, logit, mix, dx, dg, stream)


def gated_scan_bwd_varlen(x: Optional[torch.Tensor], g: torch.Tensor, h: torch.Tensor, dh: torch.Tensor, seqlens, state: Optional[torch.Tensor] = None,
                          dstate: Optional[torch.Tensor] = None, logit: bool = False, mix: bool = False, dx: Optional[torch.Tensor] = None, dg: Optional[torch.Tensor] = None,
                          stream=None):
    """gated_scan_bwd on packed sequences (see gated_scan_varlen)."""
    f = _fast(h, stream)
    if f:
        r = f[0].scan_bwd_varlen(f[1], f[2], x, g, h, dh, seqlens, state, dstate, logit, mix, dx, dg)
        if r is not None:
            return r
    _one_device(x, g, h, dh, state, dstate, dx, dg)
    if h.dim() != 2:
        raise ValueError(f"h must be [total, D], not {list(h.shape)}")
    total = h.shape[0]
    with _on(stream, h.device):
        cu, _, n_seq, _, keep = _chunk_offsets(h, seqlens if isinstance(seqlens, (list, tuple)) else list(seqlens), 128, stream)
    r = _scan_bwd("gated_scan_bwd_varlen", x, g, h, dh, n_seq, total, (cu, n_seq, total), state, dstate, logit, mix, dx, dg, stream)
    for t in r:
        if t is not None:
            t._triinv_keepalive = keep  # the launch is asynchronous: the offsets live as long as a result
    return r


def gated_scan_step(x: torch.Tensor, g: torch.Tensor, state: torch.Tensor, slots: Optional[torch.Tensor] = None, logit: bool = False, mix: bool = False,
                    h: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """One token of gated_scan: x, g [B, D]; state [n_slot, D] fp32 is updated in place; the new states' values in x's type are returned.  slots [B] int32: each
    sequence's place in state (outside of it: padding)."""
    f = _fast(x, stream)
    if f:
        r = f[0].scan_step(f[1], f[2], x, g, state, slots, logit, mix, h)
        if r is not None:
            return r
    _one_device(x, g, state, slots, h)
    if x.dim() != 2 or state.dim() != 2:
        raise ValueError(f"x must be [B, D] and state [n_slot, D], not {list(x.shape)} and {list(state.shape)}")
    B, D = x.shape
    _has(g, "g", x.shape, g.dtype)
    g_code = _gate_type(g, x.dtype)
    _has(state, "state", (state.shape[0], D), torch.float32)
    _has(slots, "slots", (B,), torch.int32)
    (px, sx), (pg, sg) = _rows(x, "x", 1), _rows(g, "g", 1)
    if h is None:
        with _on(stream, x.device):
            h = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    ph, sh = _rows(h, "h", 1, x.shape, x.dtype)
    st = binding.lib().gated_scan_step(px, pg, _dev(state, "state"), _opt(slots, "slots"), ph, B, state.shape[0], D, sx, sg, sh, dtype_code(x.dtype), g_code, _flags(logit, mix),
                                       _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, "gated_scan_step")
    return h
