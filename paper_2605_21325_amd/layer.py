"""ctypes binding of the layer's operators beside the chunk inverse -- argument marshalling only, as in binding.py: attention over
chunks with one decay per head, the same layer's single token, the root-mean-square norm with the residual's addition.

A call uses the current stream (or `stream`); tensors it makes itself are allocated on it.  Everything must be contiguous and in device memory.
Autograd records none of them (as it does none of binding.py's): a gradient is the call of its own beside each.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import binding
from .binding import OK, TriInvError, _chunk_offsets, _dev, _stream_ptr, dtype_code


def _opt(t: Optional[torch.Tensor], name: str) -> Optional[int]:
    return None if t is None else _dev(t, name)


def _has(t: Optional[torch.Tensor], name: str, shape, dtype) -> None:
    """Refuses a tensor the kernel would misread: the C-ABI sees an address only."""
    if t is None:
        return
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must be {list(shape)}, not {list(t.shape)}")
    if t.dtype != dtype:
        raise TypeError(f"{name} is {t.dtype}, not {dtype}")


def _on(stream, device):
    """Allocations belong to the stream the kernels run on: what is dropped when the call returns goes to work that stands behind them.  A stream
    object of another library stands for its handle (0: the device's default stream)."""
    if stream is None:
        return _NOWHERE
    if not isinstance(stream, torch.cuda.Stream):
        handle = int(stream.cuda_stream)
        stream = torch.cuda.ExternalStream(handle, device=device) if handle else torch.cuda.default_stream(device)
    return torch.cuda.stream(stream)


_connected = None  # the native argument handling that knows these entry points


def _fast(t: torch.Tensor, stream):
    """(native argument handling, device, stream) for a plain call on the current stream, or None (see binding.py)."""
    if binding._lib is not binding._fast_lib or stream is not None or not t.is_cuda:
        return None
    if binding._fast is not _connected:
        _connect()
    dev = binding._device_index()
    return binding._fast, dev, binding._raw_stream(dev)


def _connect() -> None:
    global _connected
    L = binding.lib()
    binding._fast.connect_layer(*(ctypes.cast(f, ctypes.c_void_p).value for f in (
        L.gdn_chunk_attn, L.gdn_chunk_attn_varlen, L.gdn_chunk_attn_workspace, L.gdn_chunk_attn_bwd, L.gdn_chunk_attn_bwd_varlen,
        L.gdn_chunk_attn_bwd_workspace, L.gdn_step, L.add_rms_norm, L.add_rms_norm_bwd)))
    _connected = binding._fast


class _Nothing:
    def __enter__(self):
        return self

    def __exit__(self, *a):
        return False


_NOWHERE = _Nothing()


def _attn_checked(Q, K, U, g, W, state, lead, n_seq):
    H_k, d_k = Q.shape[-2:]
    H, d_v = U.shape[-2:]
    _has(K, "K", (*lead, H_k, d_k), Q.dtype)
    _has(U, "U", (*lead, H, d_v), Q.dtype)
    _has(Q, "Q", (*lead, H_k, d_k), Q.dtype)
    _has(W, "W", (*lead, H, d_k), Q.dtype)
    _has(g, "g", (*lead, H), torch.float32)
    _has(state, "state", (n_seq, H, d_k, d_v), torch.float32)
    return H, H_k, d_k, d_v


def _workspace(n_seq, n_chunk, H, d_k, d_v, has_w, device):
    n = ctypes.c_int64()
    st = binding.lib().gdn_chunk_attn_workspace(n_seq, n_chunk, H, d_k, d_v, has_w, ctypes.byref(n))
    if st != OK:
        raise TriInvError(st, "gdn_chunk_attn")
    return (torch.empty(n.value, dtype=torch.uint8, device=device) if n.value else None), n.value


def gdn_chunk_attn(Q: torch.Tensor, K: torch.Tensor, U: torch.Tensor, g: Optional[torch.Tensor], C: int, W: Optional[torch.Tensor] = None,
                   state: Optional[torch.Tensor] = None, scale: Optional[float] = None, O: Optional[torch.Tensor] = None,
                   final_state: Optional[torch.Tensor] = None, stream=None):
    """(O, final_state) of linear attention with one decay per head, chunk by chunk: Q, K [B, Tlen, H_k, d_k], U [B, Tlen, H, d_v], g the
    chunk-local cumulative log-decay [B, Tlen, H] or None.  With W [B, Tlen, H, d_k] the gated delta rule: U and W as gdn_chunk_tri_solve_multi
    gives them.  state: [B, H, d_k, d_v] fp32, the state before the first token (None: zeros).  scale: d_k ** -0.5 by default."""
    f = _fast(Q, stream)
    if f:
        r = f[0].chunk_attn(f[1], f[2], Q, K, U, g, C, W, state, scale, O, final_state)
        if r is not None:
            return r
    B, T = Q.shape[:2]
    H, H_k, d_k, d_v = _attn_checked(Q, K, U, g, W, state, (B, T), B)
    _has(O, "O", U.shape, U.dtype)
    _has(final_state, "final_state", (B, H, d_k, d_v), torch.float32)
    with _on(stream, U.device):
        O = torch.empty_like(U) if O is None else O
        final_state = torch.empty((B, H, d_k, d_v), dtype=torch.float32, device=U.device) if final_state is None else final_state
        ws, n = _workspace(B, B * ((T + C - 1) // C) if C > 0 else 0, H, d_k, d_v, W is not None, U.device)
    st = binding.lib().gdn_chunk_attn(_dev(Q, "Q"), _dev(K, "K"), _dev(U, "U"), _opt(W, "W"), _opt(g, "g"), _opt(state, "state"), _dev(O, "O"),
                                      _dev(final_state, "final_state"), _opt(ws, "workspace"), n, B, T, H, H_k, d_k, d_v, C, dtype_code(Q.dtype),
                                      d_k ** -0.5 if scale is None else scale, _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, "gdn_chunk_attn")
    return O, final_state


def gdn_chunk_attn_varlen(Q: torch.Tensor, K: torch.Tensor, U: torch.Tensor, g: Optional[torch.Tensor], seqlens, C: int,
                          W: Optional[torch.Tensor] = None, state: Optional[torch.Tensor] = None, scale: Optional[float] = None,
                          O: Optional[torch.Tensor] = None, final_state: Optional[torch.Tensor] = None, stream=None):
    """gdn_chunk_attn on packed sequences: Q, K [total, H_k, d_k], U [total, H, d_v], W [total, H, d_k], g [total, H]; seqlens = host sequence of
    lengths; states [len(seqlens), H, d_k, d_v]."""
    f = _fast(Q, stream)
    if f:
        r = f[0].chunk_attn_varlen(f[1], f[2], Q, K, U, g, seqlens, C, W, state, scale, O, final_state)
        if r is not None:
            return r
    total = Q.shape[0]
    seqlens = seqlens if isinstance(seqlens, (list, tuple)) else list(seqlens)
    n_seq = len(seqlens)
    H, H_k, d_k, d_v = _attn_checked(Q, K, U, g, W, state, (total,), n_seq)
    _has(O, "O", U.shape, U.dtype)
    _has(final_state, "final_state", (n_seq, H, d_k, d_v), torch.float32)
    with _on(stream, U.device):
        cu_s, cu_c, n_seq, n_chunk, keep = _chunk_offsets(Q, seqlens, C, stream)
        O = torch.empty_like(U) if O is None else O
        final_state = torch.empty((n_seq, H, d_k, d_v), dtype=torch.float32, device=U.device) if final_state is None else final_state
        ws, n = _workspace(n_seq, n_chunk, H, d_k, d_v, W is not None, U.device)
    st = binding.lib().gdn_chunk_attn_varlen(_dev(Q, "Q"), _dev(K, "K"), _dev(U, "U"), _opt(W, "W"), _opt(g, "g"), _opt(state, "state"), _dev(O, "O"),
                                             _dev(final_state, "final_state"), _opt(ws, "workspace"), n, cu_s, cu_c, n_seq, total, n_chunk, H, H_k, d_k, d_v,
                                             C, dtype_code(Q.dtype), d_k ** -0.5 if scale is None else scale, _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, "gdn_chunk_attn_varlen")
    O._triinv_keepalive = final_state._triinv_keepalive = keep  # the launch is asynchronous: the offsets live as long as a result
    return O, final_state


def _attn_bwd(where, Q, K, U, g, dO, C, W, state, dstate, scale, stream, lead, n_seq, n_token, n_chunk, map_args):
    H, H_k, d_k, d_v = _attn_checked(Q, K, U, g, W, state, lead, n_seq)
    _has(dO, "dO", U.shape, U.dtype)
    _has(dstate, "dstate", (n_seq, H, d_k, d_v), torch.float32)
    size = ctypes.c_int64()
    st = binding.lib().gdn_chunk_attn_bwd_workspace(n_token, n_chunk, H, d_k, d_v, C, W is not None, ctypes.byref(size))
    if st != OK:
        raise TriInvError(st, where)
    with _on(stream, U.device):
        dQ, dK, dU = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(U)
        dW = None if W is None else torch.empty_like(W)
        dg = None if g is None else torch.empty_like(g)
        dstate0 = None if state is None else torch.empty_like(state)
        ws = torch.empty(max(16, size.value), dtype=torch.uint8, device=U.device)
    st = getattr(binding.lib(), where)(_dev(Q, "Q"), _dev(K, "K"), _dev(U, "U"), _opt(W, "W"), _opt(g, "g"), _opt(state, "state"), _dev(dO, "dO"), _opt(dstate, "dstate"),
                                       _dev(dQ, "dQ"), _dev(dK, "dK"), _dev(dU, "dU"), _opt(dW, "dW"), _opt(dg, "dg"), _opt(dstate0, "dstate0"), _dev(ws, "workspace"),
                                       ws.numel(), *map_args, H, H_k, d_k, d_v, C, dtype_code(Q.dtype), d_k ** -0.5 if scale is None else scale, _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, where)
    return dQ, dK, dU, dW, dg, dstate0


def gdn_chunk_attn_bwd(Q: torch.Tensor, K: torch.Tensor, U: torch.Tensor, g: Optional[torch.Tensor], dO: torch.Tensor, C: int, W: Optional[torch.Tensor] = None,
                       state: Optional[torch.Tensor] = None, dstate: Optional[torch.Tensor] = None, scale: Optional[float] = None, stream=None):
    """(dQ, dK, dU, dW, dg, dstate0) of gdn_chunk_attn, from its inputs and the gradients dO of O and dstate (or None) of final_state; None in the
    place of the gradient of what was not given."""
    f = _fast(Q, stream)
    if f:
        r = f[0].chunk_attn_bwd(f[1], f[2], Q, K, U, g, dO, C, W, state, dstate, scale)
        if r is not None:
            return r
    B, T = Q.shape[:2]
    return _attn_bwd("gdn_chunk_attn_bwd", Q, K, U, g, dO, C, W, state, dstate, scale, stream, (B, T), B, B * T, B * ((T + C - 1) // C) if C > 0 else 0, (B, T))


def gdn_chunk_attn_bwd_varlen(Q: torch.Tensor, K: torch.Tensor, U: torch.Tensor, g: Optional[torch.Tensor], dO: torch.Tensor, seqlens, C: int,
                              W: Optional[torch.Tensor] = None, state: Optional[torch.Tensor] = None, dstate: Optional[torch.Tensor] = None,
                              scale: Optional[float] = None, stream=None):
    """gdn_chunk_attn_bwd on packed sequences (see gdn_chunk_attn_varlen)."""
    f = _fast(Q, stream)
    if f:
        r = f[0].chunk_attn_bwd_varlen(f[1], f[2], Q, K, U, g, dO, seqlens, C, W, state, dstate, scale)
        if r is not None:
            return r
    total = Q.shape[0]
    with _on(stream, Q.device):
        cu_s, cu_c, n_seq, n_chunk, keep = _chunk_offsets(Q, seqlens if isinstance(seqlens, (list, tuple)) else list(seqlens), C, stream)
    got = _attn_bwd("gdn_chunk_attn_bwd_varlen", Q, K, U, g, dO, C, W, state, dstate, scale, stream, (total,), n_seq, total, n_chunk,
                    (cu_s, cu_c, n_seq, total, n_chunk))
    for x in got:
        if x is not None:
            x._triinv_keepalive = keep  # the launch is asynchronous: the offsets live as long as a result
    return got


def gdn_step(q: torch.Tensor, k: torch.Tensor, v: torch.Tensor, g: Optional[torch.Tensor], state: torch.Tensor, beta: Optional[torch.Tensor] = None,
             slots: Optional[torch.Tensor] = None, scale: Optional[float] = None, o: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """One token of the layer: q, k [B, H_k, d_k], v [B, H, d_v], g [B, H] the token's log-decay or None; state [n_slot, H, d_k, d_v] fp32 is
    updated in place.  beta [B, H]: the delta rule.  slots [B] int32: each sequence's place in state (outside of it: padding)."""
    f = _fast(q, stream)
    if f:
        r = f[0].step(f[1], f[2], q, k, v, g, state, beta, slots, scale, o)
        if r is not None:
            return r
    B, H_k, d_k = q.shape
    H, d_v = v.shape[1:]
    _has(k, "k", q.shape, q.dtype)
    _has(v, "v", (B, H, d_v), q.dtype)
    _has(g, "g", (B, H), torch.float32)
    _has(beta, "beta", (B, H), torch.float32)
    _has(slots, "slots", (B,), torch.int32)
    _has(state, "state", (state.shape[0], H, d_k, d_v), torch.float32)
    _has(o, "o", v.shape, v.dtype)
    if o is None:
        with _on(stream, v.device):
            o = torch.empty_like(v)
    st = binding.lib().gdn_step(_dev(q, "q"), _dev(k, "k"), _dev(v, "v"), _opt(g, "g"), _opt(beta, "beta"), _dev(state, "state"), _opt(slots, "slots"),
                                _dev(o, "o"), B, state.shape[0], H, H_k, d_k, d_v, dtype_code(q.dtype), d_k ** -0.5 if scale is None else scale, _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, "gdn_step")
    return o


def _norm(x, weight, residual, eps, group, y, scales, stream):
    D = x.shape[-1]
    N = x.numel() // D if D else 0
    _has(weight, "weight", (D,), x.dtype)
    _has(residual, "residual", x.shape, x.dtype)
    with _on(stream, x.device):
        total = None if residual is None else torch.empty_like(x)
    st = binding.lib().add_rms_norm(_dev(x, "x"), _opt(residual, "residual"), _dev(weight, "weight"), _dev(y, "y"), _opt(scales, "scales"), _opt(total, "sum"), N, D,
                                    group, dtype_code(x.dtype), eps, _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, "add_rms_norm")
    return x if total is None else total


def add_rms_norm(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6, stream=None):
    """(y, s): s = x + residual in x's type (x itself without one), y = s / sqrt(mean(s^2) + eps) * weight over the last dimension."""
    f = _fast(x, stream)
    if f:
        r = f[0].norm(f[1], f[2], x, weight, residual, eps, -1)
        if r is not None:
            return r
    with _on(stream, x.device):
        y = torch.empty_like(x)
    return y, _norm(x, weight, residual, eps, -1, y, None, stream)


def add_rms_norm_fp8(x: torch.Tensor, weight: torch.Tensor, residual: Optional[torch.Tensor] = None, eps: float = 1e-6, group: int = 0, stream=None):
    """(y, scales, s): as add_rms_norm with y / scale in torch.float8_e4m3fn; scales fp32, one a row [...] (group = 0) or one for every 128
    columns [..., D / 128] (group = 128)."""
    f = _fast(x, stream) if group >= 0 else None
    if f:
        r = f[0].norm(f[1], f[2], x, weight, residual, eps, group)
        if r is not None:
            return r
    with _on(stream, x.device):
        y = torch.empty(x.shape, dtype=torch.float8_e4m3fn, device=x.device)
        # (one a row: a trailing dimension of one group)
        scales = torch.empty((*x.shape[:-1], x.shape[-1] // group if group > 0 else 1), dtype=torch.float32, device=x.device)
    return y, scales, _norm(x, weight, residual, eps, group if group >= 0 else -2, y, scales, stream)


def add_rms_norm_bwd(dy: torch.Tensor, s: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6, dsum: Optional[torch.Tensor] = None, stream=None):
    """(dx, dweight) of add_rms_norm: s as it returned it, dsum the gradient that arrives at s itself; dx is that of x and of the residual, dweight fp32."""
    f = _fast(s, stream)
    if f:
        r = f[0].norm_bwd(f[1], f[2], dy, s, weight, eps, dsum)
        if r is not None:
            return r
    D = s.shape[-1]
    N = s.numel() // D if D else 0
    _has(dy, "dy", s.shape, s.dtype)
    _has(weight, "weight", (D,), s.dtype)
    _has(dsum, "dsum", s.shape, s.dtype)
    with _on(stream, s.device):
        dx = torch.empty_like(s)
        dweight = torch.empty(D, dtype=torch.float32, device=s.device)
        ws = torch.empty(max(1, min(N, 512)) * D, dtype=torch.float32, device=s.device)
    st = binding.lib().add_rms_norm_bwd(_dev(dy, "dy"), _dev(s, "s"), _dev(weight, "weight"), _opt(dsum, "dsum"), _dev(dx, "dx"), _dev(dweight, "dweight"),
                                        _dev(ws, "workspace"), 4 * ws.numel(), N, D, dtype_code(s.dtype), eps, _stream_ptr(stream))
    if st != OK:
        raise TriInvError(st, "add_rms_norm_bwd")
    return dx, dweight
