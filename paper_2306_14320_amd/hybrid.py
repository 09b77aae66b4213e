"""Binding of the operators of hybrid sequence layers of ``libim2win.so``
(``include/im2win_seq.h``): the gated linear recurrence, its gradients and its
form for single tokens; the norm of queries and keys for each head with the
position rotation and its gradients; and window attention with first tokens
that stay visible, its gradients and its form for single tokens out of a ring
cache.

Conventions are those of ``sequence.py``: the ``im2win_*`` functions mirror
the C entry points and take device pointers, the tensor helpers check every
tensor against the descriptor and allocate outputs and workspaces on the
call's stream, tokens are rows, and ``seq_starts`` gives the sequences' first
rows (equal lengths without it).
"""
import ctypes
from typing import NamedTuple, Optional

import torch

from . import _check, load_library
from .sequence import (_Desc, _P, _SZ, _I64, _bytes, _dense, _device_of, _dtype_code, _new, _out, _row_stride, _rows,
                       _stream_on, _torch_dtype, _workspace)

__all__ = [
    "im2win_recurrence_desc", "im2win_gated_recurrence_chunks", "im2win_gated_recurrence_workspace_bytes",
    "im2win_gated_recurrence", "im2win_gated_recurrence_backward_workspace_bytes", "im2win_gated_recurrence_backward",
    "im2win_gated_recurrence_step",
    "gated_recurrence_desc_for", "gated_recurrence_chunk_states", "gated_recurrence", "gated_recurrence_backward",
    "gated_recurrence_step", "RecurrenceGradients",
    "im2win_qk_desc", "im2win_qk_norm_rope", "im2win_qk_norm_rope_backward_workspace_bytes",
    "im2win_qk_norm_rope_backward",
    "qk_norm_rope_desc_for", "qk_norm_rope", "qk_norm_rope_backward", "QkGradients",
    "im2win_window_desc", "im2win_window_attention", "im2win_window_attention_step_workspace_bytes",
    "im2win_window_attention_step", "im2win_window_attention_backward_workspace_bytes",
    "im2win_window_attention_backward",
    "window_attention_desc_for", "window_attention", "window_attention_backward", "window_attention_step",
    "AttentionGradients",
]


class im2win_recurrence_desc(_Desc):
    """Mirror of the C ``im2win_recurrence_desc``."""
    _fields_ = [("tokens", _I64), ("channels", _I64), ("sequences", _I64), ("ld_x", _I64), ("ld_r", _I64),
                ("ld_i", _I64), ("dtype", ctypes.c_int32), ("c", ctypes.c_float)]


class im2win_qk_desc(_Desc):
    """Mirror of the C ``im2win_qk_desc``."""
    _fields_ = [("tokens", _I64), ("q_heads", _I64), ("k_heads", _I64), ("head_dim", _I64), ("rot_dim", _I64),
                ("ld_q", _I64), ("ld_k", _I64), ("dtype", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("eps", ctypes.c_float)]


class im2win_window_desc(_Desc):
    """Mirror of the C ``im2win_window_desc``."""
    _fields_ = [("tokens", _I64), ("sequences", _I64), ("q_heads", _I64), ("kv_heads", _I64), ("head_dim", _I64),
                ("window", _I64), ("sinks", _I64), ("ld_q", _I64), ("ld_k", _I64), ("ld_v", _I64),
                ("dtype", ctypes.c_int32), ("scale", ctypes.c_float)]


_REC = ctypes.POINTER(im2win_recurrence_desc)
_QK = ctypes.POINTER(im2win_qk_desc)
_WIN = ctypes.POINTER(im2win_window_desc)

SIGNATURES = {
    "im2win_gated_recurrence_chunks": [_REC, ctypes.POINTER(_I64)],
    "im2win_gated_recurrence_workspace_bytes": [_REC, ctypes.POINTER(_SZ)],
    "im2win_gated_recurrence": [_REC] + [_P] * 10 + [_SZ, _P],
    "im2win_gated_recurrence_backward_workspace_bytes": [_REC, ctypes.POINTER(_SZ)],
    "im2win_gated_recurrence_backward": [_REC] + [_P] * 15 + [_SZ, _P],
    "im2win_gated_recurrence_step": [_REC] + [_P] * 6 + [_I64, _P, _P],
    "im2win_qk_norm_rope": [_QK] + [_P] * 9,
    "im2win_qk_norm_rope_backward_workspace_bytes": [_QK, ctypes.POINTER(_SZ)],
    "im2win_qk_norm_rope_backward": [_QK] + [_P] * 13 + [_SZ, _P],
    "im2win_window_attention": [_WIN] + [_P] * 6 + [_I64] + [_P] * 5,
    "im2win_window_attention_step_workspace_bytes": [_WIN, ctypes.POINTER(_SZ)],
    "im2win_window_attention_backward_workspace_bytes": [_WIN, ctypes.POINTER(_SZ)],
    "im2win_window_attention_backward": [_WIN] + [_P] * 11 + [_SZ, _P],
    "im2win_window_attention_step": [_WIN] + [_P] * 5 + [_I64] + [_P] * 4 + [_SZ, _P],
}


# ---------------------------------------------------------------------------
# C entry points, same names and arguments (raising Im2winError on failure)
# ---------------------------------------------------------------------------

def im2win_gated_recurrence_chunks(desc) -> int:
    out = _I64()
    _check(load_library().im2win_gated_recurrence_chunks(ctypes.byref(desc), ctypes.byref(out)))
    return out.value


def im2win_gated_recurrence_workspace_bytes(desc) -> int:
    return _bytes("im2win_gated_recurrence_workspace_bytes", desc)


def im2win_gated_recurrence(desc, x, r, i, lam, seq_starts, initial_state, y, final_state, chunk_states, workspace,
                            workspace_bytes, stream) -> None:
    _check(load_library().im2win_gated_recurrence(ctypes.byref(desc), x, r, i, lam, seq_starts, initial_state, y,
                                                  final_state, chunk_states, workspace, workspace_bytes, stream))


def im2win_gated_recurrence_backward_workspace_bytes(desc) -> int:
    return _bytes("im2win_gated_recurrence_backward_workspace_bytes", desc)


def im2win_gated_recurrence_backward(desc, dy, x, r, i, lam, seq_starts, initial_state, d_final_state, chunk_states,
                                     dx, dr, di, dlam, d_initial_state, workspace, workspace_bytes, stream) -> None:
    _check(load_library().im2win_gated_recurrence_backward(
        ctypes.byref(desc), dy, x, r, i, lam, seq_starts, initial_state, d_final_state, chunk_states, dx, dr, di, dlam,
        d_initial_state, workspace, workspace_bytes, stream))


def im2win_gated_recurrence_step(desc, x, r, i, lam, slots, state, state_slots, y, stream) -> None:
    _check(load_library().im2win_gated_recurrence_step(ctypes.byref(desc), x, r, i, lam, slots, state, state_slots, y,
                                                       stream))


def im2win_qk_norm_rope(desc, q, k, wq, wk, positions, freqs, yq, yk, stream) -> None:
    _check(load_library().im2win_qk_norm_rope(ctypes.byref(desc), q, k, wq, wk, positions, freqs, yq, yk, stream))


def im2win_qk_norm_rope_backward_workspace_bytes(desc) -> int:
    return _bytes("im2win_qk_norm_rope_backward_workspace_bytes", desc)


def im2win_qk_norm_rope_backward(desc, dyq, dyk, q, k, wq, wk, positions, freqs, dq, dk, dwq, dwk, workspace,
                                 workspace_bytes, stream) -> None:
    _check(load_library().im2win_qk_norm_rope_backward(ctypes.byref(desc), dyq, dyk, q, k, wq, wk, positions, freqs, dq,
                                                       dk, dwq, dwk, workspace, workspace_bytes, stream))


def im2win_window_attention(desc, q, k, v, seq_starts, k_cache, v_cache, cache_slots, past, slots, y, lse, stream) -> None:
    _check(load_library().im2win_window_attention(ctypes.byref(desc), q, k, v, seq_starts, k_cache, v_cache,
                                                  cache_slots, past, slots, y, lse, stream))


def im2win_window_attention_step_workspace_bytes(desc) -> int:
    return _bytes("im2win_window_attention_step_workspace_bytes", desc)


def im2win_window_attention_step(desc, q, k, v, k_cache, v_cache, cache_slots, past, slots, y, workspace,
                                 workspace_bytes, stream) -> None:
    _check(load_library().im2win_window_attention_step(ctypes.byref(desc), q, k, v, k_cache, v_cache, cache_slots, past,
                                                       slots, y, workspace, workspace_bytes, stream))


def im2win_window_attention_backward_workspace_bytes(desc) -> int:
    return _bytes("im2win_window_attention_backward_workspace_bytes", desc)


def im2win_window_attention_backward(desc, dy, q, k, v, y, lse, seq_starts, dq, dk, dv, workspace, workspace_bytes,
                                     stream) -> None:
    _check(load_library().im2win_window_attention_backward(ctypes.byref(desc), dy, q, k, v, y, lse, seq_starts, dq, dk,
                                                           dv, workspace, workspace_bytes, stream))


# ---------------------------------------------------------------------------
# Gated linear recurrence
# ---------------------------------------------------------------------------

_F32 = torch.float32


def gated_recurrence_desc_for(x, r, i, sequences=1, c=8.0) -> im2win_recurrence_desc:
    """Descriptor of the gated linear recurrence of x, r and i (T x D, rows of
    any stride): `sequences` packed sequences, c the gate's exponent."""
    if not isinstance(x, torch.Tensor) or x.dim() != 2:
        raise ValueError("x must be T x D")
    return im2win_recurrence_desc(x.shape[0], x.shape[1], sequences, _row_stride(x, "x"), _row_stride(r, "r"),
                                  _row_stride(i, "i"), _dtype_code(x.dtype), c)


def _rec_inputs(x, r, i, lam, d):
    ty, dev, rows = _torch_dtype(d), _device_of(x, "x"), (d.tokens, d.channels)
    return dev, ty, rows, (_rows(x, "x", rows, ty, d.ld_x, dev), _rows(r, "r", rows, ty, d.ld_r, dev),
                           _rows(i, "i", rows, ty, d.ld_i, dev), _dense(lam, "lam", (d.channels,), _F32, dev))


def gated_recurrence_chunk_states(x, desc, stream=None) -> torch.Tensor:
    """A tensor for gated_recurrence's chunk_states (chunks x D, fp32), on x's device."""
    return _new((im2win_gated_recurrence_chunks(desc), desc.channels), _F32, x, stream)


def gated_recurrence(x, r, i, lam, desc, seq_starts=None, initial_state=None, y=None, final_state=None,
                     chunk_states=None, workspace=None, stream=None):
    """y of h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigmoid(i_t) x_t, a_t =
    exp(-c softplus(lam) sigmoid(r_t)), T x D in x's dtype.  The state before a
    sequence is initial_state's (sequences x D, fp32) or zero; final_state, if
    given, receives the state behind each sequence, and chunk_states
    (gated_recurrence_chunk_states) what the gradients would compute again."""
    d = desc
    dev, ty, rows, (xp, rp, ip, lp) = _rec_inputs(x, r, i, lam, d)
    state = (d.sequences, d.channels)
    sp = _dense(seq_starts, "seq_starts", (d.sequences + 1,), torch.int32, dev)
    inp = _dense(initial_state, "initial_state", state, _F32, dev)
    fp = _dense(final_state, "final_state", state, _F32, dev)
    cp = None if chunk_states is None else _dense(chunk_states, "chunk_states", (im2win_gated_recurrence_chunks(d), d.channels), _F32, dev)
    y, yp = _out(y, "y", rows, ty, x, dev, stream)
    workspace, wsp, wsb = _workspace(workspace, im2win_gated_recurrence_workspace_bytes(d), x, stream)
    im2win_gated_recurrence(d, xp, rp, ip, lp, sp, inp, yp, fp, cp, wsp, wsb, _stream_on(stream, dev))
    return y


class RecurrenceGradients(NamedTuple):
    dx: torch.Tensor                # T x D, x's dtype
    dr: torch.Tensor                # T x D, x's dtype
    di: torch.Tensor                # T x D, x's dtype
    dlam: torch.Tensor              # D, fp32
    d_initial_state: Optional[torch.Tensor]   # sequences x D, fp32; None without an initial state


def gated_recurrence_backward(dy, x, r, i, lam, desc, seq_starts=None, initial_state=None, d_final_state=None,
                              chunk_states=None, workspace=None, stream=None) -> RecurrenceGradients:
    """Gradients of gated_recurrence for dy (T x D, dense) and, where it is
    given, d_final_state.  chunk_states is what gated_recurrence wrote for the
    same inputs; without it the forward pass runs again."""
    d = desc
    dev, ty, rows, (xp, rp, ip, lp) = _rec_inputs(x, r, i, lam, d)
    state = (d.sequences, d.channels)
    dyp = _dense(dy, "dy", rows, ty, dev)
    if dyp is None:
        raise ValueError("dy must be a tensor")
    sp = _dense(seq_starts, "seq_starts", (d.sequences + 1,), torch.int32, dev)
    inp = _dense(initial_state, "initial_state", state, _F32, dev)
    dfp = _dense(d_final_state, "d_final_state", state, _F32, dev)
    cp = None if chunk_states is None else _dense(chunk_states, "chunk_states", (im2win_gated_recurrence_chunks(d), d.channels), _F32, dev)
    g = RecurrenceGradients(_new(rows, ty, x, stream), _new(rows, ty, x, stream), _new(rows, ty, x, stream),
                            _new((d.channels,), _F32, x, stream),
                            None if initial_state is None else _new(state, _F32, x, stream))
    workspace, wsp, wsb = _workspace(workspace, im2win_gated_recurrence_backward_workspace_bytes(d), x, stream)
    im2win_gated_recurrence_backward(d, dyp, xp, rp, ip, lp, sp, inp, dfp, cp,
                                     *[None if v is None else v.data_ptr() for v in g], wsp, wsb, _stream_on(stream, dev))
    return g


def gated_recurrence_step(x, r, i, lam, state, desc, slots=None, y=None, stream=None):
    """One token of each request: inputs have a row for each, state is a pool
    of slots x D (fp32) that moves on in place, slots (int32) the request's
    place in it (its own index when None; outside of the pool: y = 0, nothing
    moves)."""
    dev, ty, rows, (xp, rp, ip, lp) = _rec_inputs(x, r, i, lam, desc)
    if not isinstance(state, torch.Tensor):
        raise ValueError("state must be a tensor")
    pool = state.shape[0]
    stp = _dense(state, "state", (pool, desc.channels), _F32, dev)
    slp = _dense(slots, "slots", (desc.tokens,), torch.int32, dev)
    y, yp = _out(y, "y", rows, ty, x, dev, stream)
    im2win_gated_recurrence_step(desc, xp, rp, ip, lp, slp, stp, pool, yp, _stream_on(stream, dev))
    return y


# ---------------------------------------------------------------------------
# Norm of queries and keys with the position rotation
# ---------------------------------------------------------------------------

def qk_norm_rope_desc_for(q, k, rot_dim=None, eps=1e-6, interleaved=False) -> im2win_qk_desc:
    """Descriptor of the norm and rotation of q (T x H x head size) and k (T x
    K x head size), rows of any stride: the first rot_dim channels of a head
    (all when None) are rotated, as pairs (p, p + rot_dim/2), or as neighbours
    where interleaved."""
    lq, lk = _row_stride(q, "q"), _row_stride(k, "k")
    if q.dim() != 3 or k.dim() != 3 or q.shape[0] != k.shape[0] or q.shape[2] != k.shape[2] or q.dtype != k.dtype:
        raise ValueError(f"q must be T x H x D and k T x K x D of one dtype (got {tuple(q.shape)} and {tuple(k.shape)})")
    t, h, dim = q.shape
    return im2win_qk_desc(t, h, k.shape[1], dim, dim if rot_dim is None else rot_dim, lq, lk, _dtype_code(q.dtype),
                          int(bool(interleaved)), eps)


def _qk_inputs(q, k, wq, wk, positions, freqs, d):
    ty, dev = _torch_dtype(d), _device_of(q, "q")
    sq, sk = (d.tokens, d.q_heads, d.head_dim), (d.tokens, d.k_heads, d.head_dim)
    return dev, ty, sq, sk, (
        _rows(q, "q", sq, ty, d.ld_q, dev), _rows(k, "k", sk, ty, d.ld_k, dev),
        _dense(wq, "wq", (d.head_dim,), _F32, dev), _dense(wk, "wk", (d.head_dim,), _F32, dev),
        _dense(positions, "positions", (d.tokens,), torch.int32, dev), _dense(freqs, "freqs", (d.rot_dim // 2,), _F32, dev))


def qk_norm_rope(q, k, wq, wk, desc, positions=None, freqs=None, q_out=None, k_out=None, stream=None):
    """(q', k'): every head's channels x / rms(x) * w, the first rot_dim of them
    rotated by positions[t] * freqs (int32 and fp32; needed where rot_dim > 0).
    q_out may be q itself where q is dense, k_out likewise."""
    dev, ty, sq, sk, (qp, kp, wqp, wkp, pp, fp) = _qk_inputs(q, k, wq, wk, positions, freqs, desc)
    q_out, yqp = _out(q_out, "q_out", sq, ty, q, dev, stream)
    k_out, ykp = _out(k_out, "k_out", sk, ty, q, dev, stream)
    im2win_qk_norm_rope(desc, qp, kp, wqp, wkp, pp, fp, yqp, ykp, _stream_on(stream, dev))
    return q_out, k_out


class QkGradients(NamedTuple):
    dq: torch.Tensor     # T x H x head size, q's dtype
    dk: torch.Tensor     # T x K x head size, q's dtype
    dwq: torch.Tensor    # head size, fp32
    dwk: torch.Tensor    # head size, fp32


def qk_norm_rope_backward(dyq, dyk, q, k, wq, wk, desc, positions=None, freqs=None, dq=None, dk=None, workspace=None,
                          stream=None) -> QkGradients:
    """Gradients of qk_norm_rope for dyq and dyk (dense); dq may be dyq itself,
    dk likewise."""
    dev, ty, sq, sk, (qp, kp, wqp, wkp, pp, fp) = _qk_inputs(q, k, wq, wk, positions, freqs, desc)
    dyqp, dykp = _dense(dyq, "dyq", sq, ty, dev), _dense(dyk, "dyk", sk, ty, dev)
    dq, dqp = _out(dq, "dq", sq, ty, q, dev, stream)
    dk, dkp = _out(dk, "dk", sk, ty, q, dev, stream)
    dwq, dwk = _new((desc.head_dim,), _F32, q, stream), _new((desc.head_dim,), _F32, q, stream)
    workspace, wsp, wsb = _workspace(workspace, im2win_qk_norm_rope_backward_workspace_bytes(desc), q, stream)
    im2win_qk_norm_rope_backward(desc, dyqp, dykp, qp, kp, wqp, wkp, pp, fp, dqp, dkp, dwq.data_ptr(), dwk.data_ptr(),
                                 wsp, wsb, _stream_on(stream, dev))
    return QkGradients(dq, dk, dwq, dwk)


# ---------------------------------------------------------------------------
# Attention with a sliding window
# ---------------------------------------------------------------------------

def window_attention_desc_for(q, k, v, window, sinks=0, sequences=1, scale=None) -> im2win_window_desc:
    """Descriptor of the attention of q (T x H x head size) over k and v (T x K
    x head size), rows of any stride, in `sequences` packed sequences: a token
    sees itself, the window - 1 tokens before it, and the first `sinks` of its
    sequence; scale is head size ** -0.5 when None."""
    ld = [_row_stride(t, n) for t, n in ((q, "q"), (k, "k"), (v, "v"))]
    if q.dim() != 3 or k.dim() != 3 or k.shape != v.shape or q.shape[::2] != k.shape[::2] or not q.dtype == k.dtype == v.dtype:
        raise ValueError("q must be T x H x D, k and v T x K x D, of one dtype (got %s, %s and %s)"
                         % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
    t, h, dim = q.shape
    return im2win_window_desc(t, sequences, h, k.shape[1], dim, window, sinks, *ld, _dtype_code(q.dtype),
                              dim ** -0.5 if scale is None else scale)


def _att_inputs(q, k, v, d):
    ty, dev, rows = _torch_dtype(d), _device_of(q, "q"), (d.tokens, d.q_heads, d.head_dim)
    keys = (d.tokens, d.kv_heads, d.head_dim)
    return dev, ty, rows, (_rows(q, "q", rows, ty, d.ld_q, dev), _rows(k, "k", keys, ty, d.ld_k, dev),
                           _rows(v, "v", keys, ty, d.ld_v, dev))


def _caches(k_cache, v_cache, d, ty, dev):
    """The pointers of both caches and their slots."""
    if not isinstance(k_cache, torch.Tensor) or not isinstance(v_cache, torch.Tensor):
        raise ValueError("k_cache and v_cache must be tensors")
    shape = (k_cache.shape[0], d.sinks + d.window, d.kv_heads, d.head_dim)
    return _dense(k_cache, "k_cache", shape, ty, dev), _dense(v_cache, "v_cache", shape, ty, dev), shape[0]


def window_attention(q, k, v, desc, seq_starts=None, k_cache=None, v_cache=None, past=None, slots=None, y=None,
                     lse=None, stream=None):
    """y = softmax(scale q k) v over the visible keys, T x H x head size in q's
    dtype.  With k_cache and v_cache (slots x (sinks + window) x K x head size)
    the sequences go on from requests that have had past (int32, zeros when
    None) tokens, in the slots named (int32, sequence b's is b when None;
    outside of the cache: y = 0, nothing is kept), and their caches are moved
    on.  lse (T x H, fp32), if given, receives what the gradients need."""
    d = desc
    dev, ty, rows, (qp, kp, vp) = _att_inputs(q, k, v, d)
    sp = _dense(seq_starts, "seq_starts", (d.sequences + 1,), torch.int32, dev)
    kcp = vcp = None
    pool = 0
    if k_cache is not None or v_cache is not None:
        kcp, vcp, pool = _caches(k_cache, v_cache, d, ty, dev)
    pp = _dense(past, "past", (d.sequences,), torch.int32, dev)
    slp = _dense(slots, "slots", (d.sequences,), torch.int32, dev)
    lp = _dense(lse, "lse", (d.tokens, d.q_heads), _F32, dev)
    y, yp = _out(y, "y", rows, ty, q, dev, stream)
    im2win_window_attention(d, qp, kp, vp, sp, kcp, vcp, pool, pp, slp, yp, lp, _stream_on(stream, dev))
    return y


class AttentionGradients(NamedTuple):
    dq: torch.Tensor     # T x H x head size, q's dtype
    dk: torch.Tensor     # T x K x head size, q's dtype
    dv: torch.Tensor     # T x K x head size, q's dtype


def window_attention_backward(dy, q, k, v, y, lse, desc, seq_starts=None, workspace=None, stream=None) -> AttentionGradients:
    """Gradients of window_attention without a cache for dy (dense), with the y
    and lse that it wrote."""
    d = desc
    dev, ty, rows, (qp, kp, vp) = _att_inputs(q, k, v, d)
    keys = (d.tokens, d.kv_heads, d.head_dim)
    for t, name in ((dy, "dy"), (y, "y"), (lse, "lse")):
        if not isinstance(t, torch.Tensor):
            raise ValueError(f"{name} must be a tensor")
    dyp, yp = _dense(dy, "dy", rows, ty, dev), _dense(y, "y", rows, ty, dev)
    lp = _dense(lse, "lse", (d.tokens, d.q_heads), _F32, dev)
    sp = _dense(seq_starts, "seq_starts", (d.sequences + 1,), torch.int32, dev)
    g = AttentionGradients(_new(rows, ty, q, stream), _new(keys, ty, q, stream), _new(keys, ty, q, stream))
    workspace, wsp, wsb = _workspace(workspace, im2win_window_attention_backward_workspace_bytes(d), q, stream)
    im2win_window_attention_backward(d, dyp, qp, kp, vp, yp, lp, sp, *[t.data_ptr() for t in g], wsp, wsb, _stream_on(stream, dev))
    return g


def window_attention_step(q, k, v, k_cache, v_cache, past, desc, slots=None, y=None, workspace=None, stream=None):
    """One token of each request, at position past[i] (int32; not moved on):
    its key and value go to the request's cache, y is the attention over what
    the cache then holds of the request.  slots (int32) as for the other
    single-token calls."""
    d = desc
    dev, ty, rows, (qp, kp, vp) = _att_inputs(q, k, v, d)
    kcp, vcp, pool = _caches(k_cache, v_cache, d, ty, dev)
    pp = _dense(past, "past", (d.tokens,), torch.int32, dev)
    slp = _dense(slots, "slots", (d.tokens,), torch.int32, dev)
    y, yp = _out(y, "y", rows, ty, q, dev, stream)
    workspace, wsp, wsb = _workspace(workspace, im2win_window_attention_step_workspace_bytes(d), q, stream)
    im2win_window_attention_step(d, qp, kp, vp, kcp, vcp, pool, pp, slp, yp, wsp, wsb, _stream_on(stream, dev))
    return y
