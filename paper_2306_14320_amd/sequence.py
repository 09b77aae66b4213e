"""Binding of the sequence operators of ``libim2win.so``
(``include/im2win_seq.h``): the short causal convolution, its gradients and
its form for single tokens, the root-mean-square norm with the residual's
addition, and the selective state space scan, its gradients and its form for
single tokens.

The ``im2win_*`` functions mirror the C entry points and take device pointers;
the tensor helpers below them check every tensor against the descriptor and
allocate outputs and workspaces with ``torch.empty`` on the call's stream.
Tokens are rows: x is T x D with contiguous channels and a row stride of its
own; ``seq_starts`` (int32, sequences + 1 values on the device) gives the
sequences' first rows, and without it the sequences are of equal length.
Rows that no sequence holds are neither read nor written, so the outputs'
rows there hold what the memory held.
"""
import ctypes
from typing import NamedTuple, Optional

import torch

from . import (_DTYPES, _check, _empty, _stream, _torch_stream, IM2WIN_F32, load_library)

__all__ = [
    "im2win_conv1d_desc", "im2win_causal_conv1d", "im2win_causal_conv1d_backward_workspace_bytes",
    "im2win_causal_conv1d_backward", "im2win_causal_conv1d_step",
    "causal_conv1d_desc_for", "causal_conv1d", "causal_conv1d_backward", "causal_conv1d_step", "Conv1dGradients",
    "im2win_norm_desc", "im2win_add_rms_norm", "im2win_add_rms_norm_fp8",
    "im2win_add_rms_norm_backward_workspace_bytes", "im2win_add_rms_norm_backward",
    "rms_norm_desc_for", "add_rms_norm", "add_rms_norm_fp8", "add_rms_norm_backward",
    "im2win_scan_desc", "im2win_selective_scan_workspace_bytes", "im2win_selective_scan", "im2win_selective_scan_step",
    "im2win_selective_scan_backward_workspace_bytes", "im2win_selective_scan_backward",
    "selective_scan_desc_for", "selective_scan", "selective_scan_backward", "selective_scan_step", "ScanGradients",
]

_P, _SZ, _I64 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int64


class _Desc(ctypes.Structure):
    def __repr__(self):
        return "%s(%s)" % (type(self).__name__, ", ".join("%s=%s" % (f[0], getattr(self, f[0])) for f in self._fields_))


class im2win_conv1d_desc(_Desc):
    """Mirror of the C ``im2win_conv1d_desc``."""
    _fields_ = [("tokens", _I64), ("channels", _I64), ("width", _I64), ("sequences", _I64), ("ld_x", _I64),
                ("dtype", ctypes.c_int32), ("silu", ctypes.c_int32)]


class im2win_norm_desc(_Desc):
    """Mirror of the C ``im2win_norm_desc``."""
    _fields_ = [("tokens", _I64), ("channels", _I64), ("ld_x", _I64), ("block", _I64),
                ("dtype", ctypes.c_int32), ("residual_dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


class im2win_scan_desc(_Desc):
    """Mirror of the C ``im2win_scan_desc``."""
    _fields_ = [("tokens", _I64), ("channels", _I64), ("states", _I64), ("groups", _I64), ("sequences", _I64),
                ("ld_x", _I64), ("ld_dt", _I64), ("ld_z", _I64), ("ld_b", _I64), ("ld_c", _I64),
                ("dtype", ctypes.c_int32), ("softplus", ctypes.c_int32)]


_CONV = ctypes.POINTER(im2win_conv1d_desc)
_SCAN = ctypes.POINTER(im2win_scan_desc)
_NORM = ctypes.POINTER(im2win_norm_desc)

SIGNATURES = {
    "im2win_causal_conv1d": [_CONV] + [_P] * 8,
    "im2win_causal_conv1d_backward_workspace_bytes": [_CONV, ctypes.POINTER(_SZ)],
    "im2win_causal_conv1d_backward": [_CONV] + [_P] * 12 + [_SZ, _P],
    "im2win_causal_conv1d_step": [_CONV] + [_P] * 5 + [_I64, _P, _P],
    "im2win_selective_scan_workspace_bytes": [_SCAN, ctypes.POINTER(_SZ)],
    "im2win_selective_scan": [_SCAN] + [_P] * 13 + [_SZ, _P],
    "im2win_selective_scan_backward_workspace_bytes": [_SCAN, ctypes.POINTER(_SZ)],
    "im2win_selective_scan_backward": [_SCAN] + [_P] * 22 + [_SZ, _P],
    "im2win_selective_scan_step": [_SCAN] + [_P] * 10 + [_I64, _P, _P],
    "im2win_add_rms_norm": [_NORM] + [_P] * 6,
    "im2win_add_rms_norm_fp8": [_NORM] + [_P] * 7,
    "im2win_add_rms_norm_backward_workspace_bytes": [_NORM, ctypes.POINTER(_SZ)],
    "im2win_add_rms_norm_backward": [_NORM] + [_P] * 7 + [_SZ, _P],
}


def _bytes(name, desc):
    out = _SZ()
    _check(getattr(load_library(), name)(ctypes.byref(desc), ctypes.byref(out)))
    return out.value


# ---------------------------------------------------------------------------
# C entry points, same names and arguments (raising Im2winError on failure)
# ---------------------------------------------------------------------------

def im2win_causal_conv1d(desc, x, w, bias, seq_starts, initial_state, y, final_state, stream) -> None:
    _check(load_library().im2win_causal_conv1d(ctypes.byref(desc), x, w, bias, seq_starts, initial_state, y,
                                               final_state, stream))


def im2win_causal_conv1d_backward_workspace_bytes(desc) -> int:
    return _bytes("im2win_causal_conv1d_backward_workspace_bytes", desc)


def im2win_causal_conv1d_backward(desc, dy, x, w, bias, seq_starts, initial_state, d_final_state, dx, dw, dbias,
                                  d_initial_state, workspace, workspace_bytes, stream) -> None:
    _check(load_library().im2win_causal_conv1d_backward(
        ctypes.byref(desc), dy, x, w, bias, seq_starts, initial_state, d_final_state, dx, dw, dbias, d_initial_state,
        workspace, workspace_bytes, stream))


def im2win_causal_conv1d_step(desc, x, w, bias, slots, state, state_slots, y, stream) -> None:
    _check(load_library().im2win_causal_conv1d_step(ctypes.byref(desc), x, w, bias, slots, state, state_slots, y,
                                                    stream))


def im2win_add_rms_norm(desc, x, residual, w, y, h, stream) -> None:
    _check(load_library().im2win_add_rms_norm(ctypes.byref(desc), x, residual, w, y, h, stream))


def im2win_add_rms_norm_fp8(desc, x, residual, w, q, scales, h, stream) -> None:
    _check(load_library().im2win_add_rms_norm_fp8(ctypes.byref(desc), x, residual, w, q, scales, h, stream))


def im2win_add_rms_norm_backward_workspace_bytes(desc) -> int:
    return _bytes("im2win_add_rms_norm_backward_workspace_bytes", desc)


def im2win_add_rms_norm_backward(desc, dy, h, w, d_residual, dx, dw, workspace, workspace_bytes, stream) -> None:
    _check(load_library().im2win_add_rms_norm_backward(ctypes.byref(desc), dy, h, w, d_residual, dx, dw, workspace,
                                                       workspace_bytes, stream))


def im2win_selective_scan_workspace_bytes(desc) -> int:
    return _bytes("im2win_selective_scan_workspace_bytes", desc)


def im2win_selective_scan(desc, x, dt, A, B, C, D, z, dt_bias, seq_starts, initial_state, y, final_state, workspace,
                          workspace_bytes, stream) -> None:
    _check(load_library().im2win_selective_scan(ctypes.byref(desc), x, dt, A, B, C, D, z, dt_bias, seq_starts,
                                                initial_state, y, final_state, workspace, workspace_bytes, stream))


def im2win_selective_scan_backward_workspace_bytes(desc) -> int:
    return _bytes("im2win_selective_scan_backward_workspace_bytes", desc)


def im2win_selective_scan_backward(desc, dy, x, dt, A, B, C, D, z, dt_bias, seq_starts, initial_state, d_final_state,
                                   dx, ddt, dA, dB, dC, dD, dz, ddt_bias, d_initial_state, workspace, workspace_bytes,
                                   stream) -> None:
    _check(load_library().im2win_selective_scan_backward(
        ctypes.byref(desc), dy, x, dt, A, B, C, D, z, dt_bias, seq_starts, initial_state, d_final_state, dx, ddt, dA,
        dB, dC, dD, dz, ddt_bias, d_initial_state, workspace, workspace_bytes, stream))


def im2win_selective_scan_step(desc, x, dt, A, B, C, D, z, dt_bias, slots, state, state_slots, y, stream) -> None:
    _check(load_library().im2win_selective_scan_step(ctypes.byref(desc), x, dt, A, B, C, D, z, dt_bias, slots, state,
                                                     state_slots, y, stream))


# ---------------------------------------------------------------------------
# Tensor helpers
# ---------------------------------------------------------------------------

def _torch_dtype(desc):
    return torch.float32 if desc.dtype == IM2WIN_F32 else torch.bfloat16


def _dtype_code(dtype):
    if dtype not in _DTYPES:
        raise ValueError(f"unsupported dtype {dtype} (float32 or bfloat16)")
    return _DTYPES[dtype]


def _row_stride(t, name):
    """Elements from one row to the next of a tensor whose rows are contiguous
    (its trailing dimensions, without gaps)."""
    if not isinstance(t, torch.Tensor) or t.dim() < 2:
        raise ValueError(f"{name} must be a tensor of rows")
    width = 1
    for size, stride in zip(reversed(t.shape[1:]), reversed(t.stride()[1:])):
        if size != 1 and stride != width:
            raise ValueError(f"{name}: the elements of a row must lie one behind the other")
        width *= size
    return t.stride(0) if t.shape[0] > 1 else width


def _device_of(t, name):
    """The index of t's device, which has to be the current one (the call
    launches there)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    dev = t.get_device()
    if dev != torch._C._cuda_getDevice():
        raise ValueError(f"{name} is on device {dev}, the current device is {torch.cuda.current_device()}")
    return dev


def _refuse(t, name, shape, dtype, dev, layout):
    """Says what is wrong with t, which no fast check accepted."""
    if not isinstance(t, torch.Tensor) or t.get_device() != dev:
        raise ValueError(f"{name} must be a tensor on device {dev}")
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, the call needs {shape}")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, the call needs {dtype}")
    raise ValueError(f"{name} {layout}")


def _rows(t, name, shape, dtype, ld, dev):
    """Pointer of a T x ... input whose rows are ld elements apart."""
    if isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype and t.get_device() == dev:
        strides = t.stride()
        if strides[0] == ld and strides[-1] == 1 and len(strides) == 2:     # the common case
            return t.data_ptr()
        if _row_stride(t, name) == ld or shape[0] <= 1:
            return t.data_ptr()
    return _refuse(t, name, shape, dtype, dev, f"has rows that are not {ld} elements apart, as the descriptor says")


def _dense(t, name, shape, dtype, dev):
    """Pointer of a contiguous tensor; None stays None."""
    if t is None:
        return None
    if isinstance(t, torch.Tensor) and t.shape == shape and t.dtype is dtype and t.is_contiguous() and t.get_device() == dev:
        return t.data_ptr()
    return _refuse(t, name, shape, dtype, dev, "must be contiguous")


def _new(shape, dtype, like, stream):
    """An output on the call's stream."""
    if stream is None:
        return like.new_empty(shape, dtype=dtype)
    return _empty(shape, dtype, like.device, stream)


def _out(t, name, shape, dtype, like, dev, stream):
    """An output and its pointer: t, or a new tensor."""
    if t is None:
        t = _new(shape, dtype, like, stream)
        return t, t.data_ptr()
    return t, _dense(t, name, shape, dtype, dev)


def _workspace(ws, need, like, stream):
    """A workspace of at least `need` bytes, its pointer and size."""
    if ws is None:
        if need == 0:
            return None, None, 0
        ws = _new((need,), torch.uint8, like, stream)
    elif not isinstance(ws, torch.Tensor) or ws.get_device() != like.get_device() or not ws.is_contiguous():
        raise ValueError("workspace must be a contiguous tensor on the inputs' device")
    return ws, ws.data_ptr(), ws.numel() * ws.element_size()


def _stream_on(stream, dev):
    """The call's HIP stream: the device's current one unless one is given."""
    return torch._C._cuda_getCurrentRawStream(dev) if stream is None else _stream(stream)


def causal_conv1d_desc_for(x, w, sequences=1, silu=True) -> im2win_conv1d_desc:
    """Descriptor of the short causal convolution of x (T x D, rows of any
    stride) with the taps w (D x W): `sequences` packed sequences, SiLU on the
    sum unless silu is false."""
    ld = _row_stride(x, "x")
    if x.dim() != 2 or w.dim() != 2 or w.shape[0] != x.shape[1]:
        raise ValueError(f"x must be T x D and w D x W (got {tuple(x.shape)} and {tuple(w.shape)})")
    return im2win_conv1d_desc(x.shape[0], x.shape[1], w.shape[1], sequences, ld, _dtype_code(x.dtype), int(bool(silu)))


def _conv_inputs(x, w, bias, seq_starts, initial_state, d):
    dt, dev = _torch_dtype(d), _device_of(x, "x")
    return dev, dt, (
        _rows(x, "x", (d.tokens, d.channels), dt, d.ld_x, dev),
        _dense(w, "w", (d.channels, d.width), dt, dev),
        _dense(bias, "bias", (d.channels,), dt, dev),
        _dense(seq_starts, "seq_starts", (d.sequences + 1,), torch.int32, dev),
        _dense(initial_state, "initial_state", (d.sequences, d.width - 1, d.channels), dt, dev))


def causal_conv1d(x, w, desc, bias=None, seq_starts=None, initial_state=None, y=None, final_state=None, stream=None):
    """y[t] = act(bias + sum_k w[:, k] x[t - W + 1 + k]), T x D in x's dtype.
    The inputs before a sequence are initial_state's (sequences x W-1 x D) or
    zero; final_state, if given, receives each sequence's last W-1 inputs."""
    dev, dt, (xp, wp, bp, sp, ip) = _conv_inputs(x, w, bias, seq_starts, initial_state, desc)
    y, yp = _out(y, "y", (desc.tokens, desc.channels), dt, x, dev, stream)
    fp = _dense(final_state, "final_state", (desc.sequences, desc.width - 1, desc.channels), dt, dev)
    im2win_causal_conv1d(desc, xp, wp, bp, sp, ip, yp, fp, _stream_on(stream, dev))
    return y


class Conv1dGradients(NamedTuple):
    dx: torch.Tensor                # T x D, x's dtype
    dw: torch.Tensor                # D x W, fp32
    dbias: Optional[torch.Tensor]   # D, fp32; None without a bias
    d_initial_state: Optional[torch.Tensor]


def causal_conv1d_backward(dy, x, w, desc, bias=None, seq_starts=None, initial_state=None, d_final_state=None,
                           workspace=None, stream=None) -> Conv1dGradients:
    """Gradients of causal_conv1d for dy (T x D, dense) and, where it is given,
    d_final_state.  d_initial_state is returned where initial_state is given."""
    d = desc
    dev, dt, (xp, wp, bp, sp, ip) = _conv_inputs(x, w, bias, seq_starts, initial_state, d)
    state = (d.sequences, d.width - 1, d.channels)
    dyp = _dense(dy, "dy", (d.tokens, d.channels), dt, dev)
    dfp = _dense(d_final_state, "d_final_state", state, dt, dev)
    dx, dxp = _out(None, "dx", (d.tokens, d.channels), dt, x, dev, stream)
    dw, dwp = _out(None, "dw", (d.channels, d.width), torch.float32, x, dev, stream)
    dbias, dbp = (None, None) if bias is None else _out(None, "dbias", (d.channels,), torch.float32, x, dev, stream)
    di, dip = (None, None) if initial_state is None else _out(None, "d_initial_state", state, dt, x, dev, stream)
    workspace, wsp, wsb = _workspace(workspace, im2win_causal_conv1d_backward_workspace_bytes(d), x, stream)
    im2win_causal_conv1d_backward(d, dyp, xp, wp, bp, sp, ip, dfp, dxp, dwp, dbp, dip, wsp, wsb, _stream_on(stream, dev))
    return Conv1dGradients(dx, dw, dbias, di)


def causal_conv1d_step(x, w, state, desc, bias=None, slots=None, y=None, stream=None):
    """One token of each request: x is requests x D, state a pool of slots x
    W-1 x D that moves on in place, slots (int32) the request's place in it
    (its own index when None; outside of the pool: y = 0, nothing moves)."""
    dt, dev = _torch_dtype(desc), _device_of(x, "x")
    xp = _rows(x, "x", (desc.tokens, desc.channels), dt, desc.ld_x, dev)
    wp = _dense(w, "w", (desc.channels, desc.width), dt, dev)
    bp = _dense(bias, "bias", (desc.channels,), dt, dev)
    if not isinstance(state, torch.Tensor):
        raise ValueError("state must be a tensor")
    pool = state.shape[0]
    stp = _dense(state, "state", (pool, desc.width - 1, desc.channels), dt, dev)
    slp = _dense(slots, "slots", (desc.tokens,), torch.int32, dev)
    y, yp = _out(y, "y", (desc.tokens, desc.channels), dt, x, dev, stream)
    im2win_causal_conv1d_step(desc, xp, wp, bp, slp, stp, pool, yp, _stream_on(stream, dev))
    return y


def rms_norm_desc_for(tokens, channels, dtype, residual_dtype=None, eps=1e-5, block=0, ld_x=None) -> im2win_norm_desc:
    """Descriptor of the norm of `tokens` rows: x and y of dtype, the residual
    and h of residual_dtype (dtype when None); block: channels per scale of
    the 8-bit output (0: one scale a row); ld_x: row stride of x."""
    return im2win_norm_desc(tokens, channels, channels if ld_x is None else ld_x, block, _dtype_code(dtype),
                            _dtype_code(residual_dtype or dtype), eps)


def _residual_dtype(desc):
    return torch.float32 if desc.residual_dtype == IM2WIN_F32 else torch.bfloat16


def _norm_inputs(x, w, residual, h, d, stream):
    """x, w, residual, h and their pointers; h is x itself where there is no
    residual, and no other type, to add."""
    dev, shape, rd = _device_of(x, "x"), (d.tokens, d.channels), _residual_dtype(d)
    xp = _rows(x, "x", shape, _torch_dtype(d), d.ld_x, dev)
    wp = _dense(w, "w", (d.channels,), torch.float32, dev)
    rp = _dense(residual, "residual", shape, rd, dev)
    if h is None and residual is None and d.residual_dtype == d.dtype:
        return dev, xp, wp, rp, x, None
    h, hp = _out(h, "h", shape, rd, x, dev, stream)
    return dev, xp, wp, rp, h, hp


def add_rms_norm(x, w, desc, residual=None, y=None, h=None, stream=None):
    """(y, h): h = x + residual in the residual's type, y = h / rms(h) * w in
    x's.  h may be the residual itself (the sum in place); without a residual
    of another type h is x."""
    dev, xp, wp, rp, h, hp = _norm_inputs(x, w, residual, h, desc, stream)
    y, yp = _out(y, "y", (desc.tokens, desc.channels), _torch_dtype(desc), x, dev, stream)
    im2win_add_rms_norm(desc, xp, rp, wp, yp, hp, _stream_on(stream, dev))
    return y, h


def add_rms_norm_fp8(x, w, desc, residual=None, q=None, scales=None, h=None, stream=None):
    """(q, scales, h): y = h / rms(h) * w as float8_e4m3fn values q times one
    fp32 scale for each row or block (T x D/block)."""
    dev, xp, wp, rp, h, hp = _norm_inputs(x, w, residual, h, desc, stream)
    t, d = desc.tokens, desc.channels
    q, qp = _out(q, "q", (t, d), torch.float8_e4m3fn, x, dev, stream)
    scales, sp = _out(scales, "scales", (t, d // (desc.block or d)), torch.float32, x, dev, stream)
    im2win_add_rms_norm_fp8(desc, xp, rp, wp, qp, sp, hp, _stream_on(stream, dev))
    return q, scales, h


def add_rms_norm_backward(dy, h, w, desc, d_residual=None, dx=None, workspace=None, stream=None):
    """(dx, dw) for dy and the gradient d_residual that h has from elsewhere:
    dx (the residual's type; may be d_residual itself) is the gradient of both
    x and the residual, dw is fp32.  An h whose rows have gaps (x itself, as
    add_rms_norm returns it without a residual) is copied to a dense one."""
    dev, shape, rd = _device_of(dy, "dy"), (desc.tokens, desc.channels), _residual_dtype(desc)
    dyp = _dense(dy, "dy", shape, _torch_dtype(desc), dev)
    if isinstance(h, torch.Tensor) and h.shape == shape and not h.is_contiguous():
        _rows(h, "h", shape, rd, _row_stride(h, "h"), dev)
        if stream is None:
            h = h.contiguous()
        else:
            with torch.cuda.stream(_torch_stream(stream)):
                h = h.contiguous()
    hp = _dense(h, "h", shape, rd, dev)
    wp = _dense(w, "w", (desc.channels,), torch.float32, dev)
    drp = _dense(d_residual, "d_residual", shape, rd, dev)
    dx, dxp = _out(dx, "dx", shape, rd, dy, dev, stream)
    dw, dwp = _out(None, "dw", (desc.channels,), torch.float32, dy, dev, stream)
    workspace, wsp, wsb = _workspace(workspace, im2win_add_rms_norm_backward_workspace_bytes(desc), dy, stream)
    im2win_add_rms_norm_backward(desc, dyp, hp, wp, drp, dxp, dwp, wsp, wsb, _stream_on(stream, dev))
    return dx, dw


def selective_scan_desc_for(x, dt, A, B, C, z=None, sequences=1, softplus=True) -> im2win_scan_desc:
    """Descriptor of the selective scan of x and dt (T x D), A (D x N), B and
    C (T x G x N) and the gate z (T x D or None); rows may have any stride."""
    if x.dim() != 2 or A.dim() != 2 or B.dim() != 3 or A.shape[0] != x.shape[1] or B.shape[2] != A.shape[1]:
        raise ValueError("x must be T x D, A D x N and B T x G x N (got %s, %s and %s)"
                         % (tuple(x.shape), tuple(A.shape), tuple(B.shape)))
    t, d = x.shape
    return im2win_scan_desc(t, d, A.shape[1], B.shape[1], sequences, _row_stride(x, "x"), _row_stride(dt, "dt"),
                            d if z is None else _row_stride(z, "z"), _row_stride(B, "B"), _row_stride(C, "C"),
                            _dtype_code(x.dtype), int(bool(softplus)))


def _scan_inputs(x, dt, A, B, C, D, z, dt_bias, d):
    """The device, the element type and the pointers of the scan's inputs."""
    dev, ty = _device_of(x, "x"), _torch_dtype(d)
    rows, proj = (d.tokens, d.channels), (d.tokens, d.groups, d.states)
    return dev, ty, (
        _rows(x, "x", rows, ty, d.ld_x, dev),
        _rows(dt, "dt", rows, ty, d.ld_dt, dev),
        _dense(A, "A", (d.channels, d.states), torch.float32, dev),
        _rows(B, "B", proj, ty, d.ld_b, dev),
        _rows(C, "C", proj, ty, d.ld_c, dev),
        _dense(D, "D", (d.channels,), torch.float32, dev),
        None if z is None else _rows(z, "z", rows, ty, d.ld_z, dev),
        _dense(dt_bias, "dt_bias", (d.channels,), torch.float32, dev))


def selective_scan(x, dt, A, B, C, desc, D=None, z=None, dt_bias=None, seq_starts=None, initial_state=None, y=None,
                   final_state=None, workspace=None, stream=None):
    """y of the scan h_t = exp(s_t A) h_{t-1} + s_t x_t B_t, s = softplus(dt +
    dt_bias), y = (C h + D x) silu(z), T x D in x's dtype.  The state before a
    sequence is initial_state's (sequences x D x N, fp32) or zero; final_state,
    if given, receives the state behind each sequence."""
    d = desc
    dev, ty, (xp, dtp, ap, bp, cp, dp, zp, tbp) = _scan_inputs(x, dt, A, B, C, D, z, dt_bias, d)
    state = (d.sequences, d.channels, d.states)
    sp = _dense(seq_starts, "seq_starts", (d.sequences + 1,), torch.int32, dev)
    ip = _dense(initial_state, "initial_state", state, torch.float32, dev)
    fp = _dense(final_state, "final_state", state, torch.float32, dev)
    y, yp = _out(y, "y", (d.tokens, d.channels), ty, x, dev, stream)
    workspace, wsp, wsb = _workspace(workspace, im2win_selective_scan_workspace_bytes(d), x, stream)
    im2win_selective_scan(d, xp, dtp, ap, bp, cp, dp, zp, tbp, sp, ip, yp, fp, wsp, wsb, _stream_on(stream, dev))
    return y


class ScanGradients(NamedTuple):
    dx: torch.Tensor                # T x D, x's dtype
    ddt: torch.Tensor               # T x D, x's dtype
    dA: torch.Tensor                # D x N, fp32
    dB: torch.Tensor                # T x G x N, x's dtype
    dC: torch.Tensor                # T x G x N, x's dtype
    dD: Optional[torch.Tensor]      # D, fp32; None without D
    dz: Optional[torch.Tensor]      # T x D, x's dtype; None without a gate
    ddt_bias: Optional[torch.Tensor]          # D, fp32; None without a bias
    d_initial_state: Optional[torch.Tensor]   # sequences x D x N, fp32; None without an initial state


def selective_scan_backward(dy, x, dt, A, B, C, desc, D=None, z=None, dt_bias=None, seq_starts=None,
                            initial_state=None, d_final_state=None, workspace=None, stream=None) -> ScanGradients:
    """Gradients of selective_scan for dy (T x D, dense) and, where it is given,
    d_final_state."""
    d = desc
    dev, ty, (xp, dtp, ap, bp, cp, dp, zp, tbp) = _scan_inputs(x, dt, A, B, C, D, z, dt_bias, d)
    rows, proj, state = (d.tokens, d.channels), (d.tokens, d.groups, d.states), (d.sequences, d.channels, d.states)
    sp = _dense(seq_starts, "seq_starts", (d.sequences + 1,), torch.int32, dev)
    ip = _dense(initial_state, "initial_state", state, torch.float32, dev)
    dyp = _dense(dy, "dy", rows, ty, dev)
    dfp = _dense(d_final_state, "d_final_state", state, torch.float32, dev)

    def new(shape, dtype, wanted=True):
        return _new(shape, dtype, x, stream) if wanted else None

    f32 = torch.float32
    g = ScanGradients(new(rows, ty), new(rows, ty), new((d.channels, d.states), f32), new(proj, ty), new(proj, ty),
                      new((d.channels,), f32, D is not None), new(rows, ty, z is not None),
                      new((d.channels,), f32, dt_bias is not None), new(state, f32, initial_state is not None))
    workspace, wsp, wsb = _workspace(workspace, im2win_selective_scan_backward_workspace_bytes(d), x, stream)
    im2win_selective_scan_backward(d, dyp, xp, dtp, ap, bp, cp, dp, zp, tbp, sp, ip, dfp,
                                   *[None if v is None else v.data_ptr() for v in g], wsp, wsb, _stream_on(stream, dev))
    return g


def selective_scan_step(x, dt, A, B, C, state, desc, D=None, z=None, dt_bias=None, slots=None, y=None, stream=None):
    """One token of each request: inputs have a row for each, state is a pool
    of slots x D x N (fp32) that moves on in place, slots (int32) the
    request's place in it (its own index when None; outside of the pool: y =
    0, nothing moves)."""
    dev, ty, (xp, dtp, ap, bp, cp, dp, zp, tbp) = _scan_inputs(x, dt, A, B, C, D, z, dt_bias, desc)
    if not isinstance(state, torch.Tensor):
        raise ValueError("state must be a tensor")
    pool = state.shape[0]
    stp = _dense(state, "state", (pool, desc.channels, desc.states), torch.float32, dev)
    slp = _dense(slots, "slots", (desc.tokens,), torch.int32, dev)
    y, yp = _out(y, "y", (desc.tokens, desc.channels), ty, x, dev, stream)
    im2win_selective_scan_step(desc, xp, dtp, ap, bp, cp, dp, zp, tbp, slp, stp, pool, yp, _stream_on(stream, dev))
    return y
