"""The operators of a gated-linear-recurrence block on torch tensors
(argument marshalling only; the kernels are declared in
include/lstm_approx_ops.h).

Every function takes CUDA tensors of one device whose last axis is
contiguous, launches on torch's current stream of that device (or on
``stream``) without waiting for it, and allocates what is not passed in.
Invalid tensors raise ``ValueError``, errors of the library
:class:`LSTMApproxError`.  With ``stream``, the caller orders it after the
work that fills the inputs, as for any other use of a second stream.
"""
from __future__ import annotations

import contextlib
import ctypes
import threading
from typing import Optional

import torch

from ._binding import LSTMApproxError, OK, load

OP_FP32, OP_BF16, OP_FP16, OP_E4M3 = range(4)
SCAN_CHUNK = 64
_CODES = {torch.float32: OP_FP32, torch.bfloat16: OP_BF16, torch.float16: OP_FP16, torch.float8_e4m3fn: OP_E4M3}
_MSG_LEN = 256


_F32, _I32, _U8, _E4M3 = torch.float32, torch.int32, torch.uint8, torch.float8_e4m3fn
_held = threading.local()


def _need(ok: bool, text: str) -> None:
    if not ok:
        raise ValueError(text)


def _check(t, name: str, dev: int, dtype, shape) -> int:
    """The address of a tensor of this device, type and shape whose last axis is contiguous."""
    if t.dtype is not dtype:
        raise ValueError(f"{name} must be {dtype}, not {t.dtype}")
    if t.shape != shape:
        raise ValueError(f"{name} must have the shape {tuple(shape)}, not {tuple(t.shape)}")
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on the CUDA device of the other tensors")
    if not t.is_contiguous() and t.stride(-1) != 1 and t.shape[-1] > 1:
        raise ValueError(f"{name}'s last axis must be contiguous")
    return t.data_ptr()


def _dense(t, name: str, dev: int, dtype, shape) -> Optional[int]:
    """_check of a contiguous tensor; None passes NULL."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != shape or t.get_device() != dev or not t.is_contiguous():
        _check(t, name, dev, dtype, shape)
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _code(t, name: str) -> int:
    c = _CODES.get(t.dtype, OP_E4M3)
    if c == OP_E4M3:
        raise ValueError(f"{name} must be float32, bfloat16 or float16, not {t.dtype}")
    return c


def _pitch(t, name: str) -> int:
    """The element pitch of the rows of t [..., D], which lie at one pitch."""
    if t.dim() == 2:
        return t.stride(0)
    pitch = span = None
    for k in range(t.dim() - 2, -1, -1):
        if t.shape[k] == 1:
            continue
        if pitch is None:
            pitch = span = t.stride(k)
        elif t.stride(k) != span:
            raise ValueError(f"{name}'s rows must lie at one pitch")
        span *= t.shape[k]
    return t.shape[-1] if pitch is None else pitch


@contextlib.contextmanager
def _elsewhere(dev: int, stream, tensors):
    with torch.cuda.device(dev):
        if stream is None:
            yield
        else:
            with torch.cuda.stream(stream):  # what is allocated below belongs to this stream
                yield
            for t in tensors:  # and what came from another one is not handed out again before it is done
                if t is not None:
                    t.record_stream(stream)


_HERE = contextlib.nullcontext()


def _on(dev: int, stream, tensors):
    """The context in which a call launches and allocates."""
    if stream is None and dev == torch._C._cuda_getDevice():
        return _HERE
    return _elsewhere(dev, stream, tensors)


def _call(dev: int, name: str, *args) -> None:
    """lib.name(*args, current stream of dev, msg): raises what it reports."""
    try:
        msg = _held.msg
    except AttributeError:
        msg = _held.msg = ctypes.create_string_buffer(_MSG_LEN)
    rc = getattr(load(), name)(*args, torch._C._cuda_getCurrentRawStream(dev), msg, _MSG_LEN)
    if rc != OK:
        raise LSTMApproxError(rc, msg.value.decode())


def _cuda(t, name: str) -> int:
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be a CUDA tensor")
    return dev


# ---------------------------------------------------------------------------
# norm

def _norm(x, weight, residual, eps, group, out, scales, residual_out, rstd, stream):
    dev, code = _cuda(x, "x"), _code(x, "x")
    shape, D = x.shape, x.shape[-1]
    rows = x.numel() // D if D else 0
    with _on(dev, stream, (x, weight, residual, out, scales, residual_out, rstd)):
        px, pitch, pres, res_pitch = _check(x, "x", dev, x.dtype, shape), _pitch(x, "x"), None, 0
        if residual is not None:
            pres, res_pitch = _check(residual, "residual", dev, x.dtype, shape), _pitch(residual, "residual")
            if residual_out is None:
                residual_out = torch.empty(shape, dtype=x.dtype, device=x.device)
        if group:
            groups = shape[:-1] + (max(1, -(-D // group)),)
            if scales is None:
                scales = torch.empty(groups, dtype=torch.float32, device=x.device)
            _dense(scales, "scales", dev, _F32, groups)
        kind = torch.float8_e4m3fn if group else x.dtype
        if out is None:
            out = torch.empty(shape, dtype=kind, device=x.device)
        _call(dev, "lstm_approx_rms_norm", code, group, px, pitch, pres, res_pitch,
              _dense(weight, "weight", dev, _F32, (D,)), eps, rows, D, _dense(out, "out", dev, kind, shape),
              None if scales is None else scales.data_ptr(), _dense(residual_out, "residual_out", dev, x.dtype, shape),
              _dense(rstd, "rstd", dev, _F32, shape[:-1]))
    return out, scales, residual_out


def rms_norm(x, weight, residual=None, *, eps: float = 1e-6, out=None, residual_out=None, rstd=None, stream=None):
    """Root-mean-square norm over the last axis of s = x (+ residual):
    s / sqrt(mean(s^2) + eps) * weight.

    x, residual [..., D] fp32, bf16 or fp16; weight [D] fp32.  Returns (out,
    s): s in x's type, None without a residual (and without residual_out).
    ``residual_out`` may be ``residual`` itself; ``rstd`` [...] fp32 receives
    1 / sqrt(mean(s^2) + eps) for :func:`rms_norm_backward`.
    """
    out, _, total = _norm(x, weight, residual, eps, 0, out, None, residual_out, rstd, stream)
    return out, total


def rms_norm_quant(x, weight, residual=None, *, eps: float = 1e-6, group: int = 128, out=None, scales=None,
                   residual_out=None, rstd=None, stream=None):
    """:func:`rms_norm` with the output in 8 bits: returns (q, scales, s), q
    [..., D] float8_e4m3fn and scales [..., ceil(D / group)] fp32 with
    q * scale ~ the norm's output.  group: 32, 64, 128, 256 or >= D.
    """
    _need(group > 0, "group must be positive")
    return _norm(x, weight, residual, eps, group, out, scales, residual_out, rstd, stream)


def rms_norm_backward(dy, s, weight, rstd, dsum=None, *, dx=None, dweight=None, workspace=None, stream=None):
    """Gradients of :func:`rms_norm`: (dx, dweight).

    s is the forward call's sum (x itself without a residual), rstd what it
    wrote there, dsum the gradient that reaches s by another way.  dx is the
    gradient of x and of the residual alike; it may be dy or dsum itself.
    """
    dev, code = _cuda(dy, "dy"), _code(dy, "dy")
    shape, D = dy.shape, dy.shape[-1]
    rows = dy.numel() // D if D else 0
    with _on(dev, stream, (dy, s, weight, rstd, dsum, dx, dweight, workspace)):
        if dx is None:
            dx = torch.empty(shape, dtype=dy.dtype, device=dy.device)
        if dweight is None:
            dweight = torch.empty(D, dtype=torch.float32, device=dy.device)
        if workspace is None:
            need = load().lstm_approx_rms_norm_workspace_bytes(rows, D)
            workspace = torch.empty(max(need, 16), dtype=torch.uint8, device=dy.device)
        _call(dev, "lstm_approx_rms_norm_backward", code, _check(dy, "dy", dev, dy.dtype, shape), _pitch(dy, "dy"),
              _check(s, "s", dev, dy.dtype, shape), _pitch(s, "s"), _dense(weight, "weight", dev, _F32, (D,)),
              _dense(rstd, "rstd", dev, _F32, shape[:-1]),
              None if dsum is None else _check(dsum, "dsum", dev, dy.dtype, shape),
              0 if dsum is None else _pitch(dsum, "dsum"), rows, D, _dense(dx, "dx", dev, dy.dtype, shape),
              _dense(dweight, "dweight", dev, _F32, (D,)), workspace.data_ptr(), workspace.nbytes)
    return dx, dweight


# ---------------------------------------------------------------------------
# recurrence

def _strides(*tensors):
    return (ctypes.c_longlong * (2 * len(tensors)))(*(s for t in tensors for s in t.stride()[:2]))


def gated_scan_states(T: int, B: int, D: int, device=None):
    """An empty ``states`` for :func:`gated_scan`: [ceil(T / SCAN_CHUNK), B, D] fp32."""
    return torch.empty(-(-T // SCAN_CHUNK), B, D, dtype=torch.float32, device=device or "cuda")


def gated_scan(x, r, i, decay, h0=None, *, c: float = 8.0, lengths=None, reset=None, y=None, h_last=None,
               states=None, workspace=None, stream=None):
    """The recurrence h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigma(i_t) x_t,
    a_t = exp(-c softplus(decay) sigma(r_t)), over x, r, i [T, B, D] (any t and
    b strides): returns (y, h_last), y_t = h_t in x's type, h_last [B, D] fp32.

    decay [D] fp32; h0 [B, D] fp32 or None; lengths [B] int32: the timesteps
    of each stream; reset [T, B] bool or uint8: where true, the state before
    counts as zero.  ``states`` (:func:`gated_scan_states`) receives what
    :func:`gated_scan_backward` needs.
    """
    dev, code = _cuda(x, "x"), _code(x, "x")
    _need(x.dim() == 3, "x must be [T, B, D]")
    shape = x.shape
    T, B, D = shape
    with _on(dev, stream, (x, r, i, decay, h0, lengths, reset, y, h_last, states, workspace)):
        if y is None:
            y = torch.empty(shape, dtype=x.dtype, device=x.device)
        if h_last is None:
            h_last = torch.empty(B, D, dtype=_F32, device=x.device)
        if workspace is None:
            workspace = _scan_workspace(T, B, D, x.device)
        f32 = _F32
        px, pr, pi, py = (_check(t, n, dev, x.dtype, shape) for t, n in ((x, "x"), (r, "r"), (i, "i"), (y, "y")))
        _call(dev, "lstm_approx_gated_scan", code, px, pr, pi, _dense(decay, "decay", dev, f32, (D,)), c,
              _dense(h0, "h0", dev, f32, (B, D)), _dense(lengths, "lengths", dev, _I32, (B,)),
              _reset(reset, dev, (T, B)), T, B, D, py, _strides(x, r, i, y), _dense(h_last, "h_last", dev, f32, (B, D)),
              _dense(states, "states", dev, f32, (-(-T // SCAN_CHUNK), B, D)), workspace.data_ptr(), workspace.nbytes)
    return y, h_last


def _scan_workspace(T: int, B: int, D: int, device):
    need = load().lstm_approx_gated_scan_workspace_bytes(T, B, D)
    return torch.empty(max(need, 16), dtype=_U8, device=device)


def _reset(reset, dev, shape):
    if reset is None:
        return None
    return _dense(reset, "reset", dev, torch.uint8 if reset.dtype == torch.uint8 else torch.bool, shape)


def gated_scan_backward(dy, x, r, i, decay, states, dh_last=None, *, c: float = 8.0, lengths=None, reset=None,
                        dx=None, dr=None, di=None, ddecay=None, dh0=None, workspace=None, stream=None):
    """Gradients of :func:`gated_scan` (same x, r, i, decay, c, lengths and
    reset; the states it wrote): (dx, dr, di, ddecay, dh0).  dx, dr and di may be
    given with any t and b strides, as slices of one projection's gradient.
    """
    dev, code = _cuda(x, "x"), _code(x, "x")
    _need(x.dim() == 3, "x must be [T, B, D]")
    shape, f32 = x.shape, _F32
    T, B, D = shape
    with _on(dev, stream, (dy, x, r, i, decay, states, dh_last, lengths, reset, dx, dr, di, ddecay, dh0, workspace)):
        dx, dr, di = (torch.empty(shape, dtype=x.dtype, device=x.device) if t is None else t for t in (dx, dr, di))
        if ddecay is None:
            ddecay = torch.empty(D, dtype=f32, device=x.device)
        if dh0 is None:
            dh0 = torch.empty(B, D, dtype=f32, device=x.device)
        if workspace is None:
            workspace = _scan_workspace(T, B, D, x.device)
        pdy, px, pr, pi, pdx, pdr, pdi = (
            _check(t, n, dev, x.dtype, shape)
            for t, n in ((dy, "dy"), (x, "x"), (r, "r"), (i, "i"), (dx, "dx"), (dr, "dr"), (di, "di")))
        _call(dev, "lstm_approx_gated_scan_backward", code, pdy, _dense(dh_last, "dh_last", dev, f32, (B, D)), px, pr, pi,
              _dense(decay, "decay", dev, f32, (D,)), c,
              _dense(states, "states", dev, f32, (-(-T // SCAN_CHUNK), B, D)),
              _dense(lengths, "lengths", dev, _I32, (B,)), _reset(reset, dev, (T, B)), T, B, D, pdx, pdr, pdi,
              _strides(dy, x, r, i, dx, dr, di), _dense(ddecay, "ddecay", dev, f32, (D,)),
              _dense(dh0, "dh0", dev, f32, (B, D)), workspace.data_ptr(), workspace.nbytes)
    return dx, dr, di, ddecay, dh0


def gated_step(x, r, i, decay, state, *, c: float = 8.0, slots=None, reset=None, y=None, stream=None):
    """One timestep of :func:`gated_scan` for x, r, i [B, D]: returns y [B, D]
    and updates state [n_slots, D] fp32 in place.  slots [B] int32: the row of
    state of each stream (None: row b); one outside [0, n_slots) marks an idle
    stream, whose y is zero.  reset [B]: where true the state counts as zero.
    """
    dev, code = _cuda(x, "x"), _code(x, "x")
    _need(x.dim() == 2 and state.dim() == 2, "x must be [B, D] and state [n_slots, D]")
    shape, f32 = x.shape, _F32
    B, D = shape
    with _on(dev, stream, (x, r, i, decay, state, slots, reset, y)):
        if y is None:
            y = torch.empty(shape, dtype=x.dtype, device=x.device)
        _call(dev, "lstm_approx_gated_step", code, _check(x, "x", dev, x.dtype, shape), x.stride(0),
              _check(r, "r", dev, x.dtype, shape), r.stride(0), _check(i, "i", dev, x.dtype, shape), i.stride(0),
              _dense(decay, "decay", dev, f32, (D,)), c, _dense(state, "state", dev, f32, (state.shape[0], D)),
              state.shape[0], _dense(slots, "slots", dev, _I32, (B,)), _reset(reset, dev, (B,)), B, D,
              _dense(y, "y", dev, x.dtype, shape))
    return y


# ---------------------------------------------------------------------------
# 4-bit matrices

class W4Weight:
    """A matrix [N, K] in 4 bits per value: q [N, pitch] uint8 (column k in the
    low or high half of byte k // 2; pitch a multiple of 16), scale [N, ceil(K
    / group)] fp32, bf16 or fp16, zero of the same shape in uint8 or None (8):
    W[n, k] = (q - zero) scale.  Holds the tensors; nothing is copied.
    """

    def __init__(self, q, scale, zero, K: int, group: int):
        dev = _cuda(q, "q")
        _need(K >= 1 and group in (32, 64, 128), "K must be positive and group 32, 64 or 128")
        _need(q.dim() == 2 and q.dtype == torch.uint8 and (q.stride(1) == 1 or q.shape[1] < 2),
              "q must be [N, pitch] uint8 with contiguous rows")
        N, G = q.shape[0], -(-K // group)
        pitch = q.stride(0) if N > 1 else max(q.stride(0), q.shape[1])
        _need(q.shape[1] >= -(-K // 32) * 16 and pitch % 16 == 0 and q.data_ptr() % 16 == 0,
              "q's rows must be 16-byte aligned and hold ceil(K / 32) * 16 bytes")
        self.code = _code(scale, "scale")
        _dense(scale, "scale", dev, scale.dtype, (N, G))
        _dense(zero, "zero", dev, torch.uint8, (N, G))
        self.q, self.scale, self.zero, self.N, self.K, self.group, self.pitch = q, scale, zero, N, K, group, pitch
        self.device_index = dev


def w4_quantize(w, group: int = 128, *, scale_dtype=torch.float16, stream=None) -> W4Weight:
    """w [N, K] (fp32, bf16 or fp16, finite) in 4 bits with a scale and a zero
    point per group of columns, by the rule of lstm_approx_w4_quantize."""
    dev, code = _cuda(w, "w"), _code(w, "w")
    _need(w.dim() == 2 and w.shape[1] >= 1, "w must be [N, K]")
    _need(group in (32, 64, 128), "group must be 32, 64 or 128")
    N, K = w.shape
    G = -(-K // group)
    with _on(dev, stream, (w,)):
        q = torch.empty(N, -(-K // 32) * 16, dtype=torch.uint8, device=w.device)
        scale = torch.empty(N, G, dtype=scale_dtype, device=w.device)
        zero = torch.empty(N, G, dtype=torch.uint8, device=w.device)
        _call(dev, "lstm_approx_w4_quantize", code, _check(w, "w", dev, w.dtype, w.shape), w.stride(0), N, K, group,
              q.data_ptr(), q.shape[1], scale.data_ptr(), _code(scale, "scale"), zero.data_ptr())
        return W4Weight(q, scale, zero, K, group)


def w4_matvec(x, w: W4Weight, *, x_scale=None, bias=None, out=None, out_dtype=None, stream=None):
    """y = x W^T (+ bias) for x [..., K] (a few rows) and a 4-bit matrix W [N, K].

    x: fp32, bf16, fp16, or float8_e4m3fn with x_scale [..., ceil(K / 128)] or
    [..., 1] fp32 (the outputs of :func:`rms_norm_quant`).  bias [N] fp32.
    Returns y [..., N] in out's type, out_dtype, or x's (bf16 for 8-bit x).
    """
    dev, code = _cuda(x, "x"), _CODES.get(x.dtype, -1)
    shape, K, N = x.shape, w.K, w.N
    _need(w.device_index == dev, "x must be on w's device")
    _need(code >= 0 and len(shape) >= 1 and shape[-1] == K, f"x must be floating-point [..., {K}]")
    lead = shape[:-1]
    M = x.numel() // K
    with _on(dev, stream, (x, w.q, w.scale, w.zero, x_scale, bias, out)):
        x_group = 0
        if code == OP_E4M3:
            _need(x_scale is not None, "8-bit x needs x_scale")
            groups = x_scale.shape[-1]
            _need(groups in (1, -(-K // 128)), f"x_scale must be [..., 1] or [..., {-(-K // 128)}]")
            x_group = K if groups == 1 else 128
            _dense(x_scale, "x_scale", dev, torch.float32, lead + (groups,))
        else:
            _need(x_scale is None, "x_scale is for 8-bit x")
        if out is None:
            out_dtype = out_dtype or (torch.bfloat16 if code == OP_E4M3 else x.dtype)
            out = torch.empty(lead + (N,), dtype=out_dtype, device=x.device)
        y_code = _code(out, "out")
        _call(dev, "lstm_approx_w4_matvec", code, _check(x, "x", dev, x.dtype, shape), _pitch(x, "x"),
              None if x_scale is None else x_scale.data_ptr(), x_group, w.q.data_ptr(), w.pitch, w.scale.data_ptr(),
              w.code, None if w.zero is None else w.zero.data_ptr(), _dense(bias, "bias", dev, torch.float32, (N,)),
              M, N, K, w.group, _dense(out, "out", dev, out.dtype, lead + (N,)), y_code)
    return out
