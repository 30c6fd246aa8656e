"""The operators of a gated-linear-recurrence block on torch tensors (the
kernels are declared in include/lstm_approx_ops.h).

Every function takes CUDA tensors of one device whose last axis is
contiguous, launches on torch's current stream of that device (or on
``stream``) without waiting for it, and allocates what is not passed in.
Invalid tensors raise ``ValueError``, errors of the library
:class:`LSTMApproxError`.  With ``stream``, the caller orders it after the
work that fills the inputs, as for any other use of a second stream.

Nothing is recorded for torch's differentiation: inputs that require gradients
are read like others, and outputs have no history.  The gradients are calls of
their own.

The tensors are checked and passed on by the compiled module ``_torch_ops``
(csrc/torch_ops.cpp), built with the library.
"""
from __future__ import annotations

import torch

from ._binding import load

load()
try:
    from . import _torch_ops as _ops
except ImportError as e:
    raise RuntimeError("the operators' module _torch_ops is missing or does not load: build it with "
                       "__graft_entry__.build() or python -m paper_1905_00689_gb300.build") from e

OP_FP32, OP_BF16, OP_FP16, OP_E4M3 = range(4)
SCAN_CHUNK = DELTA_CHUNK = 64
_CODES = {torch.float32: OP_FP32, torch.bfloat16: OP_BF16, torch.float16: OP_FP16}


def _need(ok: bool, text: str) -> None:
    if not ok:
        raise ValueError(text)


def _on(stream, function, *args):
    """function(*args) on another stream than the current one: what it allocates belongs to that stream, and what
    the caller passed in is not handed out again before the stream is done with it."""
    with torch.cuda.stream(stream):
        result = function(*args)
    for t in args:
        if isinstance(t, torch.Tensor) and t.is_cuda:
            t.record_stream(stream)
    return result


# ---------------------------------------------------------------------------
# norm

def rms_norm(x, weight, residual=None, *, eps: float = 1e-6, out=None, residual_out=None, rstd=None, sum_low=None,
             stream=None):
    """Root-mean-square norm over the last axis of s = x (+ residual):
    s / sqrt(mean(s^2) + eps) * weight.

    x, residual [..., D] fp32, bf16 or fp16; weight [D] fp32.  Returns (out,
    s): s in x's type, None without a residual (and without residual_out).
    ``residual_out`` may be ``residual`` itself; ``rstd`` [...] fp32 receives
    1 / sqrt(mean(s^2) + eps) for :func:`rms_norm_backward`.

    ``sum_low``: with ``rstd`` and a residual in 16 bits, s has what its rounding
    took off as its attribute ``sum_low`` (int16 [..., D], for the backward pass:
    2 bytes a value written and kept).  False: it is not made.  A tensor: it
    is written there, for callers that keep it themselves, since an attribute
    stays with this one tensor object (``save_for_backward`` of an output loses
    it).
    """
    args = (x, weight, residual, eps, 0, out, None, residual_out, rstd, sum_low)
    out, _, total = _ops.rms_norm(*args) if stream is None else _on(stream, _ops.rms_norm, *args)
    return out, total


def rms_norm_quant(x, weight, residual=None, *, eps: float = 1e-6, group: int = 128, out=None, scales=None,
                   residual_out=None, rstd=None, stream=None):
    """:func:`rms_norm` with the output in 8 bits: returns (q, scales, s), q
    [..., D] float8_e4m3fn and scales [..., ceil(D / group)] fp32 with
    q * scale ~ the norm's output.  group: 32, 64, 128, 256 or >= D.
    """
    _need(group > 0, "group must be positive")
    args = (x, weight, residual, eps, group, out, scales, residual_out, rstd, False)
    return _ops.rms_norm(*args) if stream is None else _on(stream, _ops.rms_norm, *args)


def rms_norm_backward(dy, s, weight, rstd, dsum=None, *, sum_low=None, dx=None, dweight=None, workspace=None,
                      stream=None):
    """Gradients of :func:`rms_norm`: (dx, dweight).

    s is the forward call's sum (x itself without a residual), rstd what it
    wrote there, dsum the gradient that reaches s by another way.  dx is the
    gradient of x and of the residual alike; it may be dy or dsum itself.
    Where s has a ``sum_low`` and s and rstd are what that call left, neither of
    them changed or copied since, the gradients are those of the sum before its
    rounding to 16 bits; else (a copy, say) dweight is off by that rounding.  A
    further norm of s itself has an rstd of its own: its gradients are at s.
    ``sum_low``: the forward call's, where the caller kept it; False: none.
    """
    args = (dy, s, weight, rstd, dsum, dx, dweight, workspace, sum_low)
    return _ops.rms_norm_backward(*args) if stream is None else _on(stream, _ops.rms_norm_backward, *args)


# ---------------------------------------------------------------------------
# recurrence

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
    args = (x, r, i, decay, h0, c, lengths, reset, y, h_last, states, workspace)
    return _ops.gated_scan(*args) if stream is None else _on(stream, _ops.gated_scan, *args)


def gated_scan_backward(dy, x, r, i, decay, states, dh_last=None, *, c: float = 8.0, lengths=None, reset=None,
                        dx=None, dr=None, di=None, ddecay=None, dh0=None, workspace=None, stream=None):
    """Gradients of :func:`gated_scan` (same x, r, i, decay, c, lengths and
    reset; the states it wrote): (dx, dr, di, ddecay, dh0).  dx, dr and di may be
    given with any t and b strides, as slices of one projection's gradient.
    """
    args = (dy, x, r, i, decay, states, dh_last, c, lengths, reset, dx, dr, di, ddecay, dh0, workspace)
    return _ops.gated_scan_backward(*args) if stream is None else _on(stream, _ops.gated_scan_backward, *args)


def gated_step(x, r, i, decay, state, *, c: float = 8.0, slots=None, reset=None, y=None, stream=None):
    """One timestep of :func:`gated_scan` for x, r, i [B, D]: returns y [B, D]
    and updates state [n_slots, D] fp32 in place.  slots [B] int32: the row of
    state of each stream (None: row b); one outside [0, n_slots) marks an idle
    stream, whose y is zero.  reset [B]: where true the state counts as zero.
    """
    args = (x, r, i, decay, state, c, slots, reset, y)
    return _ops.gated_step(*args) if stream is None else _on(stream, _ops.gated_step, *args)


# ---------------------------------------------------------------------------
# recurrence with a matrix state

def delta_scan_states(q, v):
    """An empty ``states`` for :func:`delta_scan` of q [T, B, Hk, Dk] and v [T, B, H, Dv]: [ceil(T / DELTA_CHUNK), B, H,
    Dk + DELTA_CHUNK, Dv] fp32."""
    _need(q.dim() == 4 and v.dim() == 4, "q must be [T, B, Hk, Dk] and v [T, B, H, Dv]")
    return torch.empty(-(-q.shape[0] // DELTA_CHUNK), *v.shape[1:3], q.shape[3] + DELTA_CHUNK, v.shape[3], dtype=torch.float32,
                       device=q.device)


def delta_scan(q, k, v, g, beta, h0=None, *, scale=None, lengths=None, reset=None, o=None, h_last=None, states=None,
               workspace=None, stream=None):
    """The gated delta rule over a sequence: for every stream and value head, with S_t [Dk, Dv] in 32 bits,

        u_t = beta_t (v_t - e^{g_t} S_{t-1}^T k_t);  S_t = e^{g_t} S_{t-1} + k_t u_t^T;  o_t = scale S_t^T q_t

    q, k [T, B, Hk, Dk] and v [T, B, H, Dv] (fp32, bf16 or fp16, any t, b and
    head strides; H a multiple of Hk: value head h goes with query and key head
    h // (H // Hk); Dk <= 128), g (the decay's logarithm, at most 0) and beta
    [T, B, H] fp32.  k is used as it is: models give it length 1.  Returns (o,
    h_last): o [T, B, H, Dv] in v's type, h_last [B, H, Dk, Dv] fp32.

    scale: None for Dk ** -0.5.  h0 [B, H, Dk, Dv] fp32 or None; lengths [B]
    int32: the timesteps of each stream; reset [T, B] bool or uint8: where true, the
    state before counts as zero.  ``states`` (:func:`delta_scan_states`) receives
    what :func:`delta_scan_backward` needs.  h_last may be h0 itself; no other output
    shares memory with an input or another output.  Values are finite, below 2 ** 127.
    """
    args = (q, k, v, g, beta, h0, scale, lengths, reset, o, h_last, states, workspace)
    return _ops.delta_scan(*args) if stream is None else _on(stream, _ops.delta_scan, *args)


def delta_scan_backward(do, q, k, v, g, beta, states, dh_last=None, *, scale=None, lengths=None, reset=None, dq=None,
                        dk=None, dv=None, dg=None, dbeta=None, dh0=None, workspace=None, stream=None):
    """Gradients of :func:`delta_scan` (same q, k, v, g, beta, scale, lengths and
    reset; the states it wrote): (dq, dk, dv, dg, dbeta, dh0), those of q and k
    summed over the value heads that share them.  dq, dk and dv may be given with
    any t, b and head strides, as slices of one projection's gradient.  No output
    shares memory with an input or another output (dh0 may be dh_last itself).
    """
    args = (do, q, k, v, g, beta, states, dh_last, scale, lengths, reset, dq, dk, dv, dg, dbeta, dh0, workspace)
    return _ops.delta_scan_backward(*args) if stream is None else _on(stream, _ops.delta_scan_backward, *args)


def delta_step(q, k, v, g, beta, state, *, scale=None, slots=None, reset=None, o=None, stream=None):
    """One timestep of :func:`delta_scan` for q, k [B, Hk, Dk], v [B, H, Dv], g and
    beta [B, H]: returns o [B, H, Dv] and updates state [n_slots, H, Dk, Dv]
    fp32 in place.  slots [B] int32: the row of
    state of each stream (None: row b); one outside [0, n_slots) marks an idle
    stream, whose o is zero; those in range are distinct.  reset [B]: where true the
    state counts as zero.
    """
    args = (q, k, v, g, beta, state, scale, slots, reset, o)
    return _ops.delta_step(*args) if stream is None else _on(stream, _ops.delta_step, *args)


# ---------------------------------------------------------------------------
# 4-bit matrices

class W4Weight:
    """A matrix [N, K] in 4 bits per value: q [N, pitch] uint8 (column k in the
    low or high half of byte k // 2; pitch a multiple of 16), scale [N, ceil(K
    / group)] fp32, bf16 or fp16, zero of the same shape in uint8 or None (8):
    W[n, k] = (q - zero) scale.  Holds the tensors; nothing is copied.
    """

    def __init__(self, q, scale, zero, K: int, group: int):
        _need(K >= 1 and group in (32, 64, 128), "K must be positive and group 32, 64 or 128")
        _need(q.is_cuda and q.dim() == 2 and q.dtype == torch.uint8 and (q.stride(1) == 1 or q.shape[1] < 2),
              "q must be a CUDA tensor [N, pitch] uint8 with contiguous rows")
        N, G = q.shape[0], -(-K // group)
        pitch = q.stride(0) if N > 1 else max(q.stride(0), q.shape[1])
        _need(q.shape[1] >= -(-K // 32) * 16 and pitch % 16 == 0 and q.data_ptr() % 16 == 0,
              "q's rows must be 16-byte aligned and hold ceil(K / 32) * 16 bytes")
        _need(scale.dtype in _CODES, "scale must be float32, bfloat16 or float16")
        _need(zero is None or zero.dtype == torch.uint8, "zero must be uint8")
        for name, t in (("scale", scale), ("zero", zero)):
            _need(t is None or (t.device == q.device and t.shape == (N, G) and t.is_contiguous()),
                  f"{name} must be contiguous [{N}, {G}] on q's device")
        self.q, self.scale, self.zero, self.N, self.K, self.group, self.pitch = q, scale, zero, N, K, group, pitch


def w4_quantize(w, group: int = 128, *, scale_dtype=torch.float16, stream=None) -> W4Weight:
    """w [N, K] (fp32, bf16 or fp16, finite) in 4 bits with a scale and a zero
    point per group of columns, by the rule of lstm_approx_w4_quantize."""
    _need(w.dim() == 2 and w.shape[1] >= 1, "w must be [N, K]")
    _need(group in (32, 64, 128), "group must be 32, 64 or 128")
    _need(scale_dtype in _CODES, "scale_dtype must be float32, bfloat16 or float16")
    N, K = w.shape

    def run(w):
        q = torch.empty(N, -(-K // 32) * 16, dtype=torch.uint8, device=w.device)
        scale = torch.empty(N, -(-K // group), dtype=scale_dtype, device=w.device)
        zero = torch.empty(N, -(-K // group), dtype=torch.uint8, device=w.device)
        _ops.w4_quantize(w, group, q, scale, zero)
        return W4Weight(q, scale, zero, K, group)
    return run(w) if stream is None else _on(stream, run, w)


def w4_matvec(x, w: W4Weight, *, x_scale=None, bias=None, out=None, out_dtype=None, workspace=None, stream=None):
    """y = x W^T (+ bias) for x [..., K] (a few rows) and a 4-bit matrix W [N, K].

    x: fp32, bf16, fp16, or float8_e4m3fn with x_scale [..., ceil(K / 128)] or
    [..., 1] fp32 (the outputs of :func:`rms_norm_quant`).  bias [N] fp32.
    Returns y [..., N] in out's type, out_dtype, or x's (bf16 for 8-bit x).
    """
    code = -1 if out_dtype is None else _CODES.get(out_dtype, -2)
    _need(code > -2, "out_dtype must be float32, bfloat16 or float16")
    args = (x, w.q, w.scale, w.zero, w.K, w.group, w.pitch, x_scale, bias, out, code, workspace)
    return _ops.w4_matvec(*args) if stream is None else _on(stream, _ops.w4_matvec, *args)


# ---------------------------------------------------------------------------
# updates

class AdamWState:
    """The moving averages that :func:`adamw_step` keeps for a list of tensors:
    exp_avg and exp_avg_sq, lists of tensors of the parameters' shapes.  In
    32 bits both are fp32.  In 8 bits they are float8_e4m3fn with lists of scales,
    [ceil(n / 256)] fp32 for a tensor of n values, one for each 256 of them:
    exp_avg * scale is the average, (exp_avg_sq * scale) ** 2 that of the
    squares.  Holds the tensors; nothing is copied.
    """

    def __init__(self, exp_avg, exp_avg_sq, exp_avg_scale=None, exp_avg_sq_scale=None):
        _need((exp_avg_scale is None) == (exp_avg_sq_scale is None), "both averages have scales, or none")
        lists = [list(x) for x in (exp_avg, exp_avg_sq, exp_avg_scale, exp_avg_sq_scale) if x is not None]
        _need(len({len(x) for x in lists}) == 1, "the lists must be of one length")
        kind = torch.float32 if exp_avg_scale is None else torch.float8_e4m3fn
        _need(all(t.dtype == kind for x in lists[:2] for t in x),
              f"averages must be {kind}" + (" (8-bit ones need scales)" if exp_avg_scale is None else ""))
        self.exp_avg, self.exp_avg_sq = lists[:2]
        self.exp_avg_scale, self.exp_avg_sq_scale = lists[2:] if len(lists) == 4 else (None, None)

    @classmethod
    def zeros(cls, params, bits: int = 32):
        """Averages of zero for `params`, in 32 or 8 bits."""
        _need(bits in (8, 32), "averages have 8 or 32 bits")
        params = list(params)
        if bits == 32:
            return cls(*([torch.zeros(p.shape, dtype=torch.float32, device=p.device) for p in params] for _ in range(2)))
        return cls(*([torch.zeros(p.shape, dtype=torch.uint8, device=p.device).view(torch.float8_e4m3fn) for p in params]
                     for _ in range(2)),
                   *([torch.ones(-(-p.numel() // 256), dtype=torch.float32, device=p.device) for p in params]
                     for _ in range(2)))


def adamw_step(params, grads, state: AdamWState, step, *, lr, betas=(0.9, 0.999), eps: float = 1e-8,
               weight_decay: float = 0.01, copies=None, grad_scale=None, skip=None, seed: int = 0, stream=None) -> None:
    """One AdamW update of many tensors, in place.  For each, with t the step:

        g' = grad_scale g;  m = b1 m + (1 - b1) g';  v = b2 v + (1 - b2) g'^2
        p = p (1 - lr weight_decay) - lr / (1 - b1^t) m / (sqrt(v / (1 - b2^t)) + eps)

    params, grads: lists of contiguous CUDA tensors of one device, fp32, bf16 or
    fp16 each (a parameter in 16 bits is rounded to the nearest, so steps below
    half a unit of it are lost); a gradient of None leaves its tensor as it is.
    What is written overlaps nothing else of the call (a gradient or copy may be the
    parameter itself).
    state: :class:`AdamWState`; 8-bit averages are rounded at random (`seed`, step and
    position choose), so that they move on average by what they should; one that is
    not finite takes those of its 256 values along, from the next step on.  copies: a
    list of tensors (or None) that receive the parameters in a type of their own, as
    the next forward pass reads them.  eps is 0 (where both averages are zero the parameter
    becomes NaN then) or between 2 ** -126 and 2 ** 126.

    step: the number of this update, from 1; or a CUDA int32 tensor of one value that
    holds it, for captured graphs (read, not changed: count it up before the call, in
    the graph).  lr may likewise be a CUDA fp32 tensor.  grad_scale: a CUDA fp32
    tensor of one value (a clipping factor, the reciprocal of a loss scale); skip: a
    CUDA bool of one value, where true nothing changes.
    """
    _need(len(betas) == 2, "betas must be two numbers")
    _need(all(hasattr(x, "__iter__") for x in (params, grads)), "params and grads must be sequences of tensors")
    params, grads, copies = (x if x is None or isinstance(x, (list, tuple)) else list(x) for x in (params, grads, copies))
    args = (params, grads, state.exp_avg, state.exp_avg_sq, state.exp_avg_scale, state.exp_avg_sq_scale, copies, step, lr,
            betas[0], betas[1], eps, weight_decay, grad_scale, skip, seed)
    if stream is None:
        _ops.adamw_step(*args)
        return
    _on(stream, _ops.adamw_step, *args)
    for t in (t for x in args[:7] if x is not None for t in x if isinstance(t, torch.Tensor)):
        t.record_stream(stream)
