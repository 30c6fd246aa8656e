"""Progressive approximate-LSTM inference on GB300 (sm_103a), and the
operators of a gated-linear-recurrence block beside it.

The compute path is the C-ABI library ``liblstm_approx.so`` (CUDA kernels,
declared in include/lstm_approx.h and include/lstm_approx_ops.h); this package
is its thin Python binding.
Importing the package does not load the library; constructing
:class:`LSTMApprox` (or calling :func:`load`) does, and raises if it has not
been built.
"""
from ._binding import (  # noqa: F401
    BF16, FP32, LSTMApprox, LSTMApproxError, dense_run, dense_set_launch_order, dense_workspace_bytes, load, plan,
    run_static, PLAN_KEYS,
    PATH_NONE, PATH_PERSISTENT, PATH_SIMT, PATH_TENSOR,
    OPT_CLUSTER, OPT_FORCE_PATH, OPT_LAUNCH_ORDER, OPT_PERSISTENT_VARIANT, OPT_TAU_LAYOUT, OPT_TENSOR_SEQ,
    OPT_TEST_STALL, OPT_TIMING, OPT_WAIT_LIMIT, OPT_XPROJ,
    Q_CLUSTER, Q_DEVICE_BYTES, Q_LAST_PATH, Q_LAUNCHES, Q_PERSISTENT_VARIANT, Q_TENSOR_LOOP,
    Q_TENSOR_SEQ,
)

# The operators work on torch tensors and are imported (with torch) when first used.
_OPERATORS = (
    "AdamWState", "DELTA_CHUNK", "OP_BF16", "OP_E4M3", "OP_FP16", "OP_FP32", "SCAN_CHUNK", "W4Weight", "adamw_step",
    "delta_scan", "delta_scan_backward", "delta_scan_states", "delta_step", "gated_scan", "gated_scan_backward", "gated_scan_states", "gated_step", "rms_norm", "rms_norm_backward",
    "rms_norm_quant", "w4_matvec", "w4_quantize",
)


def __getattr__(name):
    if name in _OPERATORS:
        from . import _operators
        for n in _OPERATORS:
            globals()[n] = getattr(_operators, n)
        return globals()[name]
    raise AttributeError(f"module {__name__!r} has no attribute {name!r}")


def __dir__():
    return sorted(set(globals()) | set(_OPERATORS))
