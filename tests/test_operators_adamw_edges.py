"""The AdamW step at the ends of its arguments' and values' ranges."""
import ctypes

import numpy as np
import pytest

import operator_reference as ref
from test_operators_adamw import EINVAL


class Tensor(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("p", "m", "v", "copy", "g", "m_scale", "v_scale")] + \
               [("n", ctypes.c_longlong)] + [(n, ctypes.c_int) for n in ("p_dtype", "g_dtype", "copy_dtype")]


@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [1e-40, 1e-45, 1e-60, 2.0 ** -127, 1e38, 1e300])
def test_eps_without_a_reciprocal_is_refused(lib, bits, eps):
    """0 / eps is 0, and would be 0 times the reciprocal of zero (no call gets as far as a launch here)."""
    t, msg = Tensor(p=256, m=256, v=256, g=256, m_scale=256, v_scale=256, n=10), ctypes.create_string_buffer(256)
    assert lib.lstm_approx_adamw_step(1, ctypes.byref(t), bits, 1, None, 0.1, None, 0.9, 0.99, eps, 0.0, None, None, 0, None,
                                      msg, 256) == EINVAL
    assert b"eps" in msg.value


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("eps", [2.0 ** -126, 2.0 ** 126])
def test_least_and_largest_eps(cuda_device, bits, eps):
    """Averages of zero leave the parameter to its decay; a step of m / (sqrt(v) + eps) is lost beside the largest eps and is
    the rate's size beside the least."""
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    p, g = [torch.ones(300, device="cuda")], [torch.zeros(300, device="cuda")]
    g[0][256:] = 1.0
    adamw_step(p, g, AdamWState.zeros(p, bits), 1, lr=0.25, weight_decay=0.5, eps=eps)
    want = np.full(300, 0.875)
    if eps < 1:
        want[256:] -= 0.25
    ref.check(p[0], want, 1.0, 32 * ref.U32, what="p")
