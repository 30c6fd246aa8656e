"""The digits of sums of the gated delta rule that cancel: what 32 bits hold of a state, of u and of their gradients reaches
16-bit outputs too."""
import numpy as np
import pytest

import operator_reference as ref

# Neither the upper 8 bits of X nor the next 8 hold its last place; X - Y = 2^-20 is the result's size, exact in 32 bits
X, Y = 1 + 2.0 ** -9 + 2.0 ** -20, 1 + 2.0 ** -9


def run(dtype, T, Dk=16, Dv=16, **values):
    """One stream and head, everything zero but `values` ({name: {index: value}}); o, h_last and the gradients."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    dt = ref.torch_dtype(dtype)

    def make(name, shape, kind=dt):
        t = torch.zeros(shape, dtype=kind, device="cuda")
        for at, v in values.get(name, {}).items():
            t[at] = v
        return t
    q, k = make("q", (T, 1, 1, Dk)), make("k", (T, 1, 1, Dk))
    v, do = make("v", (T, 1, 1, Dv)), make("do", (T, 1, 1, Dv))
    g, beta = make("g", (T, 1, 1), torch.float32), make("beta", (T, 1, 1), torch.float32)
    h0, dh_last = make("h0", (1, 1, Dk, Dv), torch.float32), make("dh_last", (1, 1, Dk, Dv), torch.float32)
    states = delta_scan_states(q, v)
    o, last = delta_scan(q, k, v, g, beta, h0, scale=1.0, states=states)
    grads = delta_scan_backward(do, q, k, v, g, beta, states, dh_last, scale=1.0)
    return [ref.f64(t) for t in (o, last, *grads)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_outputs_of_a_state(cuda_device, dtype):
    """o = S^T q, q = (1, -1): the difference of two rows of the state; no roundings but that of 2^-20, which is none."""
    o = run(dtype, 1, q={(0, 0, 0, 0): 1.0, (0, 0, 0, 1): -1.0}, h0={(0, 0, 0, 3): X, (0, 0, 1, 3): Y})[0]
    want = np.zeros_like(o)
    want[0, 0, 0, 3] = 2.0 ** -20
    np.testing.assert_array_equal(o, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("t", [2, 17, 40, 63])
def test_outputs_of_a_chunk(cuda_device, dtype, t):
    """u_0 = X v_0 and u_1 = Y v_1 along orthogonal keys, read together at t."""
    o = run(dtype, t + 1, k={(0, 0, 0, 0): 1.0, (1, 0, 0, 1): 1.0}, v={(0, 0, 0, 5): 1.0, (1, 0, 0, 5): 1.0},
            beta={(0, 0, 0): X, (1, 0, 0): Y}, q={(t, 0, 0, 0): 1.0, (t, 0, 0, 1): -1.0})[0]
    want = np.zeros_like(o)
    want[t, 0, 0, 5] = 2.0 ** -20
    np.testing.assert_array_equal(o, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_gradients_of_a_key(cuda_device, dtype):
    """dk = dS u, u = (1, -1): the difference of two columns of the state's gradient; dk = -S dv, dv = (1, -1): of the state."""
    dk = run(dtype, 1, v={(0, 0, 0, 2): 1.0, (0, 0, 0, 9): -1.0}, beta={(0, 0, 0): 1.0},
             dh_last={(0, 0, 4, 2): X, (0, 0, 4, 9): Y})[3]
    want = np.zeros_like(dk)
    want[0, 0, 0, 4] = 2.0 ** -20
    np.testing.assert_array_equal(dk, want)
    # du = M^T dO = (1, -1) (q = k); the state's row along k is zero
    dk = run(dtype, 1, q={(0, 0, 0, 0): 1.0}, k={(0, 0, 0, 0): 1.0}, beta={(0, 0, 0): 1.0}, do={(0, 0, 0, 2): 1.0, (0, 0, 0, 9): -1.0},
             h0={(0, 0, 4, 2): X, (0, 0, 4, 9): Y})[3]
    want[0, 0, 0, 4] = -2.0 ** -20
    np.testing.assert_array_equal(dk, want)


@pytest.mark.gpu
def test_decays_inside_a_chunk(cuda_device):
    """A value written at 0 and read at 1 along the same key, with nothing between but the decay g: o = e^g, within a unit of the
    last place of expf, four parts' splits and products and the sum of each, half a unit: 2 + 10 half units.  (2^z of a rounded
    z = g / ln 2 is off by |g| of them.)  The gradient of that value is the same number, made of the same parts."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    B, Dk, Dv = 400, 8, 1
    g = torch.zeros(2, B, 1, device="cuda")
    g[1, :, 0] = -20.0 - 20.0 * torch.rand(B, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    q, k, v = (torch.zeros(2, B, 1, d, device="cuda") for d in (Dk, Dk, Dv))
    q[1, ..., 0], k[0, ..., 0], v[0] = 1.0, 1.0, 1.0
    beta, do = torch.ones(2, B, 1, device="cuda"), torch.zeros(2, B, 1, Dv, device="cuda")
    do[1] = 1.0
    states = delta_scan_states(q, v)
    o, _ = delta_scan(q, k, v, g, beta, states=states, scale=1.0)
    grads = delta_scan_backward(do, q, k, v, g, beta, states, scale=1.0)
    want = np.exp(ref.f64(g[1, :, 0]))
    for got in (o[1, :, 0, 0], grads[2][0, :, 0, 0], grads[0][1, :, 0, 0]):
        assert (np.abs(ref.f64(got) - want) <= 12 * 2.0 ** -24 * want).all()
