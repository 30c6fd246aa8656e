"""The state of the gated delta rule over thousands of timesteps."""
import numpy as np
import pytest

import delta_reference as delta
import operator_reference as ref

U = 2.0 ** -24  # half a unit in the last place, of the value
PRODUCTS = 2.0 ** -18  # of the sum of magnitudes, an error of the products of a chunk; four follow one another


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,Dk,Dv", [("fp32", 64, 16), ("bf16", 64, 40), ("bf16", 128, 20), ("fp16", 33, 17)])
@pytest.mark.parametrize("g", [0.0, -1e-5])
def test_a_state_that_hardly_changes(cuda_device, dtype, Dk, Dv, g):
    """Without decay and with steps of 1e-6 the state takes a rounded addition a chunk, nothing that is cut: half a unit of
    its last place each, 64 of them.  With a decay the chunk's e^G (two units: that of expf and of the correction), below
    one, and the product add three half units.  What the chunks add, 4096 e-6 of what a step sees, has the products'
    error.  The same for the gradient of the state, from the end."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    T, B, H = 4096, 1, 1
    q, k, v, gs, beta = delta.tensors((T, B), H, H, Dk, Dv, dtype, 5)
    gs.fill_(g)
    beta.fill_(1e-6)
    args = (q, k, v, gs, beta)
    gen = torch.Generator(device="cuda").manual_seed(6)
    h0, dh_last = (torch.randn(B, H, Dk, Dv, generator=gen, device="cuda") for _ in range(2))
    do = (torch.randn(T, B, H, Dv, generator=gen, device="cuda") * 2.0 ** -12).to(q.dtype)
    states = delta_scan_states(q, v)
    _, last = delta_scan(*args, h0, states=states, scale=2.0 ** -8)
    grads = delta_scan_backward(do, *args, states, dh_last, scale=2.0 ** -8)
    vals = [ref.f64(t) for t in args]
    _, want = delta.scan(*vals, ref.f64(h0), scale=2.0 ** -8)
    back = delta.scan_backward(ref.f64(do), *vals, ref.f64(h0), scale=2.0 ** -8, dh_last=ref.f64(dh_last))
    halves = (1 if g == 0 else 4) * (T // 64) * U

    def columns(S):
        return np.sqrt((S ** 2).sum(-2)).max()
    seen = np.abs(vals[2]).max() + max(columns(ref.f64(h0)), columns(want))     # |v - S^T k|, of any column
    allowed = halves * np.maximum(np.abs(want), np.abs(ref.f64(h0))) + 4 * PRODUCTS * T * 1e-6 * seen + 2 * U
    assert (np.abs(ref.f64(last) - want) <= allowed).all()
    seen = 1e-6 * columns(back[5]) * 2 + 2.0 ** -8 * np.abs(ref.f64(do)).max()  # beta dU (|k| = 1), and what dO gives
    allowed = halves * np.maximum(np.abs(back[5]), np.abs(ref.f64(dh_last))) + 4 * PRODUCTS * T * seen + 2 * U
    assert (np.abs(ref.f64(grads[5]) - back[5]) <= allowed).all()
