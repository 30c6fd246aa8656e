"""Channels that forget fast: a_t and the gradients by the size of their own, not by that of the largest channel.

Errors in roundoffs u = 2^-24, with t = -log a and |r|, |i| <= 2.  t: softplus 8 (expf and log1pf), c 1, sigma(r) 11
(2^-22 of the exponential, the reciprocal, one addition, |r| twice for its scaled argument), the product 1: under 24.  a:
4 (2^-22) and t times those of t and of the exponential's argument (2): 4 + 26 t."""
import numpy as np
import pytest

import operator_reference as ref

C = 8.0
U = ref.U32
RATES = np.concatenate([np.geomspace(0.01, 40.0, 120), [0.1249, 0.1251, 0.349, 0.351, 0.69, 0.70, 20.0, 60.0]])


def tensors(T, B, dtype, seed, rates=RATES):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    draw = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    D = len(rates)
    d = torch.tensor(rates / C, dtype=torch.float64)
    decay = torch.where(d > 15, d, torch.log(torch.expm1(d))).float().cuda()
    x, dy = (draw(T, B, D).to(ref.torch_dtype(dtype)) for _ in range(2))
    r, i = (draw(T, B, D).clamp(-2, 2).to(ref.torch_dtype(dtype)) for _ in range(2))
    return x, r, i, decay, dy, draw(B, D)


@pytest.mark.gpu
def test_decay_of_one_timestep(cuda_device):
    """With x = 0 the state is a h and the gradient of h_0 is a g: a itself, relative to itself, forward, in a step and
    back, for t between 0.001 and 50."""
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states, gated_step
    x, r, i, decay, dy, h0 = tensors(1, 40, "fp32", 1)
    x.zero_()
    _, _, la, a, _ = ref.gates(ref.f64(r[0]), ref.f64(i[0]), ref.f64(decay), C)
    tol = (4 + 26 * -la) * U + 2 * U
    states = gated_scan_states(1, *h0.shape)
    _, last = gated_scan(x, r, i, decay, h0, c=C, states=states)
    ref.check(last, a * ref.f64(h0), a * np.abs(ref.f64(h0)), tol, what="scan")
    state = h0.clone()
    gated_step(x[0], r[0], i[0], decay, state, c=C)
    ref.check(state, a * ref.f64(h0), a * np.abs(ref.f64(h0)), tol, what="step")
    dh0 = gated_scan_backward(dy, x, r, i, decay, states, c=C)[4]
    ref.check(dh0, a * ref.f64(dy[0]), a * np.abs(ref.f64(dy[0])), tol, what="dh0")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("T,B", [(1, 3), (70, 2)])
def test_gradients_by_channel(cuda_device, T, B, dtype):
    """dr, ddecay and dh0 of every channel against the magnitudes of its own terms.  A term g a t (si x a / m + h)
    has a twice (52 t + 8), t (24), si, 1 / m and the products (60, with m's own share of t): 92 + 52 t; 1 - sigma(r), up to
    9 times smaller than sigma(r): 100.  Over a sequence the states' and gradients' own errors come twice on top, each
    at most 1 / (1 - a) <= 4 times what one timestep adds (channels with t >= 0.35 where sigma(r) is smallest)."""
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states
    rates = RATES if T == 1 else np.geomspace(3.0, 40.0, 50)
    x, r, i, decay, dy, h0 = tensors(T, B, dtype, 2, rates)
    states = gated_scan_states(T, B, len(rates))
    gated_scan(x, r, i, decay, h0, c=C, states=states)
    _, dr, _, ddecay, dh0 = gated_scan_backward(dy, x, r, i, decay, states, c=C)
    X, R, I, DY, DEC = (ref.f64(v) for v in (x, r, i, dy, decay))
    want = ref.scan_backward(DY, X, R, I, DEC, C, h0=ref.f64(h0))
    sr, si, la, a, m = ref.gates(R, I, DEC, C)
    t = -la
    h, g = np.abs(ref.f64(h0)), np.zeros_like(h0.cpu().numpy(), dtype=np.float64)
    before = np.zeros_like(X)
    for k in range(T):
        before[k] = h
        h = a[k] * h + m[k] * si[k] * np.abs(X[k])
    size = np.zeros_like(X)
    for k in range(T - 1, -1, -1):
        g = g + np.abs(DY[k])
        size[k] = g * a[k] * t[k] * (si[k] * np.abs(X[k]) * a[k] / m[k] + before[k])
        g = g * a[k]
    share = (192 + 52 * t) * U
    if T > 1:
        share = share + 8 * (60 + 52 * t.max(0)) * U
    ref.check(dr, want[1], size * (1 - sr), share, dtype, "dr")
    ratio = ref.sigmoid(DEC) / ref.softplus(DEC)
    ref.check(ddecay, want[3], (size * share).sum((0, 1)) * ratio + T * B * U * size.sum((0, 1)) * ratio, 1.0, what="ddecay")
    ref.check(dh0, want[4], g, (share.max(0) if T > 1 else share[0]) * max(1, T), what="dh0")
