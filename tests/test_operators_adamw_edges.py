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


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("apart", [0, 1])
@pytest.mark.parametrize("eps", [2.0 ** -100, 1e-8])
def test_gradients_of_any_finite_size(cuda_device, bits, apart, eps):
    """A gradient whose square is beyond the type: v is infinite, the parameter stays where its decay takes it, in this step and the
    next, and its neighbours' step is theirs.  One whose square is below 2^-126 (few bits) or none: the step of those bits."""
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    n = 600
    p, g = [torch.ones(n + 1, device="cuda")[apart:apart + n]], [torch.zeros(n + 1, device="cuda")[apart:apart + n]]
    g[0][:] = 0.5
    sizes = {3: 1e20, 40: -3e38, 300: 2.0 ** -70, 301: -2.0 ** -73, 302: 2.0 ** -63, 303: 1.8e19}
    for i, x in sizes.items():
        g[0][i] = x
    state = AdamWState.zeros(p, bits)
    adamw_step(p, g, state, 1, lr=0.25, weight_decay=0.5, betas=(0.5, 0.5), eps=eps)
    # the step of v in 32 bits as it is held: few bits below 2^-126
    grad = ref.f64(g[0]).astype(np.float32)
    with np.errstate(over="ignore"):
        v = (grad * grad) * np.float32(0.5)
    step = 0.25 * grad / (np.sqrt(v.astype(np.float64) * 2.0) + eps)
    ref.check(p[0], 0.875 - step, 1.0 + np.abs(step), 32 * ref.U32, what="p")
    v1 = ref.f64(state.exp_avg_sq[0])
    if bits == 32:
        ref.check(v1, v.astype(np.float64), np.where(np.isinf(v), 0.0, v), 8 * ref.U32, what="v")
    else:
        assert np.isinf(ref.f64(state.exp_avg_sq_scale[0])[0]) and np.isfinite(ref.f64(state.exp_avg_sq_scale[0])[1:]).all()
        assert np.isfinite(ref.f64(state.exp_avg_scale[0])).all()
    before = ref.f64(p[0])
    adamw_step(p, [torch.zeros_like(p[0])], state, 2, lr=0.25, weight_decay=0.5, betas=(0.5, 0.5), eps=eps)
    for i in (3, 40):
        assert abs(float(p[0][i]) - before[i] * 0.875) <= 4 * ref.U32
    assert torch.isfinite(p[0]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("eps", [1e-8, 0.0])
def test_scales_follow_from_the_formula_alone(cuda_device, eps):
    """Each operation rounded by itself, the root as sqrtf's: the bits of the scales of 2^17 blocks, whose largest value an average
    alone makes.  (eps of 0 takes other roots; a parameter whose averages are zero is NaN then.)"""
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    blocks = 1 << 17
    rng = np.random.default_rng(8)
    scale = (rng.random(blocks) + 1).astype(np.float32) * np.float32(2.0) ** rng.integers(-20, 20, blocks).astype(np.float32)
    codes = torch.zeros(blocks, 256, device="cuda")
    codes[:, 77] = 448.0
    codes = codes.to(torch.float8_e4m3fn).view(-1)
    held = torch.tensor(scale, device="cuda")
    state = AdamWState([codes.clone()], [codes.clone()], [held.clone()], [held.clone()])
    p = [torch.zeros(blocks * 256, dtype=torch.bfloat16, device="cuda")]
    adamw_step(p, [torch.zeros_like(p[0])], state, 5, lr=0.1, betas=(0.9, 0.7), eps=eps)
    most, part = np.float32(448) * scale, np.float32(1) / np.float32(448)
    m, u = most * np.float32(0.9), np.sqrt(most * most * np.float32(0.7))
    np.testing.assert_array_equal(state.exp_avg_scale[0].cpu().numpy(), m * part)
    np.testing.assert_array_equal(state.exp_avg_sq_scale[0].cpu().numpy(), u * part)


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_tensors_that_overlap_are_refused(cuda_device, bits):
    """A tensor under two names of which one is written; nothing has changed after a refusal.  Two parameters may share a gradient,
    and tensors may lie one behind the other."""
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    kind = torch.float32 if bits == 32 else torch.float8_e4m3fn
    n = 256

    def flat(count, dtype=torch.float32):
        return torch.ones(count, device="cuda").to(dtype)

    def lists(p=None, g=None, m=None, v=None, ms=None, vs=None, c=None):
        pick = lambda given, make: given if given is not None else [make() for _ in range(2)]  # noqa: E731
        ones = lambda: flat(1)  # noqa: E731
        state = AdamWState(pick(m, lambda: flat(n, kind)), pick(v, lambda: flat(n, kind)),
                           *((pick(ms, ones), pick(vs, ones)) if bits == 8 else ()))
        return dict(params=pick(p, lambda: flat(n)), grads=pick(g, lambda: flat(n)), state=state, copies=c)

    one, two, half = flat(n, kind), flat(n, kind), flat(n, torch.bfloat16)
    p, long, scale = [flat(n), flat(n)], flat(2 * n), flat(1)
    bad = [lists(m=[one, two], v=[flat(n, kind), one]), lists(m=[one, one]), lists(v=[one, one]), lists(c=[half, half]),
           lists(p=p, c=[p[0].view(torch.bfloat16)[:n], None]), lists(p=p, c=[p[1], None]), lists(p=p, g=[flat(n), p[0]]),
           lists(g=[long[:n], flat(n)], c=[long[n - 1:2 * n - 1], None]), lists(p=[long[:n], long[n - 1:-1]])]
    if bits == 8:
        bad += [lists(ms=[scale, scale]), lists(ms=[flat(1), scale], vs=[scale, flat(1)])]
    for args in bad:
        with pytest.raises(ValueError):
            adamw_step(**args, step=1, lr=0.1)
    assert all((x == 1).all() for x in p + [long, scale]) and (one.float() == 1).all() and (half == 1).all()
    g = flat(n)
    good = lists(p=[long[:n], long[n:]], g=[g, g], c=[half, None])
    adamw_step(**good, step=1, lr=0.1)
    assert torch.equal(long[:n], long[n:]) and torch.equal(half, long[:n].bfloat16()) and (long != 1).all()
    good = lists(m=[one, one], g=[flat(n), None])  # (what has no gradient keeps its averages)
    adamw_step(**good, step=1, lr=0.1)
    good, want = lists(p=[flat(n), p[1]], g=[flat(n), p[1]], c=[None, p[1]]), lists()  # itself as its gradient and copy
    adamw_step(**good, step=1, lr=0.1)
    adamw_step(**want, step=1, lr=0.1)
    assert torch.equal(p[1], want["params"][1]) and (p[1] != 1).all()
