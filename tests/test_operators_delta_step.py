"""One timestep of the gated delta rule on a pool of states."""
import ctypes

import numpy as np
import pytest

import delta_reference as delta
import operator_reference as ref

EINVAL = 1


def compare(args, state, got, after, dtype, slots=None, reset=None, scale=None):
    """32-bit sums of Dk products in any order: (Dk + 16) roundoffs of the sum of the magnitudes covers the products, the
    decay (expf: 2 units in the last place) and what is formed of the sums."""
    q, k, v, g, beta = (ref.f64(t) for t in args)
    B, H, Dv = v.shape
    Hk, Dk = q.shape[1:]
    S, S1 = ref.f64(state), ref.f64(after)
    scale = Dk ** -0.5 if scale is None else scale
    tol = (Dk + 16) * ref.U32
    touched = np.zeros(len(S), bool)
    for b in range(B):
        s = b if slots is None else int(slots[b])
        if not 0 <= s < len(S):
            assert (ref.f64(got[b]) == 0).all()
            continue
        touched[s] = True
        W = np.zeros_like(S[s]) if reset is not None and reset[b] else S[s] * np.exp(np.maximum(g[b], -200.0))[:, None, None]
        for h in range(H):
            kt, qt = k[b, h // (H // Hk)], q[b, h // (H // Hk)]
            u = beta[b, h] * (v[b, h] - W[h].T @ kt)
            u_terms = beta[b, h] * (np.abs(v[b, h]) + np.abs(W[h]).T @ np.abs(kt))
            new = W[h] + np.outer(kt, u)
            terms = np.abs(W[h]) + np.outer(np.abs(kt), u_terms)
            ref.check(S1[s, h], new, terms, tol, what="state")
            ref.check(got[b, h], scale * new.T @ qt, scale * terms.T @ np.abs(qt), 2 * tol, dtype, "o")
    np.testing.assert_array_equal(S1[~touched], S[~touched])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,H,Hk,Dk,Dv", [(1, 1, 1, 1, 1), (1, 16, 16, 128, 128), (5, 6, 2, 64, 100), (3, 2, 1, 65, 33),
                                          (7, 3, 3, 17, 4), (2, 4, 2, 127, 31), (9, 1, 1, 16, 260)])
def test_step(cuda_device, B, H, Hk, Dk, Dv, dtype):
    import torch
    from paper_1905_00689_gb300 import delta_step
    args = delta.tensors((B,), H, Hk, Dk, Dv, dtype, 10 + B)
    state = torch.randn(B + 2, H, Dk, Dv, device="cuda")
    after = state.clone()
    compare(args, state, delta_step(*args, after), after, dtype)
    rng = np.random.default_rng(B)
    slots = torch.tensor(rng.permutation(B + 2)[:B], dtype=torch.int32, device="cuda")
    slots[rng.integers(B)] = int(rng.choice([-1, B + 2, 2 ** 31 - 1, -2 ** 31]))
    reset = torch.tensor(rng.random(B) < 0.4, device="cuda")
    after = state.clone()
    after[0] = state[0]
    for b in range(B):  # what a state that counts as zero holds does not matter
        if bool(reset[b]) and 0 <= int(slots[b]) < B + 2:
            after[int(slots[b])] = float("nan")
    o = torch.full((B, H, Dv), float("nan"), dtype=args[0].dtype, device="cuda")
    assert delta_step(*args, after, slots=slots, reset=reset, o=o, scale=0.25) is o
    compare(args, state, o, after, dtype, slots.cpu().numpy(), reset.cpu().numpy(), 0.25)


@pytest.mark.gpu
def test_step_layouts(cuda_device):
    """Slices of one projection's output, broadcast heads, a state at any address: the bits of the contiguous call, or (where
    the address changes which columns share a thread) the same too, since every sum keeps its order."""
    import torch
    from paper_1905_00689_gb300 import delta_step
    B, H, Hk, Dk, Dv = 5, 6, 2, 40, 36
    args = delta.tensors((B,), H, Hk, Dk, Dv, "bf16", 3, fused=True)
    state = torch.randn(B, H, Dk, Dv, device="cuda")
    want_state = state.clone()
    want = delta_step(*[t.contiguous() for t in args], want_state)
    got_state = state.clone()
    out = torch.empty(H, B, Dv, dtype=torch.bfloat16, device="cuda").transpose(0, 1)
    assert torch.equal(delta_step(*args, got_state, o=out), want) and torch.equal(got_state, want_state)
    flat = torch.empty(state.numel() + 1, device="cuda")
    off = flat[1:].view_as(state)
    off.copy_(state)
    assert torch.equal(delta_step(*args, off), want) and torch.equal(off, want_state)
    q, k, v, g, beta = args
    one = q[:, :1].expand(B, 2, Dk)
    assert torch.equal(delta_step(one, k, v, g, beta, state.clone()),
                       delta_step(one.contiguous(), k, v, g, beta, state.clone()))
    wide = torch.cat([g, beta], -1)
    assert torch.equal(delta_step(q, k, v, wide[:, :H], wide[:, H:], state.clone()), want)


@pytest.mark.gpu
def test_step_extremes(cuda_device):
    """Decays of zero and of one, a NaN in an idle stream, nothing at all, states past 2^31 values."""
    import torch
    from paper_1905_00689_gb300 import delta_step
    q, k, v, g, beta = delta.tensors((4,), 2, 1, 32, 16, "fp32", 5)
    g = torch.tensor([0.0, -float("inf"), -1e30, -0.5], device="cuda")[:, None].expand(4, 2).contiguous()
    v[3] = float("nan")
    slots = torch.tensor([2, 0, 1, -1], dtype=torch.int32, device="cuda")
    state = torch.randn(3, 2, 32, 16, device="cuda")
    after = state.clone()
    got = delta_step(q, k, v, g, beta, after, slots=slots)
    compare((q, k, torch.nan_to_num(v), g, beta), state, got, after, "fp32", slots.cpu().numpy())
    none = delta_step(q[:0], k[:0], v[:0], g[:0], beta[:0], state)
    assert none.shape == (0, 2, 16)
    rows = 2 ** 31 // (2 * 32 * 16) + 2
    pool = torch.empty(rows, 2, 32, 16, device="cuda")
    pool[-1] = state[0]
    far = torch.tensor([rows - 1], dtype=torch.int32, device="cuda")
    near = state[:1].clone()
    want = delta_step(q[:1], k[:1], v[:1], g[:1], beta[:1], near)
    assert torch.equal(delta_step(q[:1], k[:1], v[:1], g[:1], beta[:1], pool, slots=far), want)
    assert torch.equal(pool[-1], near[0])


@pytest.mark.gpu
def test_step_captured_and_on_a_stream(cuda_device):
    import torch
    from paper_1905_00689_gb300 import delta_step
    args = delta.tensors((3,), 4, 4, 64, 64, "bf16", 8)
    state, start = torch.zeros(3, 4, 64, 64, device="cuda"), torch.randn(3, 4, 64, 64, device="cuda")
    want_state = start.clone()
    want = [delta_step(*args, want_state) for _ in range(3)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    state.copy_(start)
    torch.cuda.synchronize()
    assert torch.equal(delta_step(*args, state, stream=side), want[0])
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o = delta_step(*args, state)
    state.copy_(start)
    for w in want:
        graph.replay()
        assert torch.equal(o, w)
    assert torch.equal(state, want_state)


def test_step_refusals(lib):
    P, msg = ctypes.c_void_p, ctypes.create_string_buffer(256)
    good = dict(dtype=1, q=P(256), k=P(256), v=P(256), g=P(256), beta=P(256), scale=1.0, state=P(256), n_slots=4, slots=None,
                reset=None, B=2, H=4, Hk=2, Dk=64, Dv=64, o=P(256), strides=None)
    strides = (ctypes.c_longlong * 10)(*[64] * 9, -1)
    for change in (dict(dtype=3), dict(dtype=-1), dict(q=None), dict(state=None), dict(o=None), dict(B=-1), dict(H=3),
                   dict(Hk=0), dict(H=0), dict(Dk=0), dict(Dk=129), dict(Dv=0), dict(n_slots=-1), dict(n_slots=1),
                   dict(q=P(257)), dict(g=P(258)), dict(state=P(258)), dict(strides=strides),
                   dict(B=2 ** 31 - 1, H=2 ** 20, Hk=1, slots=P(256))):
        args = {**good, **change}
        assert lib.lstm_approx_delta_step(*args.values(), None, msg, 256) == EINVAL, change
        assert msg.value


@pytest.mark.gpu
def test_step_refuses_tensors(cuda_device):
    import torch
    from paper_1905_00689_gb300 import delta_step
    args = q, k, v, g, beta = delta.tensors((3,), 4, 2, 64, 32, "bf16", 1)
    state = torch.zeros(5, 4, 64, 32, device="cuda")
    bad = [(q.float(), k, v, g, beta, state), (q, k[:2], v, g, beta, state), (q, k, v[:, :3], g, beta, state),
           (q, k, v, g.double(), beta, state), (q, k, v, g, beta.cpu(), state), (q, k, v, g, beta, state.bfloat16()),
           (q, k, v, g, beta, state[:, :, :, :16]), (q, k, v, g, beta, state[:2]), (q[0], k, v, g, beta, state),
           (q, k, v, g, beta, state.transpose(2, 3)), (q.mT.contiguous().mT, k, v, g, beta, state), (q, None, v, g, beta, state)]
    for case in bad:
        with pytest.raises((ValueError, RuntimeError)):
            delta_step(*case)
    for more in (dict(slots=torch.zeros(3, dtype=torch.int64, device="cuda")), dict(reset=torch.zeros(2, dtype=torch.bool, device="cuda")),
                 dict(o=torch.zeros(3, 4, 32, device="cuda")), dict(scale="x")):
        with pytest.raises((ValueError, RuntimeError)):
            delta_step(*args, state, **more)
    assert (state == 0).all()
