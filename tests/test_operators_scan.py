"""The gated linear recurrence: the scan over a sequence, its gradients, and the single step."""
import ctypes

import numpy as np
import pytest

import operator_reference as ref

EINVAL = 1
C = 8.0
A_MAX = 0.99
# fp32 errors of h relative to the largest |h|: every timestep rounds the state (under 3 roundoffs with the gates'
# product) and a_t itself (1), and what it adds decays with a_t <= A_MAX where the gate is open; the inputs' gates
# have under 16 roundoffs of their own, at most doubled where a gate's exponent is far from zero
TOL = (4 / (1 - A_MAX) / 4 + 32) * ref.U32  # sigma(r) >= 1/4 nearly everywhere makes the decays faster than A_MAX ** 0.25
TOL = max(TOL, 4 / (1 - A_MAX ** 0.25) * ref.U32)


def tensors(T, B, D, dtype, seed, fused=False, batch_major=False):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0):
        return (torch.randn(*shape, generator=gen, device="cuda") * std).to(ref.torch_dtype(dtype))
    if fused:
        z = normal(T, B, 3 * D)
        x, r, i = z[..., :D], z[..., D:2 * D], z[..., 2 * D:]
    elif batch_major:
        x, r, i = (normal(B, T, D).transpose(0, 1) for _ in range(3))
    else:
        x, r, i = normal(T, B, D), normal(T, B, D), normal(T, B, D)
    a = torch.rand(D, generator=gen, device="cuda") * (A_MAX - 0.6) + 0.6
    decay = torch.log(torch.expm1(-torch.log(a) / C))
    return x, r, i, decay, normal(T, B, D), torch.randn(B, D, generator=gen, device="cuda")


def reference(x, r, i, decay, **more):
    more = {k: (ref.f64(v) if k in ("h0", "dh_last") and v is not None else None if v is None else v.cpu().numpy())
            for k, v in more.items()}
    return [ref.f64(t) for t in (x, r, i, decay)], more


def compare_forward(args, got, dtype, **more):
    vals, more = reference(*args, **more)
    with np.errstate(invalid="ignore"):
        y, last, hs = ref.scan(*vals, C, **more)
    top = np.abs(hs).max() + 1e-30
    ref.check(got[0], y, top, TOL, dtype, "y")
    ref.check(got[1], last, top, TOL, what="h_last")


SIZES = [(1, 1, 1), (1, 3, 64), (2, 1, 65), (7, 2, 3), (63, 2, 7), (64, 1, 130), (65, 2, 64), (130, 3, 33), (700, 2, 96),
         (1500, 1, 66), (4200, 1, 8)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("T,B,D", SIZES)
def test_scan(cuda_device, T, B, D, dtype):
    import torch
    from paper_1905_00689_gb300 import gated_scan
    x, r, i, decay, _, h0 = tensors(T, B, D, dtype, 100 + T)
    compare_forward((x, r, i, decay), gated_scan(x, r, i, decay, c=C), dtype)
    rng = np.random.default_rng(T)
    lengths = torch.tensor(rng.integers(-1, T + 2, B), dtype=torch.int32, device="cuda")
    reset = torch.tensor(rng.random((T, B)) < 0.05, device="cuda")
    reset[0, 0] = True
    y = torch.full_like(x, float("nan"))
    got = gated_scan(x, r, i, decay, h0, c=C, lengths=lengths, reset=reset, y=y)
    assert got[0] is y
    compare_forward((x, r, i, decay), got, dtype, h0=h0, lengths=lengths, reset=reset)
    again = gated_scan(x, r, i, decay, h0, c=C, lengths=lengths, reset=reset.to(torch.uint8))
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("T,B,D", [(90, 3, 64), (70, 2, 33), (5, 4, 130)])
def test_scan_layouts(cuda_device, T, B, D, dtype):
    """Slices of one projection's output, batch-major tensors, unaligned and broadcast ones: the bits of the
    contiguous call."""
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states
    for kind in ({"fused": True}, {"batch_major": True}):
        x, r, i, decay, dy, h0 = tensors(T, B, D, dtype, 7, **kind)
        states = gated_scan_states(T, B, D)
        want = gated_scan(x.contiguous(), r.contiguous(), i.contiguous(), decay, h0)
        got = gated_scan(x, r, i, decay, h0, y=torch.empty(B, T, D, dtype=x.dtype, device="cuda").transpose(0, 1),
                         states=states)
        assert torch.equal(want[0], got[0]) and torch.equal(want[1], got[1])
        grads = gated_scan_backward(dy, x.contiguous(), r.contiguous(), i.contiguous(), decay, states)
        dz = torch.full((T, B, 3 * D), float("nan"), dtype=x.dtype, device="cuda")
        out = gated_scan_backward(dy, x, r, i, decay, states, dx=dz[..., :D], dr=dz[..., D:2 * D], di=dz[..., 2 * D:])
        for a, b in zip(grads, out):
            assert torch.equal(a, b)
        assert torch.isfinite(dz).all()
    flat = torch.zeros(T * B * D + 1, dtype=x.dtype, device="cuda")
    off = flat[1:].reshape(T, B, D)
    off.copy_(x)
    assert torch.equal(gated_scan(off, r, i, decay)[0], gated_scan(x, r, i, decay)[0])
    one = x[:, :1].expand(T, B, D)
    assert torch.equal(gated_scan(one, r, i, decay)[0], gated_scan(one.contiguous(), r, i, decay)[0])


@pytest.mark.gpu
def test_scan_far_timesteps(cuda_device):
    """Offsets past 2^31 elements."""
    import torch
    from paper_1905_00689_gb300 import gated_scan
    x, r, i, decay, _, _ = tensors(3, 1, 64, "bf16", 9)
    big = torch.empty((1 << 31) + 2048, dtype=torch.bfloat16, device="cuda")
    far = big.as_strided((3, 1, 64), (1 << 30, 64, 1))
    far.copy_(x)
    assert torch.equal(gated_scan(far, r, i, decay)[0], gated_scan(x, r, i, decay)[0])


@pytest.mark.gpu
def test_scan_masked_places_hold_anything(cuda_device):
    """NaN and infinities past a stream's length and in the state before a reset reach nothing, forward or back."""
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states
    T, B, D = 150, 4, 70
    x, r, i, decay, dy, h0 = tensors(T, B, D, "fp32", 10)
    lengths = torch.tensor([0, 40, 149, 400], dtype=torch.int32, device="cuda")
    reset = torch.zeros(T, B, dtype=torch.bool, device="cuda")
    reset[0, 1], reset[66, 2], reset[64, 3] = True, True, True
    clean, dirty = [t.clone() for t in (x, r, i, dy)], [x, r, i, dy]
    for b, n in enumerate((0, 40, 149, 150)):
        for k, t in enumerate(dirty):
            t[n:, b] = (float("nan"), float("inf"), float("-inf"), float("nan"))[k]
    h_dirty = h0.clone()
    h_dirty[1] = float("nan")  # reset at its first timestep
    more = dict(c=C, lengths=lengths, reset=reset)
    outs = []
    for (x, r, i, dy), h in ((clean, h0), (dirty, h_dirty)):
        states = gated_scan_states(T, B, D)
        y, last = gated_scan(x, r, i, decay, h, states=states, **more)
        outs.append((y, last) + gated_scan_backward(dy, x, r, i, decay, states, **more))
    for a, b in zip(*outs):
        assert torch.equal(a, b) and torch.isfinite(a).all()
    assert (outs[0][0][40:, 1] == 0).all() and torch.equal(outs[0][1][0], h0[0])
    # the state before a reset inside a sequence
    x, r, i, dy = clean
    x[30, 2] = float("inf")
    y, _ = gated_scan(x, r, i, decay, h0, **more)
    assert not torch.isfinite(y[40, 2]).all() and torch.isfinite(y[66:, 2]).all() and torch.equal(y[66:149, 2], outs[0][0][66:149, 2])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_scan_saturated_gates(cuda_device, dtype):
    """Gates far from zero on both sides and decays of every size: finite, and the reference's."""
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states
    T, B, D = 40, 1, 96
    x, r, i, decay, dy, h0 = tensors(T, B, D, dtype, 11)
    r[:, :, :16], r[:, :, 16:32], r[:, :, 32:48] = 60.0, -30.0, -200.0
    i[:, :, ::3], i[:, :, 1::3] = 90.0, -90.0
    decay[::5], decay[1::5] = 40.0, -60.0
    decay[2], decay[3] = -200.0, 1e4
    states = gated_scan_states(T, B, D)
    got = gated_scan(x, r, i, decay, h0, c=C, states=states)
    vals, _ = reference(x, r, i, decay)
    y, last, hs = ref.scan(*vals, C, h0=ref.f64(h0))
    # a state that nothing decays or feeds is kept to the last bit; below sigma(i) ~ 1e-38 the input gate is zero
    ref.check(got[0], y, np.abs(hs).max(), TOL, dtype, "y")
    grads = gated_scan_backward(dy, x, r, i, decay, states, c=C)
    want = ref.scan_backward(ref.f64(dy), *vals, C, h0=ref.f64(h0))
    for g, w, name in zip(grads[:3], want, ("dx", "dr", "di")):
        assert torch.isfinite(g).all()
        ref.check(g, w, np.abs(w).max(), 4 * TOL, dtype, name)
    assert torch.isfinite(grads[3]).all() and torch.isfinite(grads[4]).all()
    ref.check(grads[3], want[3], want[5].max(), 4 * TOL, what="ddecay")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("T,B,D", SIZES)
def test_scan_backward(cuda_device, T, B, D, dtype):
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states
    x, r, i, decay, dy, h0 = tensors(T, B, D, dtype, 200 + T)
    dh_last = torch.randn(B, D, device="cuda")
    rng = np.random.default_rng(T + 1)
    lengths = torch.tensor(rng.integers(-1, T + 2, B), dtype=torch.int32, device="cuda")
    reset = torch.tensor(rng.random((T, B)) < 0.03, device="cuda")
    for more in ({}, dict(lengths=lengths, reset=reset)):
        for h, dl in ((None, None), (h0, dh_last)):
            states = gated_scan_states(T, B, D)
            gated_scan(x, r, i, decay, h, c=C, states=states, **more)
            got = gated_scan_backward(dy, x, r, i, decay, states, dl, c=C, **more)
            vals, keep = reference(x, r, i, decay, h0=h, dh_last=dl, **more)
            dh = keep.pop("dh_last")
            want = ref.scan_backward(ref.f64(dy), *vals, C, dh_last=dh, **keep)
            for g, w, name in zip(got[:3], want, ("dx", "dr", "di")):
                # products of the two recurrences' values: both errors, relative to the largest
                ref.check(g, w, np.abs(w).max() + 1e-30, 4 * TOL, dtype, name)
            ref.check(got[3], want[3], want[5], 4 * TOL, what="ddecay")
            ref.check(got[4], want[4], np.abs(want[4]).max() + 1e-30, 4 * TOL, what="dh0")
            again = gated_scan_backward(dy, x, r, i, decay, states, dl, c=C, **more)
            assert all(torch.equal(a, b) for a, b in zip(got, again))


def test_reference_gradients_against_differences():
    """The formulas themselves, in 64 bits on the CPU."""
    rng = np.random.default_rng(5)
    T, B, D = 9, 3, 4
    x, r, i, dy = rng.standard_normal((4, T, B, D))
    decay, h0, dl = rng.standard_normal(D) - 3, rng.standard_normal((B, D)), rng.standard_normal((B, D))
    lengths, reset = np.array([9, 0, 5]), rng.random((T, B)) < 0.2
    args = [x, r, i, decay, h0]

    def loss(args):
        y, last, _ = ref.scan(*args[:4], C, args[4], lengths, reset)
        return (y * dy).sum() + (last * dl).sum()
    grads = ref.scan_backward(dy, *args[:4], C, h0, lengths, reset, dl)
    for k in range(5):
        v = rng.standard_normal(args[k].shape)
        e = 1e-6
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + e * v, args[k] - e * v
        slope = (loss(up) - loss(down)) / (2 * e)
        assert abs((grads[k] * v).sum() - slope) < 1e-7 * (1 + abs(slope))


@pytest.mark.gpu
def test_scan_gradients_against_differences(cuda_device):
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states
    T, B, D = 130, 2, 5
    x, r, i, decay, dy, h0 = tensors(T, B, D, "fp32", 12)
    dl = torch.randn(B, D, device="cuda")
    reset = torch.zeros(T, B, dtype=torch.bool, device="cuda")
    reset[70, 1] = True
    states = gated_scan_states(T, B, D)
    gated_scan(x, r, i, decay, h0, c=C, reset=reset, states=states)
    grads = [ref.f64(t) for t in gated_scan_backward(dy, x, r, i, decay, states, dl, c=C, reset=reset)]
    args = [ref.f64(t) for t in (x, r, i, decay, h0)]

    def loss(args):
        y, last, _ = ref.scan(*args[:4], C, args[4], None, reset.cpu().numpy())
        return (y * ref.f64(dy)).sum() + (last * ref.f64(dl)).sum()
    rng = np.random.default_rng(6)
    for k in range(5):
        v = rng.standard_normal(args[k].shape)
        up, down = list(args), list(args)
        up[k], down[k] = args[k] + 1e-6 * v, args[k] - 1e-6 * v
        slope = (loss(up) - loss(down)) / 2e-6
        size = np.sqrt((grads[k] ** 2).sum()) + 1
        assert abs((grads[k] * v).sum() - slope) < 1e-4 * size * np.sqrt(v.size)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,D", [(1, 1), (3, 64), (5, 33), (2, 600), (70, 130)])
def test_step(cuda_device, B, D, dtype):
    import torch
    from paper_1905_00689_gb300 import gated_step
    x, r, i, decay, _, h0 = tensors(1, B, D, dtype, 13, fused=True)
    x, r, i = x[0], r[0], i[0]
    state = h0.clone()
    y = gated_step(x, r, i, decay, state, c=C)
    vals, _ = reference(x, r, i, decay)
    want = ref.scan(*(v[None] for v in vals[:3]), vals[3], C, h0=ref.f64(h0))
    ref.check(y, want[0][0], np.abs(want[2]).max(), TOL, dtype, "y")
    ref.check(state, want[1], np.abs(want[2]).max(), TOL, what="state")
    # a pool: scattered slots, idle streams on both sides of the range, resets over states that are not finite
    n = B + 9
    pool = torch.randn(n, D, device="cuda")
    slots = torch.randperm(n, device="cuda")[:B].to(torch.int32)
    reset = torch.arange(B, device="cuda") % 3 == 1
    if B > 2:
        slots[0], slots[2] = -1, n
    for b in range(B):
        if reset[b]:
            pool[slots[b]] = float("nan")
    before = pool.clone()
    y = gated_step(x, r, i, decay, pool, c=C, slots=slots, reset=reset)
    untouched = torch.ones(n, dtype=torch.bool, device="cuda")
    for b in range(B):
        s = int(slots[b])
        if s < 0 or s >= n:
            assert (y[b] == 0).all()
            continue
        untouched[s] = False
        start = np.zeros((1, D)) if reset[b] else ref.f64(before[s:s + 1])
        w = ref.scan(*(v[None, b:b + 1] for v in vals[:3]), vals[3], C, h0=start)
        ref.check(y[b], w[0][0, 0], np.abs(w[2]).max(), TOL, dtype, "y")
        ref.check(pool[s], w[1][0], np.abs(w[2]).max(), TOL, what="state")
    assert torch.equal(pool[untouched], before[untouched])


@pytest.mark.gpu
def test_steps_are_the_scan(cuda_device):
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_step
    T, B, D = 70, 3, 66
    x, r, i, decay, _, h0 = tensors(T, B, D, "fp32", 14)
    y, last = gated_scan(x, r, i, decay, h0, c=C)
    state = h0.clone()
    for t in range(T):
        out = gated_step(x[t], r[t], i[t], decay, state, c=C)
        ref.check(out, ref.f64(y[t]), np.abs(ref.f64(y)).max(), TOL)
    ref.check(state, ref.f64(last), np.abs(ref.f64(y)).max(), TOL)


@pytest.mark.gpu
def test_scan_nothing_and_other_stream(cuda_device):
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states, gated_step
    x, r, i, decay, dy, h0 = tensors(4, 2, 66, "bf16", 15)
    none = x[:0]
    y, last = gated_scan(none, none, none, decay, h0)
    assert y.shape == (0, 2, 66) and torch.equal(last, h0)
    assert (gated_scan(none, none, none, decay)[1] == 0).all()
    grads = gated_scan_backward(none, none, none, none, decay, gated_scan_states(0, 2, 66), h0)
    assert (grads[3] == 0).all() and torch.equal(grads[4], h0)
    few = x[:, :0]
    assert gated_scan(few, few, few, decay)[1].shape == (0, 66)
    grads = gated_scan_backward(few, few, few, few, decay, gated_scan_states(4, 0, 66))
    assert (grads[3] == 0).all()
    assert gated_step(x[0, :0], r[0, :0], i[0, :0], decay, h0).shape == (0, 66)
    held = h0.clone()  # the last state over the first
    want = gated_scan(x, r, i, decay, h0)
    got = gated_scan(x, r, i, decay, held, h_last=held)
    assert torch.equal(want[0], got[0]) and torch.equal(want[1], held)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got = gated_scan(x, r, i, decay, h0, stream=s)
    s.synchronize()
    assert torch.equal(want[0], got[0])


@pytest.mark.gpu
def test_scan_in_a_graph(cuda_device):
    """Captured, then replayed on new inputs in the same buffers."""
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states
    x, r, i, decay, dy, h0 = tensors(200, 2, 64, "bf16", 16)

    def both():
        states = gated_scan_states(200, 2, 64)
        y, last = gated_scan(x, r, i, decay, h0, states=states)
        return (y, last) + gated_scan_backward(dy, x, r, i, decay, states)
    both()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for seed in (17, 18):
        for t, new in zip((x, r, i), tensors(200, 2, 64, "bf16", seed)):
            t.copy_(new)
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(held, both()):
            assert torch.equal(a, b)


FORWARD = dict(dtype=0, x=64, r=64, i=64, decay=64, c=8.0, h0=None, lengths=None, reset=None, T=2, B=2, D=8, y=64,
               strides=None, last=64, states=None, ws=64, nbytes=1 << 20)
BACKWARD = dict(dtype=0, dy=64, dl=None, x=64, r=64, i=64, decay=64, c=8.0, states=64, lengths=None, reset=None, T=2,
                B=2, D=8, dx=64, dr=64, di=64, strides=None, ddecay=64, dh0=64, ws=64, nbytes=1 << 20)
STEP = dict(dtype=0, x=64, xp=8, r=64, rp=8, i=64, ip=8, decay=64, c=8.0, state=64, n=2, slots=None, reset=None, B=2, D=8,
            y=64)
BAD = ([(FORWARD, "gated_scan", b) for b in (
            dict(dtype=3), dict(x=None), dict(r=None), dict(i=None), dict(decay=None), dict(y=None), dict(last=None),
            dict(T=-1), dict(B=-1), dict(D=0), dict(c=0.0), dict(c=float("nan")), dict(x=66), dict(dtype=1, y=65),
            dict(h0=66), dict(lengths=65), dict(states=66), dict(decay=2), dict(ws=None), dict(ws=72), dict(nbytes=16), dict(strides="negative"))]
       + [(BACKWARD, "gated_scan_backward", b) for b in (
            dict(dtype=-1), dict(dy=None), dict(states=None), dict(dx=None), dict(dr=None), dict(di=None),
            dict(ddecay=None), dict(dh0=None), dict(ws=None), dict(ws=72), dict(nbytes=16), dict(T=-1), dict(D=0),
            dict(dx=66), dict(dl=66), dict(strides="negative"))]
       + [(STEP, "gated_step", b) for b in (
            dict(dtype=3), dict(x=None), dict(r=None), dict(i=None), dict(decay=None), dict(state=None), dict(y=None),
            dict(n=1), dict(n=-1), dict(B=-1), dict(D=0), dict(c=-1.0), dict(xp=-1), dict(slots=65), dict(state=66))])


@pytest.mark.parametrize("args,name,bad", BAD)
def test_scan_refusals(args, name, bad):
    """Refused before any device work (the pointers are never read)."""
    from paper_1905_00689_gb300 import load
    a = dict(args, **bad)
    if a.get("strides") == "negative":
        a["strides"] = (ctypes.c_longlong * 14)(16, 8, 16, -8, *[16, 8] * 5)
    msg = ctypes.create_string_buffer(200)
    assert getattr(load(), "lstm_approx_" + name)(*a.values(), None, msg, 200) == EINVAL and msg.value


@pytest.mark.gpu
def test_scan_wrapper_refusals(cuda_device):
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states, gated_step
    x, r, i, decay, dy, h0 = tensors(70, 2, 64, "bf16", 19)
    states = gated_scan_states(70, 2, 64)
    for call in (lambda: gated_scan(x, r.float(), i, decay), lambda: gated_scan(x, r[:5], i, decay),
                 lambda: gated_scan(x[0], r[0], i[0], decay), lambda: gated_scan(x, r, i, decay.cpu()),
                 lambda: gated_scan(x, r, i, decay.half()), lambda: gated_scan(x, r, i, decay, h0[:1]),
                 lambda: gated_scan(x, r, i, decay, lengths=torch.ones(2, device="cuda", dtype=torch.int64)),
                 lambda: gated_scan(x, r, i, decay, reset=torch.zeros(70, 2, device="cuda")),
                 lambda: gated_scan(x, r, i, decay, states=states[:1]),
                 lambda: gated_scan(x.cpu(), r, i, decay),
                 lambda: gated_scan_backward(dy[:3], x, r, i, decay, states),
                 lambda: gated_scan_backward(dy, x, r, i, decay, states.half()),
                 lambda: gated_step(x[0], r[0], i[0], decay, h0[:, :32]),
                 lambda: gated_step(x[0], r[0], i[0], decay, h0.t().contiguous().t())):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
@pytest.mark.parametrize("axis", ["t", "b"])
def test_offsets_past_32_bits(cuda_device, axis):
    """Timesteps or streams 2^31 elements apart, forward and backward, and a state pool of more than 2^31 values."""
    import torch
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states, gated_step
    gen = torch.Generator(device="cuda").manual_seed(17)
    T, B, D = (2, 3, 64) if axis == "t" else (70, 2, 64)
    strides = (1 << 31, D, 1) if axis == "t" else (D, 1 << 31, 1)
    decay = torch.rand(D, generator=gen, device="cuda") - 5.0
    z = torch.randn(4, T, B, D, generator=gen, device="cuda").to(torch.bfloat16)
    far = [torch.empty((1 << 31) + 16 * T * B * D, dtype=torch.bfloat16, device="cuda").as_strided((T, B, D), strides, k)
           for k in (0, 0, 2, 1)]  # (three of the kinds of alignment)
    for to, values in zip(far, z):
        to.copy_(values)
    x, r, i, dy = far
    states = [gated_scan_states(T, B, D) for _ in range(2)]
    y = gated_scan(x, r, i, decay, states=states[0])
    want = gated_scan(z[0], z[1], z[2], decay, states=states[1])
    assert torch.equal(y[0], want[0]) and torch.equal(y[1], want[1]) and torch.equal(*states)
    out = torch.empty((1 << 31) + 16 * T * B * D, dtype=torch.bfloat16, device="cuda").as_strided((T, B, D), strides)
    got = gated_scan_backward(dy, x, r, i, decay, states[0], dx=out)
    want = gated_scan_backward(z[3], z[0], z[1], z[2], decay, states[1])
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del far, x, r, i, dy, out, to, got
    n = (1 << 31) // D + 3
    state = torch.zeros(n, D, device="cuda")
    slots = torch.tensor([n - 1, 0], device="cuda", dtype=torch.int32)
    h = torch.randn(2, D, generator=gen, device="cuda")
    state[slots.long()] = h
    y = gated_step(z[0, 0, :2], z[1, 0, :2], z[2, 0, :2], decay, state, slots=slots)
    assert torch.equal(y, gated_step(z[0, 0, :2], z[1, 0, :2], z[2, 0, :2], decay, h))
    assert torch.equal(state[slots.long()], h)
