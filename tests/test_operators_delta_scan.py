"""The gated delta rule over a sequence and its gradients."""
import ctypes

import numpy as np
import pytest

import delta_reference as delta
import operator_reference as ref

EINVAL = 1
# Products are sums of at most 128 terms, 8 to an addition of the MMA, whose sum is cut to 24 bits: 16 x 2^-23, and 2^-21 of a
# factor is left out: 2^-18 of the sum of magnitudes, which by Cauchy and Schwarz is at most the operands' lengths.  The output
# of a chunk is four such products deep (K S, Tm X, the update, Q S), the gradients six, each of operands no longer than the
# largest row or column of the result's kind; what one chunk leaves in the state has decayed by e^-11 (64 times an average g
# of -0.175) behind the next.
TOL = 6 * 2.0 ** -18
SIZES = [(1, 1, 1, 1, 1, 1), (1, 3, 2, 1, 64, 16), (2, 1, 1, 1, 16, 33), (63, 2, 3, 3, 128, 31), (64, 1, 2, 2, 64, 64),
         (65, 2, 4, 2, 100, 34), (130, 1, 6, 2, 48, 80), (200, 2, 2, 1, 65, 17), (321, 1, 1, 1, 128, 128)]


def lengths_and_resets(T, B, seed, share=0.03):
    import torch
    rng = np.random.default_rng(seed)
    lengths = rng.integers(-1, T + 2, B)
    lengths[rng.integers(B)] = T
    reset = rng.random((T, B)) < share
    reset[T // 2, 0] = True
    return (torch.tensor(lengths, dtype=torch.int32, device="cuda"), torch.tensor(reset, device="cuda"))


def on_host(args, more):
    return [ref.f64(t) for t in args], {k: (ref.f64(v) if k in ("h0", "dh_last") and v is not None else v.cpu().numpy() if hasattr(v, "cpu") else v)
                                        for k, v in more.items()}


def columns(S):
    return float(np.sqrt((S ** 2).sum(-2)).max()) if S.size else 0.0


def compare_forward(args, got, dtype, **more):
    vals, more = on_host(args, more)
    o, last = delta.scan(*vals, **more)
    kept = []
    delta.scan(*vals, **more, kept=kept)
    top = max(columns(kept[0]), columns(last), float(np.abs(vals[2]).max(initial=0.0)))
    scale = more.get("scale") or vals[0].shape[-1] ** -0.5
    ref.check(got[0], o, scale * top, TOL, dtype, "o")
    ref.check(got[1], last, top, TOL, what="h_last")


def compare_backward(do, args, got, dtype, **more):
    """Each gradient is a sum of products of rows or columns of the following, by Cauchy and Schwarz no larger than their
    lengths' products, whatever cancels: G, of the state's gradient (the terms scale q do and what comes from behind);
    S, of the state; V, of v and what is taken off it (k has length 1 at most); do itself."""
    vals, more = on_host(args, more)
    want = delta.scan_backward(ref.f64(do), *vals, **more)

    def rows(x):
        return float(np.sqrt((x ** 2).sum(-1)).max()) if x.size else 0.0
    kept = []
    h0 = {k: v for k, v in more.items() if k != "dh_last"}
    delta.scan(*vals, **h0, kept=kept)
    scale = more.get("scale") or vals[0].shape[-1] ** -0.5
    at_end = more.get("dh_last")
    ends = [want[5]] + ([at_end] if at_end is not None else [])
    G = max([scale * rows(ref.f64(do)), rows(want[2])] + [max(rows(x), columns(x)) for x in ends])
    S = max(rows(kept[0]), columns(kept[0]))
    V = rows(vals[2]) + columns(kept[0])
    shared = vals[2].shape[2] // vals[0].shape[2]
    q_top, k_top = shared * scale * rows(ref.f64(do)) * (S + V), shared * G * (V + S)
    for name, a, b, top in zip(("dq", "dk", "dv"), got, want, (q_top, k_top, G)):
        ref.check(a, b, top + 1e-30, TOL, dtype, name)
    ref.check(got[4], want[4], G * (V + S) + 1e-30, TOL, what="dbeta")
    ref.check(got[3], want[3], 64 * (q_top + k_top) + 1e-30, TOL, what="dg")  # up to 64 of q . dq and k . dk
    ref.check(got[5], want[5], G + 1e-30, TOL, what="dh0")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("T,B,H,Hk,Dk,Dv", SIZES)
def test_forward(cuda_device, T, B, H, Hk, Dk, Dv, dtype):
    import torch
    from paper_1905_00689_gb300 import delta_scan
    args = delta.tensors((T, B), H, Hk, Dk, Dv, dtype, T)
    compare_forward(args, delta_scan(*args), dtype)
    h0 = torch.randn(B, H, Dk, Dv, device="cuda")
    lengths, reset = lengths_and_resets(T, B, T)
    o = torch.full_like(args[2], float("nan"))
    more = dict(h0=h0, lengths=lengths, reset=reset, scale=0.3)
    got = delta_scan(*args, **more, o=o)
    assert got[0] is o
    compare_forward(args, got, dtype, **more)
    again = delta_scan(*args, **{**more, "reset": reset.to(torch.uint8)})
    assert torch.equal(got[0], again[0]) and torch.equal(got[1], again[1])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("T,B,H,Hk,Dk,Dv", SIZES)
def test_backward(cuda_device, T, B, H, Hk, Dk, Dv, dtype):
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    args = delta.tensors((T, B), H, Hk, Dk, Dv, dtype, 50 + T)
    do = torch.randn(T, B, H, Dv, device="cuda").to(args[0].dtype)
    states = delta_scan_states(args[0], args[2])
    assert states.shape == (-(-T // 64), B, H, Dk + 64, Dv)
    delta_scan(*args, states=states)
    compare_backward(do, args, delta_scan_backward(do, *args, states), dtype)
    lengths, reset = lengths_and_resets(T, B, T + 1)
    h0, dh_last = (torch.randn(B, H, Dk, Dv, device="cuda") for _ in range(2))
    more = dict(lengths=lengths, reset=reset, scale=0.3)
    states.fill_(float("nan"))  # (what no stream reaches is not read)
    delta_scan(*args, h0, **more, states=states)
    got = delta_scan_backward(do, *args, states, dh_last, **more)
    compare_backward(do, args, got, dtype, h0=h0, dh_last=dh_last, **more)
    again = delta_scan_backward(do, *args, states, dh_last, **more)
    assert all(torch.equal(a, b) for a, b in zip(got, again))


@pytest.mark.gpu
@pytest.mark.parametrize("which", ["q", "k", "v", "g", "beta", "h0"])
def test_gradients_against_differences(cuda_device, which):
    """Central differences of the 64-bit forward formula along a random direction: their own error is of the third order of
    the step (1e-4), under 1e-6 of the slope here."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    T, B, H, Hk, Dk, Dv = 70, 2, 4, 2, 24, 12
    args = delta.tensors((T, B), H, Hk, Dk, Dv, "fp32", 9)
    h0, dh_last = (torch.randn(B, H, Dk, Dv, device="cuda") for _ in range(2))
    lengths, reset = lengths_and_resets(T, B, 4, 0.02)
    do = torch.randn(T, B, H, Dv, device="cuda")
    states = delta_scan_states(args[0], args[2])
    delta_scan(*args, h0, lengths=lengths, reset=reset, states=states)
    grads = dict(zip(("q", "k", "v", "g", "beta", "h0"), delta_scan_backward(do, *args, states, dh_last, lengths=lengths, reset=reset)))
    vals = dict(zip(("q", "k", "v", "g", "beta"), (ref.f64(t) for t in args)))
    vals["h0"] = ref.f64(h0)
    way = np.random.default_rng(1).standard_normal(vals[which].shape)
    if which == "g":
        way *= vals["g"] < -1e-3  # (stays below zero)

    def loss(step):
        at = {**vals, which: vals[which] + step * way}
        o, last = delta.scan(at["q"], at["k"], at["v"], at["g"], at["beta"], at["h0"], None, lengths.cpu().numpy(), reset.cpu().numpy())
        return (o * ref.f64(do)).sum() + (last * ref.f64(dh_last)).sum()
    slope = (loss(1e-4) - loss(-1e-4)) / 2e-4
    got = (ref.f64(grads[which]) * way).sum()
    size = np.sqrt((ref.f64(grads[which]) ** 2 * way ** 2).sum())
    assert abs(got - slope) <= 1e-4 * size + 1e-5 * abs(slope)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("Dk,Dv", [(64, 32), (33, 17), (128, 50)])
def test_layouts(cuda_device, dtype, Dk, Dv):
    """Slices of one projection's output, batch-major and broadcast tensors, any address: the bits of the contiguous call."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    T, B, H, Hk = 90, 3, 4, 2
    fused = delta.tensors((T, B), H, Hk, Dk, Dv, dtype, 7, fused=True)
    plain = [t.contiguous() for t in fused]
    do = torch.randn(T, B, H, Dv, device="cuda").to(plain[0].dtype)
    states = delta_scan_states(plain[0], plain[2])
    want = delta_scan(*plain, states=states)
    grads = delta_scan_backward(do, *plain, states)
    major = [t.transpose(0, 1).contiguous().transpose(0, 1) for t in plain]
    flat = [torch.zeros(t.numel() + 1, dtype=t.dtype, device="cuda")[1:].view(t.shape).copy_(t) for t in plain]
    for q, k, v, g, beta in (fused, major, flat):
        o = torch.full((B, H, T, Dv), float("nan"), dtype=v.dtype, device="cuda").permute(2, 0, 1, 3)
        other = torch.empty_like(states)
        got = delta_scan(q, k, v, g, beta, o=o, states=other)
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(other[0], states[0]) and torch.equal(other[1, :, :, :Dk + 26], states[1, :, :, :Dk + 26])
        dz = torch.full((T, B, 2 * Hk * Dk + H * Dv), float("nan"), dtype=v.dtype, device="cuda")
        dgates = torch.full((T, B, 2 * H), float("nan"), device="cuda")
        dq, dk, dv = dz.split((Hk * Dk, Hk * Dk, H * Dv), -1)
        out = delta_scan_backward(do, q, k, v, g, beta, states, dq=dq.unflatten(-1, (Hk, Dk)), dk=dk.unflatten(-1, (Hk, Dk)),
                                  dv=dv.unflatten(-1, (H, Dv)), dg=dgates[..., :H], dbeta=dgates[..., H:])
        assert all(torch.equal(a, b) for a, b in zip(grads, out))
        assert torch.isfinite(dz).all() and torch.isfinite(dgates).all()
    q, k, v, g, beta = plain
    one = (q[:, :1].expand(T, B, Hk, Dk), k[:, :, :1].expand(T, B, Hk, Dk), v, g, beta[:1].expand(T, B, H))
    full = [t.contiguous() for t in one]
    assert torch.equal(delta_scan(*one, states=other)[0], delta_scan(*full)[0])
    assert all(torch.equal(a, b) for a, b in zip(delta_scan_backward(do, *one, other), delta_scan_backward(do, *full, other)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_masked_places_hold_anything(cuda_device, dtype):
    """NaN and infinities past a stream's length, in documents before a reset and in the state before one reach nothing,
    forward or back."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    T, B, H, Hk, Dk, Dv = 150, 3, 2, 1, 64, 32
    args = delta.tensors((T, B), H, Hk, Dk, Dv, dtype, 21)
    do = torch.randn(T, B, H, Dv, device="cuda").to(args[0].dtype)
    lengths = torch.tensor([150, 77, 0], dtype=torch.int32, device="cuda")
    reset = torch.zeros(T, B, dtype=torch.bool, device="cuda")
    for t, b in ((0, 0), (30, 0), (45, 0), (64, 0), (127, 0), (70, 1)):
        reset[t, b] = True
    h0, dh_last = (torch.randn(B, H, Dk, Dv, device="cuda") for _ in range(2))

    def run(args, do, h0):
        states = delta_scan_states(args[0], args[2])
        o, last = delta_scan(*args, h0, lengths=lengths, reset=reset, states=states)
        return (o, last) + tuple(delta_scan_backward(do, *args, states, dh_last, lengths=lengths, reset=reset))
    want = run(args, do, h0)
    for value in (float("nan"), float("inf")):
        dirty, dirty_do, dirty_h0 = [t.clone() for t in args], do.clone(), h0.clone()
        for t in dirty + [dirty_do]:
            t[77:, 1] = value
            t[:, 2] = value
            t[30:45, 0] = value   # one document
            t[100:127, 0] = value  # the rest of another, which ends inside a chunk
        dirty_h0[0] = value
        got = run(dirty, dirty_do, dirty_h0)
        clean = torch.ones(T, dtype=torch.bool, device="cuda")
        clean[30:45] = False
        clean[64:127] = False  # (what comes before the bad values in their own document is not promised)
        for a, b in zip(got[:1] + got[2:7], want[:1] + want[2:7]):
            assert torch.equal(a[clean, 0], b[clean, 0]) and torch.equal(a[:, 1:], b[:, 1:])
        assert torch.equal(got[1], want[1]) and torch.equal(got[7], want[7])


@pytest.mark.gpu
def test_extreme_decays_and_steps(cuda_device):
    """No decay at all, decays of zero, far apart ones in one chunk, steps of 0, 1 and 2, keys of length zero."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    T, B, H, Dk, Dv = 140, 4, 1, 16, 8
    q, k, v, g, beta = delta.tensors((T, B), H, H, Dk, Dv, "fp32", 3)
    g[:, 0] = 0.0
    g[:, 1] = torch.where(torch.arange(T, device="cuda") % 7 == 0, -float("inf"), -0.01)[:, None]
    g[:, 2] = torch.where(torch.arange(T, device="cuda") % 5 == 0, -150.0, -1e-3)[:, None]
    beta[:, 0], beta[::3, 1], beta[:, 3] = 1.0, 0.0, 2.0
    k[::4] = 0.0
    g[:, 3] = -0.05
    args = (q, k, v, g, beta)
    h0 = torch.randn(B, H, Dk, Dv, device="cuda")
    do = torch.randn(T, B, H, Dv, device="cuda")
    states = delta_scan_states(q, v)
    got = delta_scan(*args, h0, states=states)
    vals = [ref.f64(t) for t in args]
    vals[3] = np.maximum(vals[3], -200.0)
    o, last = delta.scan(*vals, ref.f64(h0))
    kept = []
    delta.scan(*vals, ref.f64(h0), kept=kept)
    # without decay or with steps of 2 (reflections) errors stay: those of all three chunks add up
    top = 3 * columns(kept[0])
    ref.check(got[0], o, Dk ** -0.5 * top, TOL, what="o")
    ref.check(got[1], last, top, TOL, what="h_last")
    grads = delta_scan_backward(do, *args, states)
    want = delta.scan_backward(ref.f64(do), *vals, ref.f64(h0))
    for name, a, b in zip(("dq", "dk", "dv", "dg", "dbeta", "dh0"), grads, want):
        if name == "dg":
            b = np.where(ref.f64(g) < -200.0, 0.0, b)
        tops = np.abs(b).max() * (64 if name in ("dg", "dbeta") else 8)
        ref.check(a, b, 3 * tops, TOL, what=name)


@pytest.mark.gpu
@pytest.mark.parametrize("T,B", [(0, 2), (5, 0), (0, 0)])
def test_nothing(cuda_device, T, B):
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    args = [torch.empty(T, B, *s, device="cuda") for s in ((1, 8), (1, 8), (2, 4), (2,), (2,))]
    h0 = torch.randn(B, 2, 8, 4, device="cuda")
    states = delta_scan_states(args[0], args[2])
    o, last = delta_scan(*args, h0, states=states)
    assert o.shape == (T, B, 2, 4) and torch.equal(last, h0)
    grads = delta_scan_backward(o, *args, states, h0)
    assert torch.equal(grads[5], h0) and grads[0].shape == (T, B, 1, 8) and grads[3].shape == (T, B, 2)


@pytest.mark.gpu
def test_far_values(cuda_device):
    """Offsets past 2^31 values."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    args = delta.tensors((3, 1), 1, 1, 64, 64, "bf16", 9)
    big = torch.empty((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda")
    far = []
    for i, t in enumerate(args[:3]):
        x = big.as_strided((3, 1, 1, 64), (1 << 30, 64, 64, 1), 64 * i)
        x.copy_(t)
        far.append(x)
    states, other = delta_scan_states(args[0], args[2]), delta_scan_states(args[0], args[2])
    assert torch.equal(delta_scan(*far, *args[3:], states=states)[0], delta_scan(*args, states=other)[0])
    for a, b in zip(delta_scan_backward(args[2], *far, *args[3:], states), delta_scan_backward(args[2], *args, other)):
        assert torch.equal(a, b)


@pytest.mark.gpu
def test_steps_go_on_where_the_sequence_ends(cuda_device):
    """A sequence in one call, in two calls and timestep by timestep: the same to the errors of either way."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_step
    T, B, H, Hk, Dk, Dv = 100, 2, 4, 2, 32, 24
    args = delta.tensors((T, B), H, Hk, Dk, Dv, "fp32", 15)
    o, last = delta_scan(*args)
    first, mid = delta_scan(*[t[:41] for t in args])
    rest, end = delta_scan(*[t[41:] for t in args], mid, h_last=mid)
    assert end is mid
    state = torch.zeros(B, H, Dk, Dv, device="cuda")
    steps = torch.stack([delta_step(*[x[t] for x in args], state) for t in range(T)])
    top = float(o.abs().max())
    assert float((torch.cat([first, rest]) - o).abs().max()) <= 2 * TOL * top * 6  # (o is 1 / sqrt(Dk) of the states' size)
    assert float((steps - o).abs().max()) <= 2 * TOL * top * 6
    assert float((state - last).abs().max()) <= 4 * TOL * float(last.abs().max())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_captured_streams_and_two_at_once(cuda_device, dtype):
    """Captured and replayed on new values; on another stream; two calls at once with workspaces of their own."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    T, B, H, Hk, Dk, Dv = 130, 2, 4, 2, 64, 48
    sets = [delta.tensors((T, B), H, Hk, Dk, Dv, dtype, s) for s in (1, 2)]
    dos = [torch.randn(T, B, H, Dv, device="cuda").to(sets[0][0].dtype) for _ in range(2)]

    def run(args, do, **more):
        states = delta_scan_states(args[0], args[2])
        return tuple(delta_scan(*args, states=states, **more)) + tuple(delta_scan_backward(do, *args, states, **more))
    want = [run(a, d) for a, d in zip(sets, dos)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(3):
        both = []
        for s, a, d in zip(streams, sets, dos):
            with torch.cuda.stream(s):
                both.append(run(a, d))
        torch.cuda.synchronize()
        for got, w in zip(both, want):
            assert all(torch.equal(x, y) for x, y in zip(got, w))
    states = delta_scan_states(sets[0][0], sets[0][2])
    o, last = delta_scan(*sets[0], states=states, stream=streams[0])
    grads = delta_scan_backward(dos[0], *sets[0], states, stream=streams[0])
    streams[0].synchronize()
    assert all(torch.equal(x, y) for x, y in zip((o, last, *grads), want[0]))
    held, do = [t.clone() for t in sets[0]], dos[0].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = run(held, do)
    for i in (1, 0):
        for a, b in zip(held + [do], list(sets[i]) + [dos[i]]):
            a.copy_(b)
        graph.replay()
        assert all(torch.equal(x, y) for x, y in zip(out, want[i]))


@pytest.mark.gpu
def test_many_heads_and_wide_values(cuda_device):
    """More blocks than run at once, with 32 columns each; a single wide head: against the same heads alone."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    for T, B, H, Hk, Dk, Dv in ((70, 40, 8, 4, 32, 40), (66, 2, 1, 1, 128, 1000)):
        args = delta.tensors((T, B), H, Hk, Dk, Dv, "bf16", 77)
        do = torch.randn(T, B, H, Dv, device="cuda").bfloat16()
        states = delta_scan_states(args[0], args[2])
        o, last = delta_scan(*args, states=states)
        grads = delta_scan_backward(do, *args, states)
        b = B - 1
        part = [t[:, b:b + 1] for t in args]
        compare_forward(part, (o[:, b:b + 1], last[b:b + 1]), "bf16")
        compare_backward(do[:, b:b + 1], part, [x[:, b:b + 1] for x in grads[:5]] + [grads[5][b:b + 1]], "bf16")


def test_refusals(lib):
    P, msg = ctypes.c_void_p, ctypes.create_string_buffer(256)
    sizes = dict(T=8, B=2, H=4, Hk=2, Dk=64, Dv=64)
    need = {back: lib.lstm_approx_delta_scan_workspace_bytes(1, *sizes.values(), back) for back in (0, 1)}
    assert 0 < need[0] < need[1]
    forward = dict(dtype=1, q=P(256), k=P(256), v=P(256), g=P(256), beta=P(256), scale=1.0, h0=None, lengths=None, reset=None,
                   **sizes, o=P(256), strides=None, h_last=P(256), states=None, workspace=P(256), bytes=need[0])
    backward = dict(dtype=1, d_o=P(256), dh_last=None, q=P(256), k=P(256), v=P(256), g=P(256), beta=P(256), scale=1.0, states=P(256),
                    lengths=None, reset=None, **sizes, dq=P(256), dk=P(256), dv=P(256), dg=P(256), dbeta=P(256), dh0=P(256),
                    strides=None, workspace=P(256), bytes=need[1])
    common = [dict(dtype=3), dict(q=None), dict(beta=None), dict(T=-1), dict(B=-1), dict(H=3), dict(H=0), dict(Hk=0), dict(Dk=0),
              dict(Dk=129), dict(Dv=0), dict(q=P(257)), dict(g=P(258)), dict(lengths=P(2)), dict(workspace=None),
              dict(workspace=P(264)), dict(bytes=1000), dict(T=2 ** 31 - 1, B=2 ** 31 - 1), dict(B=2 ** 30, Dv=64)]
    for call, good, more, n in ((lib.lstm_approx_delta_scan, forward, [dict(o=None), dict(h_last=None), dict(h0=P(2)), dict(states=P(2))], 16),
                                (lib.lstm_approx_delta_scan_backward, backward,
                                 [dict(d_o=None), dict(states=None), dict(dq=None), dict(dh0=None), dict(dg=P(2)), dict(dv=P(3)),
                                  dict(dh_last=P(2))], 29)):
        for change in common + more + [dict(strides=(ctypes.c_longlong * n)(*[64] * (n - 1), -1))]:
            args = {**good, **change}
            assert call(*args.values(), None, msg, 256) == EINVAL, change
            assert msg.value
    for bad in (dict(T=-1), dict(H=3), dict(Dk=129), dict(B=2 ** 31 - 1, T=2 ** 31 - 1)):
        assert lib.lstm_approx_delta_scan_workspace_bytes(1, *{**sizes, **bad}.values(), 1) == 0
    assert lib.lstm_approx_delta_scan_workspace_bytes(3, *sizes.values(), 1) == 0


@pytest.mark.gpu
def test_refuses_tensors(cuda_device):
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    q, k, v, g, beta = delta.tensors((10, 2), 4, 2, 32, 16, "bf16", 1)
    states = delta_scan_states(q, v)
    bad = [(q.float(), k, v, g, beta), (q, k[:9], v, g, beta), (q, k, v[:, :, :3], g, beta), (q, k, v, g.double(), beta),
           (q, k, v, g, beta[..., :3]), (q, k, v, g.cpu(), beta), (q[0], k, v, g, beta), (q, k, v.transpose(2, 3), g, beta),
           (q, None, v, g, beta), (q[..., :0], k[..., :0], v, g, beta)]
    for case in bad:
        with pytest.raises((ValueError, RuntimeError)):
            delta_scan(*case)
        with pytest.raises((ValueError, RuntimeError)):
            delta_scan_backward(v, *case, states)
    for more in (dict(h0=torch.zeros(2, 4, 16, 32, device="cuda")), dict(lengths=torch.zeros(2, dtype=torch.int64, device="cuda")),
                 dict(reset=torch.zeros(2, 10, dtype=torch.bool, device="cuda")), dict(o=torch.zeros(10, 2, 4, 16, device="cuda")),
                 dict(states=states[:, :1]), dict(workspace=torch.empty(100, dtype=torch.uint8, device="cuda")), dict(scale="x")):
        with pytest.raises((ValueError, RuntimeError)):
            delta_scan(q, k, v, g, beta, **more)
    with pytest.raises((ValueError, RuntimeError)):
        delta_scan_backward(v, q, k, v, g, beta, states[:, :1])
    wide = torch.zeros(4, 1, 1, 129, device="cuda")
    with pytest.raises((ValueError, RuntimeError)):
        delta_scan(wide, wide, wide, wide[..., 0], wide[..., 0])


@pytest.mark.gpu
def test_refuses_expanded_outputs(cuda_device):
    """Several places of such an output would be one; inputs may be expanded, and count as their copies do."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states, delta_step
    T, B, H, Hk, Dk, Dv = 70, 2, 4, 2, 32, 16
    q, k, v, g, beta = delta.tensors((T, B), H, Hk, Dk, Dv, "bf16", 1)
    states, do = delta_scan_states(q, v), torch.randn(T, B, H, Dv, device="cuda").bfloat16()

    def same(t):
        return t[:, :1].expand(t.shape)
    with pytest.raises(ValueError):
        delta_scan(q, k, v, g, beta, o=same(torch.empty_like(v)))
    with pytest.raises(ValueError):
        delta_step(q[0], k[0], v[0], g[0], beta[0], torch.zeros(B, H, Dk, Dv, device="cuda"), o=torch.empty_like(v[0])[:1].expand(v[0].shape))
    for name, like in (("dq", q), ("dk", k), ("dv", v), ("dg", g), ("dbeta", beta)):
        with pytest.raises(ValueError):
            delta_scan_backward(do, q, k, v, g, beta, states, **{name: same(torch.empty_like(like))})
    args = [same(t) for t in (q, k, v, g, beta)]
    got = delta_scan(*args, states=states)
    grads = delta_scan_backward(same(do), *args, states)
    args = [t.contiguous() for t in args]
    want = delta_scan(*args, states=states)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    assert all(torch.equal(a, b) for a, b in zip(grads, delta_scan_backward(same(do).contiguous(), *args, states)))


@pytest.mark.gpu
@pytest.mark.parametrize("T,B,H,Hk,Dk,Dv", [(130, 3, 4, 2, 64, 70), (0, 2, 2, 1, 16, 5)])
def test_gradient_of_the_first_state_over_that_of_the_last(cuda_device, T, B, H, Hk, Dk, Dv):
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states
    args = delta.tensors((T, B), H, Hk, Dk, Dv, "bf16", 5)
    states, do = delta_scan_states(args[0], args[2]), torch.randn(T, B, H, Dv, device="cuda").bfloat16()
    lengths = torch.tensor([T, 0, 70][:B], dtype=torch.int32, device="cuda")
    delta_scan(*args, states=states, lengths=lengths)
    held = torch.randn(B, H, Dk, Dv, device="cuda")
    want = delta_scan_backward(do, *args, states, held.clone(), lengths=lengths)
    got = delta_scan_backward(do, *args, states, held, lengths=lengths, dh0=held)
    assert got[5] is held and all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.gpu
def test_offsets_past_32_bits(cuda_device):
    """Timesteps that lie more than 2^31 values apart, read and written; a pool of more than 2^31 values."""
    import torch
    from paper_1905_00689_gb300 import delta_scan, delta_scan_backward, delta_scan_states, delta_step
    T, B, H, Hk, Dk, Dv = 3, 2, 2, 1, 16, 24
    args = delta.tensors((T, B), H, Hk, Dk, Dv, "bf16", 9)
    do = torch.randn(T, B, H, Dv, device="cuda").bfloat16()
    apart, states = 2 ** 30 + 64, delta_scan_states(args[0], args[2])
    room = torch.empty(2 * apart + 4096, dtype=torch.bfloat16, device="cuda")

    def far(like, at):  # places of their own within the first 4096 values of each timestep
        n = like[0].numel()
        return room[at:].as_strided(like.shape, (apart, *like[0].stride())), at + n
    at, moved = 0, []
    for t in args[:3]:
        view, at = far(t, at)
        moved.append(view.copy_(t))
    o, at = far(args[2], at)
    want = delta_scan(*args, states=states)
    got = delta_scan(*moved, *args[3:], o=o)
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    want = delta_scan_backward(do, *args, states)
    outs = {}
    for name, like in (("dq", args[0]), ("dk", args[1]), ("dv", args[2])):
        outs[name], at = far(like, at)
    got = delta_scan_backward(do, *moved, *args[3:], states, **outs)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    del room, moved, o, outs, got

    slots = 2 ** 31 // (64 * 64) + 3
    pool = torch.empty(slots, 1, 64, 64, device="cuda")
    q, k, v, g, beta = delta.tensors((2,), 1, 1, 64, 64, "bf16", 10)
    small = torch.randn(2, 1, 64, 64, device="cuda")
    pool[0], pool[slots - 1] = small[0], small[1]
    want = delta_step(q, k, v, g, beta, small)
    got = delta_step(q, k, v, g, beta, pool, slots=torch.tensor([0, slots - 1], dtype=torch.int32, device="cuda"))
    assert torch.equal(got, want) and torch.equal(pool[0], small[0]) and torch.equal(pool[slots - 1], small[1])
