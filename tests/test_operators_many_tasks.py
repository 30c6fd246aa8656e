"""Sizes at which a block or a thread of the operators' kernels takes more than one piece of work: several tiles of the
scan one after another, four streams of a step, a second turn of row tiles of a 4-bit product; and two calls at once."""
import numpy as np
import pytest

import operator_reference as ref
from test_operators_scan import C, TOL, reference, tensors


def checked(x, r, i, decay, dy, h0, dl, dtype, **more):
    """Forward and backward against the 64-bit reference; the outputs."""
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states
    T, B, D = x.shape
    states = gated_scan_states(T, B, D)
    got = gated_scan(x, r, i, decay, h0, c=C, states=states, **more)
    grads = gated_scan_backward(dy, x, r, i, decay, states, dl, c=C, **more)
    vals, keep = reference(x, r, i, decay, h0=h0, dh_last=dl, **more)
    dh = keep.pop("dh_last")
    y, last, hs = ref.scan(*vals, C, **keep)
    top = np.abs(hs).max()
    ref.check(got[0], y, top, TOL, dtype, "y")
    ref.check(got[1], last, top, TOL, what="h_last")
    want = ref.scan_backward(ref.f64(dy), *vals, C, dh_last=dh, **keep)
    for g, w, name in zip(grads[:3], want, ("dx", "dr", "di")):
        ref.check(g, w, np.abs(w).max(), 4 * TOL, dtype, name)
    ref.check(grads[3], want[3], want[5], 4 * TOL, what="ddecay")
    ref.check(grads[4], want[4], np.abs(want[4]).max(), 4 * TOL, what="dh0")
    return got + grads + (states,)


def masks(T, B, share, seed):
    import torch
    rng = np.random.default_rng(seed)
    lengths = rng.integers(0, T + 1, B)
    lengths[0] = T
    return dict(lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                reset=torch.tensor(rng.random((T, B)) < share, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,D", [("fp32", 1104), ("fp32", 1101), ("bf16", 1104), ("bf16", 1102), ("bf16", 1101),
                                     ("fp16", 1104)])
def test_scan_of_many_tasks(cuda_device, dtype, D):
    """18 slabs of channels, 13 streams, 5 tiles of 128 timesteps (9 of 64): 1170 and 2106 tasks, three and more to
    each of at most 304 blocks, in numbers that divide neither the slabs nor the streams; by each kind of copy."""
    import torch
    T, B = 520, 13
    x, r, i, decay, dy, h0 = tensors(T, B, D, dtype, 400)
    dl = torch.randn(B, D, device="cuda")
    for more in ({}, masks(T, B, 0.01, 5)):
        first = checked(x, r, i, decay, dy, h0, dl, dtype, **more)
        if D != 1104:
            continue
        wide = [torch.zeros(T, B, D + 2, dtype=x.dtype, device="cuda")[..., 1:1 + D] for _ in range(4)]
        for to, v in zip(wide, (x, r, i, dy)):
            to.copy_(v)
        again = calls(*wide[:3], decay, wide[3], h0, dl, **more)  # value by value, or by 4 bytes
        assert all(torch.equal(a, b) for a, b in zip(first, again))


def calls(x, r, i, decay, dy, h0, dl, **more):
    from paper_1905_00689_gb300 import gated_scan, gated_scan_backward, gated_scan_states
    states = gated_scan_states(*x.shape)
    got = gated_scan(x, r, i, decay, h0, c=C, states=states, **more)
    return got + gated_scan_backward(dy, x, r, i, decay, states, dl, c=C, **more) + (states,)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,T", [("fp32", 10300), ("bf16", 20100)])
def test_scan_of_one_long_sequence(cuda_device, dtype, T):
    """Two slabs, one stream: more tiles than blocks, in groups of 16 that one block and another take in turn."""
    import torch
    x, r, i, decay, dy, h0 = tensors(T, 1, 66, dtype, 401)
    checked(x, r, i, decay, dy, h0, torch.randn(1, 66, device="cuda"), dtype, **masks(T, 1, 0.001, 6))


@pytest.mark.gpu
def test_two_scans_at_once(cuda_device):
    """On two streams, forward and backward, each of more blocks than the GPU holds beside the other's: the bits of one
    after the other."""
    import torch
    sets = []
    for seed, (T, B, D) in ((402, (1500, 4, 2048)), (403, (2100, 3, 1000))):
        x, r, i, decay, dy, h0 = tensors(T, B, D, "bf16", seed)
        sets.append((x, r, i, decay, dy, h0, torch.randn(B, D, device="cuda")))
    want = [calls(*s) for s in sets]
    streams = [torch.cuda.Stream() for _ in sets]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(4):
        for k, stream in enumerate(streams):
            with torch.cuda.stream(stream):
                got[k].append(calls(*sets[k]))
    torch.cuda.synchronize()
    for w, runs in zip(want, got):
        for g in runs:
            assert all(torch.equal(a, b) for a, b in zip(w, g))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,D", [(1301, 130), (1302, 131), (1000, 2048), (1303, 64), (5000, 3)])
def test_step_of_many_streams(cuda_device, dtype, B, D):
    """Four streams to a thread, with a rest of one to three, idle ones and resets among them."""
    import torch
    from paper_1905_00689_gb300 import gated_step
    x, r, i, decay, _, h0 = tensors(1, B, D, dtype, 404, fused=True)
    x, r, i = x[0], r[0], i[0]
    rng = np.random.default_rng(B)
    n = B + 77
    slots = torch.tensor(rng.permutation(n)[:B], dtype=torch.int32, device="cuda")
    slots[torch.tensor(rng.random(B) < 0.1, device="cuda")] = -3
    slots[B - 1], slots[4] = n, n + 5
    reset = torch.tensor(rng.random(B) < 0.2, device="cuda")
    pool = torch.randn(n, D, device="cuda")
    live = (slots >= 0) & (slots < n)
    pool[slots[live & reset].long()] = float("nan")
    before = pool.clone()
    y = gated_step(x, r, i, decay, pool, c=C, slots=slots, reset=reset)
    (X, R, I, DEC), _ = reference(x, r, i, decay)
    _, si, _, a, m = ref.gates(R, I, DEC, C)
    on, at = live.cpu().numpy(), slots.cpu().numpy()
    start = np.zeros((B, D))
    start[on] = ref.f64(before)[at[on]]
    start[reset.cpu().numpy()] = 0.0
    want = np.where(on[:, None], a * start + m * si * X, 0.0)
    top = max(np.abs(want).max(), np.abs(start).max())
    ref.check(y, want, top, TOL, dtype, "y")
    ref.check(pool[slots[live].long()], want[on], top, TOL, what="state")
    rest = torch.ones(n, dtype=torch.bool, device="cuda")
    rest[slots[live].long()] = False
    assert torch.equal(pool[rest], before[rest])
    # without a pool: stream b owns row b
    state = h0.clone()
    y = gated_step(x, r, i, decay, state, c=C)
    want = a * ref.f64(h0) + m * si * X
    ref.check(y, want, np.abs(want).max(), TOL, dtype, "y")
    ref.check(state, want, np.abs(want).max(), TOL, what="state")


@pytest.mark.gpu
@pytest.mark.parametrize("x_type", ["fp32", "bf16", "fp16", "8-bit"])
@pytest.mark.parametrize("M,N,K,group", [(1, 50001, 96, 32), (3, 40000, 200, 128), (16, 50000, 1024, 64),
                                         (7, 39001, 700, 32), (16, 10007, 8192, 128), (2, 10007, 32768, 64)])
def test_matvec_of_many_rows_of_w(cuda_device, x_type, M, N, K, group):
    """More row tiles to a block than it has warps (a vocabulary's rows, or few warps beside a long x), with x laid out
    by the block itself and before it.  Bounds: a group's sum is formed in group / 16 steps of a few roundoffs each, K /
    group sums follow one another at most, and up to 16 warps' parts, scales and parts of x 20."""
    import torch
    from paper_1905_00689_gb300 import rms_norm_quant, w4_matvec
    from test_operators_w4 import matrix, rows
    w = matrix(N, K, group, 405)
    out = torch.float32
    if x_type == "8-bit":
        x, scale, _ = rms_norm_quant(rows(M, K, "bf16", 406), torch.ones(K, device="cuda"), group=128)
        x64 = x.double() * scale.double().repeat_interleave(128, 1)[:, :K]
    else:
        x, scale = rows(M, K, x_type, 406), None
        x64 = x.double()
    y = w4_matvec(x, w, x_scale=scale, out_dtype=out)
    tol = (K / group + 4 * group / 16 + 36) * ref.U32
    for at in range(0, N, 4096):
        to = min(N, at + 4096)
        q = torch.stack([w.q[at:to] & 15, w.q[at:to] >> 4], 2).reshape(to - at, -1)[:, :K].double()
        each = torch.arange(K, device="cuda") // group
        dense = (q - w.zero[at:to].double()[:, each]) * w.scale[at:to].double()[:, each]
        err = (y[:, at:to].double() - x64 @ dense.t()).abs()
        assert bool((err <= tol * (x64.abs() @ dense.abs().t())).all()), float(err.max())
    assert torch.equal(y, w4_matvec(x, w, x_scale=scale, out_dtype=out))
