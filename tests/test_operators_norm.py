"""The root-mean-square norm, its 8-bit output and its gradients."""
import ctypes

import numpy as np
import pytest

import operator_reference as ref

EINVAL = 1
SIZES = [(1, 1), (1, 8), (3, 7), (5, 64), (4, 256), (33, 1000), (2, 1531), (7, 2048), (3, 8200), (2, 16392), (2, 32768)]
# fp32 errors of y = s rstd w by element: s one rounding, rstd 2 ulp and half the sum's (its error over at most
# 8 VPT + 10 additions of one chain, 42 roundoffs), two products: under 32 roundoffs of |y|, plus 2 of the sum
TOL = 32 * ref.U32


def make(rows, D, dtype, seed, **more):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(rows, D, generator=gen, device="cuda") * more.get("std", 1.0)).to(ref.torch_dtype(dtype))


def weight(D, seed=3):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return 1.0 + 0.3 * torch.randn(D, generator=gen, device="cuda")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,D", SIZES)
def test_norm(cuda_device, rows, D, dtype):
    import torch
    from paper_1905_00689_gb300 import rms_norm
    x, res, w = make(rows, D, dtype, 1), make(rows, D, dtype, 2, std=3.0), weight(D)
    for residual in (None, res):
        rstd = torch.full((rows,), float("nan"), device="cuda")
        out = torch.full_like(x, float("nan"))
        y, total = rms_norm(x, w, residual, eps=1e-5, rstd=rstd, out=out)
        s, r, want = ref.norm(ref.f64(x), ref.f64(w), None if residual is None else ref.f64(residual), 1e-5)
        # |y| up to the error of s itself, one rounding of the two addends
        mag = np.abs(want)
        if residual is not None:
            mag = mag + (np.abs(ref.f64(x)) + np.abs(ref.f64(residual))) * r[:, None] * np.abs(ref.f64(w)) / 16
            ref.check(total, s, np.abs(s), 2 * ref.U32, dtype, "sum")
        else:
            assert total is None
        assert y is out
        ref.check(y, want, mag, TOL, dtype, "y")
        ref.check(rstd, r, r, TOL, what="rstd")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_norm_strides_and_in_place(cuda_device, dtype):
    """Slices of a wider tensor, aligned and not, broadcast rows, leading axes; the residual updated in place."""
    import torch
    from paper_1905_00689_gb300 import rms_norm
    w = weight(96)
    wide = make(12, 3 * 96 + 5, dtype, 5)
    for at in (0, 1, 8, 96, 101):
        x = wide[:, at:at + 96]
        y, _ = rms_norm(x, w)
        assert torch.equal(y, rms_norm(x.contiguous(), w)[0])
    row = wide[:1, :96].expand(12, 96)
    assert torch.equal(rms_norm(row, w)[0], rms_norm(row.contiguous(), w)[0])
    x3, r3 = make(12, 96, dtype, 6).reshape(3, 4, 96), make(12, 96, dtype, 7).reshape(3, 4, 96)
    y, total = rms_norm(x3, w, r3)
    held = r3.clone()
    y2, total2 = rms_norm(x3, w, held, residual_out=held)
    assert total2 is held and torch.equal(held, total) and torch.equal(y, y2) and y.shape == (3, 4, 96)
    time_major = x3.transpose(0, 1)  # rows at two strides
    with pytest.raises(ValueError, match="pitch"):
        rms_norm(time_major, w)
    assert torch.equal(rms_norm(x3[:, :1], w)[0][:, 0], rms_norm(x3[:, 0].contiguous(), w)[0])


@pytest.mark.gpu
def test_norm_far_rows(cuda_device):
    """Row offsets past 2^31 elements."""
    import torch
    from paper_1905_00689_gb300 import rms_norm
    big = torch.empty((1 << 31) + 4096, dtype=torch.bfloat16, device="cuda")
    x = big.as_strided((2, 64), (1 << 31, 1))
    x.copy_(make(2, 64, "bf16", 8))
    assert torch.equal(rms_norm(x, weight(64))[0], rms_norm(x.contiguous(), weight(64))[0])


@pytest.mark.gpu
def test_norm_special_values(cuda_device):
    """A row that is not finite stays by itself; a row of zeros; values whose squares are subnormal."""
    import torch
    from paper_1905_00689_gb300 import rms_norm
    x = make(5, 70, "fp32", 9)
    x[1, 3], x[2, 4], x[3] = float("nan"), float("inf"), 0.0
    x[4] *= 1e-21
    y, _ = rms_norm(x, weight(70), eps=1e-6)
    assert torch.isnan(y[1]).all() and torch.isnan(y[2, 4]) and (y[3] == 0).all()
    assert (y[2, :4] == 0).all() and torch.isfinite(y[[0, 4]]).all()
    ref.check(y[[0, 4]], ref.norm(ref.f64(x[[0, 4]]), ref.f64(weight(70)))[2], np.abs(ref.f64(y[[0, 4]])), TOL)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,D,group", [(1, 1, 32), (3, 70, 32), (5, 128, 128), (2, 1000, 64), (9, 1000, 256),
                                          (4, 2048, 128), (3, 1531, 2000), (2, 4096, 4096), (1, 17000, 128),
                                          (2, 24, 128)])
def test_norm_8bit(cuda_device, rows, D, group, dtype):
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_quant
    x, res, w = make(rows, D, dtype, 11), make(rows, D, dtype, 12), weight(D)
    q, scale, total = rms_norm_quant(x, w, res, eps=1e-5, group=group)
    assert q.dtype == torch.float8_e4m3fn and torch.equal(total, rms_norm(x, w, res, eps=1e-5)[1])
    _, _, y = ref.norm(ref.f64(x), ref.f64(w), ref.f64(res), 1e-5)
    # scale: the largest |y| of the group (whose error is y's, see TOL, and s's rounding) and one division
    G = -(-D // group)
    mag = np.pad(np.abs(y), ((0, 0), (0, G * group - D))).reshape(rows, G, group).max(2)
    ref.check(scale, mag / 448.0, mag / 448.0, 4 * TOL, what="scale")
    # q: within half a unit of its last place (3 bits of mantissa; smallest step 2^-9) of y / scale
    each = np.arange(D) // group
    want = y / ref.f64(scale)[:, each]
    step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(want), 2.0 ** -6))) - 3)
    assert (np.abs(ref.f64(q.float()) - want) <= step * 0.5001 + 448 * 4 * TOL).all()
    assert (q.float().abs().amax(1) == 448).all()


@pytest.mark.gpu
def test_norm_8bit_special_groups(cuda_device):
    """Groups of zeros take scale 1; one that holds NaN or infinity is not finite throughout, the others of its row
    only where the norm itself is; the smallest scale."""
    import torch
    from paper_1905_00689_gb300 import rms_norm_quant
    x = torch.ones(3, 96, device="cuda")
    x[0, 32:64] = 0.0
    w = torch.ones(96, device="cuda")
    w[95] = float("inf")
    x[1, :] = 0.0
    x[2, :] = 1e-30
    q, scale, _ = rms_norm_quant(x, w, eps=1e-6, group=32)
    assert scale[0, 1] == 1 and (q[0, 32:64].float() == 0).all()
    assert torch.isfinite(scale[0, :2]).all() and not torch.isfinite(scale[0, 2])
    assert torch.isnan((q[0].float() * scale[0].repeat_interleave(32))[64:]).all()
    assert (scale[1, :2] == 1).all()
    w[95] = 1.0
    w[:] = 1e-10
    q, scale, _ = rms_norm_quant(x, w, eps=1e-6, group=32)  # y = 1e-37: below 448 * 2^-126
    assert (scale[2] == 2.0 ** -126).all() and torch.isfinite(q.float()).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,D", SIZES + [(700, 96), (5000, 33), (1300, 520)])
def test_norm_backward(cuda_device, rows, D, dtype):
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward
    s, dy, dsum, w = (make(rows, D, dtype, 21), make(rows, D, dtype, 22), make(rows, D, dtype, 23), weight(D))
    rstd = torch.empty(rows, device="cuda")
    rms_norm(s, w, eps=1e-5, rstd=rstd)
    for extra in (None, dsum):
        dx, dw = rms_norm_backward(dy, s, w, rstd, extra)
        want, want_dw = ref.norm_backward(ref.f64(dy), ref.f64(s), ref.f64(w), None if extra is None else ref.f64(extra),
                                          1e-5)
        r = 1 / np.sqrt((ref.f64(s) ** 2).mean(1, keepdims=True) + 1e-5)
        wdy = np.abs(ref.f64(dy) * ref.f64(w))
        xhat = np.abs(ref.f64(s)) * r
        # each term with a few roundoffs of its own magnitude; the mean with those of its terms' magnitudes
        mag = r * (wdy + xhat * (wdy * xhat).mean(1, keepdims=True)) + (0 if extra is None else np.abs(ref.f64(extra)))
        ref.check(dx, want, mag, 2 * TOL, dtype, "dx")
        ref.check(dw, want_dw, (np.abs(ref.f64(dy)) * xhat).sum(0), 2 * TOL, what="dw")  # chains of 64 at most
        again = rms_norm_backward(dy, s, w, rstd, extra)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)
    inplace = dy.clone()
    assert rms_norm_backward(inplace, s, w, rstd, dsum, dx=inplace)[0] is inplace
    assert torch.equal(inplace, dx)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,at", [("fp32", 0), ("fp32", 1), ("bf16", 0), ("bf16", 1), ("fp16", 2)])
@pytest.mark.parametrize("rows,D", [(400, 2056), (330, 4104), (310, 6144), (310, 6160), (200, 8200), (160, 16392)])
def test_norm_backward_of_wide_rows(cuda_device, rows, D, dtype, at):
    """Widths on both sides of those where the columns are dealt out otherwise, several rows to a block of threads,
    out of wider tensors at every alignment; the gradients are those of contiguous copies to a few roundoffs."""
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward
    w = weight(D)
    dy, s, dsum = (make(rows, D + 8, dtype, 71 + k)[:, at:at + D] for k in range(3))
    rstd = torch.empty(rows, device="cuda")
    rms_norm(s, w, eps=1e-5, rstd=rstd)
    dx, dw = rms_norm_backward(dy, s, w, rstd, dsum)
    want, want_dw = ref.norm_backward(ref.f64(dy), ref.f64(s), ref.f64(w), ref.f64(dsum), 1e-5)
    r = 1 / np.sqrt((ref.f64(s) ** 2).mean(1, keepdims=True) + 1e-5)
    wdy, xhat = np.abs(ref.f64(dy) * ref.f64(w)), np.abs(ref.f64(s)) * r
    mag = r * (wdy + xhat * (wdy * xhat).mean(1, keepdims=True)) + np.abs(ref.f64(dsum))
    ref.check(dx, want, mag, 2 * TOL, dtype, "dx")
    ref.check(dw, want_dw, (np.abs(ref.f64(dy)) * xhat).sum(0), 2 * TOL, what="dw")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("rows,D", [(40, 64), (300, 1000), (65, 333), (20, 30)])
def test_norm_backward_of_a_16_bit_sum(cuda_device, rows, D, dtype):
    """The sum of a 16-bit forward pass brings along what its rounding took off: the gradients are those of x + residual, not
    of its rounding; a changed or copied sum falls back to what it holds."""
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward
    x, res, dy, w = (make(rows, D, dtype, 61), make(rows, D, dtype, 62, std=3.0), make(rows, D, dtype, 63), weight(D))
    rstd = torch.empty(rows, device="cuda")
    _, total = rms_norm(x, w, res, eps=1e-5, rstd=rstd)
    s = ref.f64(x) + ref.f64(res)
    assert total.sum_low.dtype == torch.int16 and total.sum_low.shape == total.shape

    def compare(got, s):
        want, want_dw = ref.norm_backward(ref.f64(dy), s, ref.f64(w), None, 1e-5)
        r = 1 / np.sqrt((s ** 2).mean(1, keepdims=True) + 1e-5)
        wdy, xhat = np.abs(ref.f64(dy) * ref.f64(w)), np.abs(s) * r
        ref.check(got[0], want, r * (wdy + xhat * (wdy * xhat).mean(1, keepdims=True)), 2 * TOL, dtype, "dx")
        ref.check(got[1], want_dw, (np.abs(ref.f64(dy)) * xhat).sum(0), 2 * TOL, what="dw")
    compare(rms_norm_backward(dy, total, w, rstd), s)
    copy = total.clone()
    rounded = torch.empty(rows, device="cuda")
    rms_norm(copy, w, eps=1e-5, rstd=rounded)
    compare(rms_norm_backward(dy, copy, w, rounded), ref.f64(copy))
    total.mul_(2.0)  # sum_low no longer belongs to it
    rms_norm(total, w, eps=1e-5, rstd=rounded)
    compare(rms_norm_backward(dy, total, w, rounded), ref.f64(total))
    assert not hasattr(rms_norm(x, w, res)[1], "sum_low")
    held = res.clone()
    rms_norm(x, w, held, residual_out=held, rstd=rstd)
    assert hasattr(held, "sum_low")
    rms_norm(x, w, held, residual_out=held)  # a later call on the same tensor takes it away
    assert not hasattr(held, "sum_low")


@pytest.mark.gpu
def test_norm_gradients_against_differences(cuda_device):
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward
    rows, D = 6, 45
    s, dy, w = make(rows, D, "fp32", 31), make(rows, D, "fp32", 32), weight(D)
    rstd = torch.empty(rows, device="cuda")
    rms_norm(s, w, rstd=rstd)
    dx, dw = rms_norm_backward(dy, s, w, rstd)
    rng = np.random.default_rng(0)
    S, W, DY = ref.f64(s), ref.f64(w), ref.f64(dy)
    for _ in range(8):
        vs, vw = rng.standard_normal(S.shape), rng.standard_normal(W.shape)
        e = 1e-5
        loss = lambda k: (ref.norm(S + k * e * vs, W + k * e * vw)[2] * DY).sum()  # noqa: E731
        slope = (loss(1) - loss(-1)) / (2 * e)  # error e^2 |third derivative| ~ 1e-8, and 1e-16 |loss| / e ~ 1e-9
        assert abs((ref.f64(dx) * vs).sum() + (ref.f64(dw) * vw).sum() - slope) < 1e-4 * np.sqrt(rows * D)


@pytest.mark.gpu
def test_norm_no_rows_and_other_stream(cuda_device):
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward, rms_norm_quant
    none, w = torch.empty(0, 64, device="cuda"), weight(64)
    assert rms_norm(none, w)[0].shape == (0, 64)
    assert rms_norm_quant(none, w)[1].shape == (0, 1)
    dx, dw = rms_norm_backward(none, none, w, torch.empty(0, device="cuda"))
    assert dx.shape == (0, 64) and (dw == 0).all()
    x = make(300, 640, "bf16", 41)
    want = rms_norm(x, weight(640))[0]
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    got, _ = rms_norm(x, weight(640), stream=s)
    s.synchronize()
    assert torch.equal(got, want)


def _args(**kw):
    a = dict(dtype=0, group=0, x=64, xp=8, res=None, rp=0, w=64, eps=1e-6, rows=2, D=8, out=64, scales=None, total=None,
             low=None, rstd=None)
    a.update(kw)
    return [a[k] for k in ("dtype", "group", "x", "xp", "res", "rp", "w", "eps", "rows", "D", "out", "scales", "total",
                           "low", "rstd")]


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(group=48), dict(group=-1), dict(x=None),
                                 dict(w=None), dict(out=None), dict(rows=-1), dict(D=0), dict(D=32769),
                                 dict(eps=-1.0), dict(eps=float("nan")), dict(scales=64), dict(group=8, scales=None),
                                 dict(x=66), dict(dtype=1, x=65), dict(w=66), dict(res=66), dict(xp=-1),
                                 dict(total=66), dict(low=64), dict(dtype=1, low=63),
                                 dict(dtype=1, group=128, scales=64, low=64), dict(rstd=2), dict(rows=1 << 31), dict(out=65)])
def test_norm_refusals(bad):
    """Refused before any device work (the pointers are never read)."""
    from paper_1905_00689_gb300 import load
    msg = ctypes.create_string_buffer(200)
    assert load().lstm_approx_rms_norm(*_args(**bad), None, msg, 200) == EINVAL and msg.value


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dy=None), dict(s=None), dict(w=None), dict(rstd=None),
                                 dict(dx=None), dict(rows=-1), dict(D=0), dict(ws=None), dict(ws=72), dict(nbytes=8),
                                 dict(dy=66), dict(dsum=65), dict(sp=-4), dict(low=64), dict(dtype=1, low=63)])
def test_norm_backward_refusals(bad):
    from paper_1905_00689_gb300 import load
    a = dict(dtype=0, dy=64, dyp=8, s=64, sp=8, low=None, w=64, rstd=64, dsum=None, dsp=0, rows=2, D=8, dx=64, dw=64, ws=64,
             nbytes=1 << 20)
    a.update(bad)
    msg = ctypes.create_string_buffer(200)
    assert load().lstm_approx_rms_norm_backward(*a.values(), None, msg, 200) == EINVAL and msg.value


@pytest.mark.gpu
def test_norm_wrapper_refusals(cuda_device):
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_quant
    x, w = make(4, 64, "bf16", 51), weight(64)
    for call in (lambda: rms_norm(x.cpu(), w), lambda: rms_norm(x, w.cpu()), lambda: rms_norm(x, w.half()),
                 lambda: rms_norm(x, w[:32]), lambda: rms_norm(x, w, x.float()), lambda: rms_norm(x, w, x[:2]),
                 lambda: rms_norm(x.t(), weight(4)), lambda: rms_norm(x.double(), w),
                 lambda: rms_norm(x, w, out=torch.empty(64, 4, device="cuda").t()),
                 lambda: rms_norm_quant(x, w, group=0)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_sum_low_is_not_stale(cuda_device):
    """A sum that an operator, a view or a copy overwrites no longer counts as the one its sum_low belongs to; what torch
    does not see moves the gradients by no more than the sum's rounding; a sum_low of another shape is left alone."""
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward
    rows, D = 64, 256
    x, res, dy, w = (make(rows, D, "bf16", 81), make(rows, D, "bf16", 82), make(rows, D, "bf16", 83), weight(D))
    rstd, rstd2 = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")

    def sum_of():
        return rms_norm(x, w, res, rstd=rstd)[1]

    def overwritten(total):
        clean = total.clone()
        rms_norm(clean, w, rstd=rstd2)
        return all(torch.equal(a, b) for a, b in zip(rms_norm_backward(dy, total, w, rstd2),
                                                     rms_norm_backward(dy, clean, w, rstd2)))
    for change in (lambda t: rms_norm(x, w, out=t), lambda t: t[3:5].zero_(), lambda t: t.view(-1).copy_(x.view(-1)),
                   lambda t: rms_norm_backward(dy, x, w, rstd, dx=t)):
        total = sum_of()
        change(total)
        assert overwritten(total)
    total = sum_of()
    assert not overwritten(total)
    other = sum_of()
    other.sum_low = other.sum_low[:32]
    assert overwritten(other)
    # behind torch's back: within half a unit in the last place of every value
    total = sum_of()
    total.data.copy_(x)
    rms_norm(x, w, rstd=rstd2)
    got, want = rms_norm_backward(dy, total, w, rstd2)[1].double(), rms_norm_backward(dy, x, w, rstd2)[1].double()
    bound = (dy.double().abs() * x.double().abs() * rstd2.double()[:, None]).sum(0) * 2.0 ** -8
    assert bool(((got - want).abs() <= 1.01 * bound).all())
