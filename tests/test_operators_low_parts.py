"""Which backward pass takes the low part of a 16-bit sum: that of the norm that made the sum, and no other."""
import numpy as np
import pytest

import operator_reference as ref
from test_operators_norm import TOL, make, weight

ROWS, D = 60, 520


def compare(got, dy, s, w, dtype):
    """The gradients of the norm of s (64 bits) with weight w, within the bounds of the other tests of them."""
    want, want_dw = ref.norm_backward(ref.f64(dy), s, ref.f64(w), None, 1e-5)
    r = 1 / np.sqrt((s ** 2).mean(1, keepdims=True) + 1e-5)
    wdy, xhat = np.abs(ref.f64(dy) * ref.f64(w)), np.abs(s) * r
    ref.check(got[0], want, r * (wdy + xhat * (wdy * xhat).mean(1, keepdims=True)), 2 * TOL, dtype, "dx")
    ref.check(got[1], want_dw, (np.abs(ref.f64(dy)) * xhat).sum(0), 2 * TOL, what="dw")


def first_norm(dtype):
    import torch
    from paper_1905_00689_gb300 import rms_norm
    x, res, dy, w = make(ROWS, D, dtype, 91), make(ROWS, D, dtype, 92, std=3.0), make(ROWS, D, dtype, 93), weight(D)
    rstd = torch.empty(ROWS, device="cuda")
    _, total = rms_norm(x, w, res, eps=1e-5, rstd=rstd)
    return total, rstd, ref.f64(x) + ref.f64(res), dy, w


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_two_norms_of_one_sum(cuda_device, dtype):
    """A final norm, or a second branch, reads the rounded sum: its gradients are at what it read, those of the norm
    that made the sum at the sum before its rounding, in either order."""
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward
    total, rstd, s, dy, w = first_norm(dtype)
    w2, rstd2 = weight(D, 4), torch.empty(ROWS, device="cuda")
    rms_norm(total, w2, eps=1e-5, rstd=rstd2)
    for _ in range(2):
        compare(rms_norm_backward(dy, total, w2, rstd2), dy, ref.f64(total), w2, dtype)
        compare(rms_norm_backward(dy, total, w, rstd), dy, s, w, dtype)
    rms_norm(total[:], w2, eps=1e-5, rstd=rstd2)  # a view of it
    compare(rms_norm_backward(dy, total, w2, rstd2), dy, ref.f64(total), w2, dtype)
    rms_norm(total, w2, eps=1e-5, rstd=rstd)  # over the first one's rstd
    compare(rms_norm_backward(dy, total, w2, rstd), dy, ref.f64(total), w2, dtype)


@pytest.mark.gpu
def test_low_part_goes_with_its_rstd(cuda_device):
    """Another view of the same rstd counts as it; a copy, or one that has been written to, does not, and gives the
    bits of a call without the low part."""
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward
    total, rstd, s, dy, w = first_norm("bf16")
    want, plain = rms_norm_backward(dy, total, w, rstd), rms_norm_backward(dy, total.clone(), w, rstd)
    assert not torch.equal(want[1], plain[1])
    same = lambda a, b: all(torch.equal(u, v) for u, v in zip(a, b))  # noqa: E731
    assert same(rms_norm_backward(dy, total, w, rstd.view(6, 10).view(ROWS)), want)
    assert same(rms_norm_backward(dy, total, w, rstd.clone()), plain)
    assert same(rms_norm_backward(dy, total, w, rstd), want)
    rstd.add_(0.0)
    assert same(rms_norm_backward(dy, total, w, rstd), plain)
    # an rstd of another place in the same storage
    both = torch.empty(2, ROWS, device="cuda")
    x, res = make(ROWS, D, "bf16", 91), make(ROWS, D, "bf16", 92, std=3.0)
    _, total = rms_norm(x, w, res, eps=1e-5, rstd=both[0])
    both.data[1] = both.data[0]
    assert same(rms_norm_backward(dy, total, w, both[0]), want) and same(rms_norm_backward(dy, total, w, both[1]), plain)


@pytest.mark.gpu
def test_low_part_of_another_shape_or_behind_a_change(cuda_device):
    """A sum_low of another shape is left alone; a change of the sum that torch does not see moves the gradients by no
    more than the sum's rounding (half a unit in the last place of every value)."""
    import torch
    from paper_1905_00689_gb300 import rms_norm_backward
    total, rstd, _, dy, w = first_norm("bf16")
    plain = rms_norm_backward(dy, total.clone(), w, rstd)
    total.sum_low = total.sum_low[:32]
    assert all(torch.equal(a, b) for a, b in zip(rms_norm_backward(dy, total, w, rstd), plain))
    total, rstd, _, dy, w = first_norm("bf16")
    x = make(ROWS, D, "bf16", 94)
    total.data.copy_(x)
    got, want = rms_norm_backward(dy, total, w, rstd)[1].double(), rms_norm_backward(dy, x, w, rstd)[1].double()
    bound = (dy.double().abs() * x.double().abs() * rstd.double()[:, None]).sum(0) * 2.0 ** -8
    assert not torch.equal(got, want) and bool(((got - want).abs() <= 1.01 * bound).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_low_part_kept_by_the_caller(cuda_device, dtype):
    """Through save_for_backward the sum comes back as another object, without its attribute: the low part handed over
    by itself gives the same gradients.  It can be declined, and refused tensors are refused."""
    import torch
    from paper_1905_00689_gb300 import rms_norm, rms_norm_backward, rms_norm_quant
    x, res, dy, w = make(ROWS, D, dtype, 91), make(ROWS, D, dtype, 92, std=3.0), make(ROWS, D, dtype, 93), weight(D)

    class Norm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, res, w):
            rstd, low = torch.empty(x.shape[:-1], device="cuda"), torch.empty_like(x, dtype=torch.int16)
            y, total = rms_norm(x, w, res, eps=1e-5, rstd=rstd, sum_low=low)
            ctx.save_for_backward(total, w, rstd, low)
            return y, total

        @staticmethod
        def backward(ctx, dy, dtotal):
            total, w, rstd, low = ctx.saved_tensors
            dx, dw = rms_norm_backward(dy, total, w, rstd, dtotal, sum_low=low)
            return dx, dx, dw
    for t in (x, res, w):
        t.requires_grad_()
    y, total = Norm.apply(x, res, w)
    y.backward(dy)
    s = ref.f64(x) + ref.f64(res)
    compare((x.grad, w.grad), dy, s, w, dtype)
    assert torch.equal(x.grad, res.grad)
    x, res, w = x.detach(), res.detach(), w.detach()
    rstd, low = torch.empty(ROWS, device="cuda"), torch.full((ROWS, D), 77, dtype=torch.int16, device="cuda")
    _, total = rms_norm(x, w, res, eps=1e-5, rstd=rstd, sum_low=low)
    assert total.sum_low is low
    want = rms_norm_backward(dy, total, w, rstd)
    plain = rms_norm_backward(dy, total.clone(), w, rstd)
    same = lambda a, b: all(torch.equal(u, v) for u, v in zip(a, b))  # noqa: E731
    assert not same(want, plain)
    assert same(rms_norm_backward(dy, total.clone(), w, rstd, sum_low=low), want)
    assert same(rms_norm_backward(dy, total, w, rstd, sum_low=False), plain)
    _, bare = rms_norm(x, w, res, eps=1e-5, rstd=rstd, sum_low=False)
    assert not hasattr(bare, "sum_low") and torch.equal(bare, total)
    _, bare = rms_norm(x, w, res, eps=1e-5, sum_low=low.zero_())  # no rstd: the caller's alone
    assert not hasattr(bare, "sum_low") and same(rms_norm_backward(dy, bare, w, rstd, sum_low=low), want)
    for call in (lambda: rms_norm(x, w, res, rstd=rstd, sum_low=low.int()), lambda: rms_norm(x, w, res, rstd=rstd, sum_low=low[:3]),
                 lambda: rms_norm(x, w, sum_low=low), lambda: rms_norm(x.float(), w, res.float(), rstd=rstd, sum_low=low),
                 lambda: rms_norm(x, w, res, rstd=rstd, sum_low=True),
                 lambda: rms_norm_backward(dy, total, w, rstd, sum_low=low.t()),
                 lambda: rms_norm_backward(dy.float(), total.float(), w, rstd, sum_low=low)):
        with pytest.raises(ValueError):
            call()
    assert not hasattr(rms_norm_quant(x, w, res, rstd=rstd)[2], "sum_low")
