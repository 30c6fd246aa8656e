"""Matrix-vector products with 4-bit weights, and their quantiser."""
import ctypes

import numpy as np
import pytest

import operator_reference as ref

EINVAL = 1
# fp32 error of a sum relative to the sum of its terms' magnitudes: no accumulator takes more than 128 terms or
# partial sums one after another, each with one rounding; scale and bias add 4
TOL = 132 * ref.U32


def matrix(N, K, group, seed, scale="fp16", zero=True, extra=0):
    """A random W4Weight whose q has `extra` further bytes per row and noise beyond column K."""
    import torch
    from paper_1905_00689_gb300 import W4Weight
    gen = torch.Generator(device="cuda").manual_seed(seed)
    G, pitch = -(-K // group), -(-K // 32) * 16
    q = torch.randint(0, 256, (N, pitch + extra), generator=gen, device="cuda", dtype=torch.uint8)
    s = (torch.rand(N, G, generator=gen, device="cuda") + 0.5).to(ref.torch_dtype(scale))
    z = torch.randint(0, 16, (N, G), generator=gen, device="cuda", dtype=torch.uint8) if zero else None
    return W4Weight(q, s, z, K, group)


def dense(w):
    return ref.w4_matrix(w.q.cpu().numpy(), ref.f64(w.scale), None if w.zero is None else w.zero.cpu().numpy(), w.K,
                         w.group)


def rows(M, K, dtype, seed, pad=0, fill=float("nan")):
    """[M][K] in a wider tensor whose further columns hold `fill`."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.full((M, K + pad), fill, device="cuda")
    x[:, :K] = torch.randn(M, K, generator=gen, device="cuda")
    return x.to(ref.torch_dtype(dtype))[:, :K]


def compare(y, x, W, dtype, bias=None):
    want, mag = x @ W.T, np.abs(x) @ np.abs(W).T
    if bias is not None:
        want, mag = want + bias, mag + np.abs(bias)
    ref.check(y, want, mag, TOL, dtype, "y")


SHAPES = [(1, 1, 1, 32), (1, 5, 33, 32), (2, 16, 64, 64), (3, 17, 100, 64), (1, 300, 257, 128), (4, 130, 1000, 32),
          (5, 63, 999, 128), (8, 129, 2048, 128), (9, 40, 512, 64), (16, 77, 1536, 128), (17, 70, 320, 32),
          (33, 48, 640, 128), (70, 20, 160, 64), (1, 4100, 96, 32), (2, 64, 8192, 64), (0, 9, 64, 32), (2, 0, 64, 32)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("M,N,K,group", SHAPES)
def test_matvec(cuda_device, M, N, K, group, dtype):
    import torch
    from paper_1905_00689_gb300 import w4_matvec
    w = matrix(N, K, group, 10 * N + K)
    x = rows(M, K, dtype, 3)
    y = w4_matvec(x, w)
    assert y.dtype == x.dtype and y.shape == (M, N)
    compare(y, ref.f64(x), dense(w), dtype)
    assert torch.equal(y, w4_matvec(x, w))


@pytest.mark.gpu
@pytest.mark.parametrize("scale", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("zero", [True, False])
@pytest.mark.parametrize("dtype,out", [("bf16", "fp32"), ("fp32", "fp16"), ("fp16", "bf16"), ("bf16", "bf16")])
def test_matvec_types(cuda_device, dtype, out, scale, zero):
    import torch
    from paper_1905_00689_gb300 import w4_matvec
    for M, N, K, group in ((1, 90, 700, 64), (6, 33, 450, 128)):
        w, x = matrix(N, K, group, 4, scale, zero, extra=16), rows(M, K, dtype, 5)
        bias = torch.randn(N, device="cuda")
        y = w4_matvec(x, w, bias=bias, out_dtype=ref.torch_dtype(out))
        compare(y, ref.f64(x), dense(w), out, ref.f64(bias))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("pad", [1, 3, 8, 24])
def test_matvec_ignores_what_lies_beyond(cuda_device, dtype, pad):
    """x as a slice of a wider tensor that holds NaN, aligned or not; noise in q beyond column K."""
    import torch
    from paper_1905_00689_gb300 import w4_matvec
    for K in (37, 64, 200, 333):
        w = matrix(50, K, 32, 6, extra=32)
        x = rows(3, K, dtype, 7, pad)
        y = w4_matvec(x, w)
        compare(y, ref.f64(x), dense(w), dtype)
        assert torch.equal(y, w4_matvec(x.contiguous(), w))
        moved = torch.empty(3 * K + 1, dtype=x.dtype, device="cuda")[1:].reshape(3, K)
        moved.copy_(x)
        assert torch.equal(y, w4_matvec(moved, w))
    one = rows(1, 64, dtype, 8)
    assert torch.equal(w4_matvec(one.expand(4, 64), matrix(9, 64, 32, 1)), w4_matvec(one.repeat(4, 1), matrix(9, 64, 32, 1)))
    y3 = w4_matvec(rows(6, 64, dtype, 9).reshape(2, 3, 64), matrix(9, 64, 32, 1))
    assert torch.equal(y3.reshape(6, 9), w4_matvec(rows(6, 64, dtype, 9), matrix(9, 64, 32, 1)))


@pytest.mark.gpu
def test_matvec_rows_and_far_weights(cuda_device):
    """Rows do not mix: one that is not finite leaves the others alone.  Weight offsets past 2^31 bytes."""
    import torch
    from paper_1905_00689_gb300 import W4Weight, w4_matvec
    w, x = matrix(100, 300, 128, 11), rows(9, 300, "bf16", 12)
    want = w4_matvec(x, w)
    bad = x.clone()
    bad[4, 7], bad[6, 299] = float("nan"), float("inf")
    got = w4_matvec(bad, w)
    keep = [0, 1, 2, 3, 5, 7, 8]
    assert torch.equal(got[keep], want[keep]) and torch.isnan(got[4]).all() and not torch.isfinite(got[6]).any()
    big = torch.empty(3 << 30, dtype=torch.uint8, device="cuda")
    q = big.as_strided((3, 160), (1 << 30, 1))
    q.copy_(w.q[:3])
    far = W4Weight(q, w.scale[:3].contiguous(), w.zero[:3].contiguous(), 300, 128)
    assert torch.equal(w4_matvec(x, far), want[:, :3])


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 40, 128), (2, 33, 1000), (5, 64, 999), (16, 130, 2048), (20, 9, 300)])
@pytest.mark.parametrize("group", [32, 64, 128])
def test_matvec_8bit(cuda_device, M, N, K, group):
    import torch
    from paper_1905_00689_gb300 import rms_norm_quant, w4_matvec
    x, weight = rows(M, K, "bf16", 13), torch.ones(K, device="cuda")
    w = matrix(N, K, group, 14)
    for x_group in (128, K):
        q, scale, _ = rms_norm_quant(x, weight, group=x_group)
        each = np.arange(K) // 128 if scale.shape[1] > 1 else np.zeros(K, int)
        vals = ref.f64(q.float()) * ref.f64(scale)[:, each]
        for out in ("bf16", "fp32", "fp16"):
            y = w4_matvec(q, w, x_scale=scale, out_dtype=ref.torch_dtype(out))
            compare(y, vals, dense(w), out)
    assert w4_matvec(q, w, x_scale=scale).dtype == torch.bfloat16


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("scale", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("N,K,group", [(1, 1, 32), (3, 50, 32), (20, 300, 128), (7, 129, 64), (16, 1024, 128)])
def test_quantize(cuda_device, N, K, group, scale, dtype):
    """Bit for bit the stated rule; half a step of error; what it makes is what the product reads."""
    import torch
    from paper_1905_00689_gb300 import w4_matvec, w4_quantize
    w = rows(N, K, dtype, 15, pad=1)
    w[0, :32] = 0.0
    w[N - 1] = w[N - 1].abs()
    sd = ref.torch_dtype(scale)
    got = w4_quantize(w, group, scale_dtype=sd)
    q, s, z = ref.w4_quantize(w.float().cpu().numpy(), group, lambda v: torch.from_numpy(v).to(sd).float().numpy())
    assert np.array_equal(got.q.cpu().numpy(), q)
    assert np.array_equal(got.scale.float().cpu().numpy(), s) and np.array_equal(got.zero.cpu().numpy(), z)
    each = np.arange(K) // group
    # half a step for q, half for zero, and what the rounded scale (2^-9 at most) loses over 15 steps
    assert (np.abs(dense(got) - ref.f64(w)) <= s[:, each] * (1.0 + 15 * 2.0 ** -9)).all()
    x = rows(2, K, "fp32", 16)
    compare(w4_matvec(x, got), ref.f64(x), dense(got), "fp32")


@pytest.mark.gpu
def test_matvec_other_stream(cuda_device):
    import torch
    from paper_1905_00689_gb300 import w4_matvec, w4_quantize
    x, dense_w = rows(3, 640, "bf16", 17), rows(200, 640, "fp32", 18)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    w = w4_quantize(dense_w, stream=s)
    got = w4_matvec(x, w, stream=s)
    s.synchronize()
    assert torch.equal(got, w4_matvec(x, w4_quantize(dense_w)))


MATVEC = dict(xd=1, x=64, xp=64, xs=None, xg=0, q=64, qp=32, scale=64, sd=2, zero=64, bias=None, M=2, N=4, K=64, group=32,
              y=64, yd=1, ws=None, nbytes=0)
QUANTIZE = dict(d=0, w=64, wp=64, N=4, K=64, group=32, q=64, qp=32, scale=64, sd=2, zero=64)
BAD = ([(MATVEC, "w4_matvec", b) for b in (
            dict(xd=4), dict(yd=3), dict(xd=-1), dict(x=None), dict(y=None), dict(q=None), dict(scale=None), dict(q=72),
            dict(qp=40), dict(qp=16), dict(group=48), dict(group=256), dict(sd=3), dict(M=-1), dict(N=-1), dict(K=0),
            dict(xs=64), dict(xd=3), dict(xd=3, xs=64, xg=32), dict(x=65), dict(xp=-1), dict(scale=65), dict(bias=66),
            dict(y=65), dict(M=400), dict(M=400, ws=72, nbytes=1 << 30), dict(M=400, ws=64, nbytes=64))]
       + [(QUANTIZE, "w4_quantize", b) for b in (
            dict(d=3), dict(w=None), dict(zero=None), dict(q=None), dict(scale=None), dict(q=68), dict(qp=30),
            dict(qp=16), dict(group=16), dict(sd=-1), dict(K=0), dict(N=-1), dict(w=66), dict(wp=-1))])


@pytest.mark.parametrize("args,name,bad", BAD)
def test_w4_refusals(args, name, bad):
    """Refused before any device work (the pointers are never read)."""
    from paper_1905_00689_gb300 import load
    msg = ctypes.create_string_buffer(200)
    a = dict(args, **bad)
    assert getattr(load(), "lstm_approx_" + name)(*a.values(), None, msg, 200) == EINVAL and msg.value


@pytest.mark.gpu
def test_w4_wrapper_refusals(cuda_device):
    import torch
    from paper_1905_00689_gb300 import W4Weight, w4_matvec, w4_quantize
    w, x = matrix(8, 64, 32, 19), rows(2, 64, "bf16", 20)
    q8 = x.to(torch.float8_e4m3fn)
    one = torch.ones(2, 1, device="cuda")
    for call in (lambda: w4_matvec(x[:, :32], w), lambda: w4_matvec(x.double(), w), lambda: w4_matvec(x.cpu(), w),
                 lambda: w4_matvec(x, w, x_scale=one), lambda: w4_matvec(q8, w), lambda: w4_matvec(q8, w, x_scale=one[:1]),
                 lambda: w4_matvec(x, w, bias=torch.ones(7, device="cuda")),
                 lambda: w4_matvec(x, w, out=torch.empty(2, 9, device="cuda")),
                 lambda: W4Weight(w.q[:, 1:], w.scale, w.zero, 64, 32), lambda: W4Weight(w.q, w.scale, w.zero, 65, 32),
                 lambda: W4Weight(w.q, w.scale, w.zero, 64, 16), lambda: W4Weight(w.q, w.scale.double(), w.zero, 64, 32),
                 lambda: W4Weight(w.q, w.scale, w.zero.int(), 64, 32), lambda: w4_quantize(x, 256),
                 lambda: w4_quantize(x[0]), lambda: w4_quantize(x, scale_dtype=torch.float64)):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_rows_past_32_bits(cuda_device):
    """Rows of W 2^27 bytes apart, 20 of them: offsets past 2^31."""
    import torch
    from paper_1905_00689_gb300 import W4Weight, w4_matvec
    near = matrix(20, 100, 32, 8)
    q = torch.empty((20 << 27), dtype=torch.uint8, device="cuda").as_strided((20, near.q.shape[1]), (1 << 27, 1))
    q.copy_(near.q)
    x = rows(2, 100, "bf16", 9)
    assert torch.equal(w4_matvec(x, W4Weight(q, near.scale, near.zero, 100, 32)), w4_matvec(x, near))
