"""The AdamW step over many tensors, with averages in 32 and in 8 bits."""
import ctypes

import numpy as np
import pytest

import operator_reference as ref

EINVAL = 1
U = ref.U32
LR, B1, B2, EPS, WD = 1e-2, 0.9, 0.999, 1e-8, 0.1
SIZES = [1, 7, 8, 255, 256, 257, 2047, 2048, 2049, 5000, 0]


def make(sizes, dtype, gdtype, seed, apart=0, bits=32):
    """Tensors cut out of one allocation each, `apart` values after a 16-byte boundary."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def cut(dt, scale=1.0, square=False):
        out = []
        for n in sizes:
            x = torch.randn(n + 16, generator=gen, device="cuda") * scale
            out.append((x.square() if square else x).to(dt)[apart:apart + n])
        return out
    p, g = cut(ref.torch_dtype(dtype)), cut(ref.torch_dtype(gdtype), 0.1)
    if bits == 32:
        return p, g, cut(torch.float32, 0.05), cut(torch.float32, 0.1, True), None, None
    m, u = ([t.clamp(-448, 448).to(torch.float8_e4m3fn) for t in cut(torch.float32, 100.0)] for _ in range(2))
    u = [t.float().abs().to(torch.float8_e4m3fn) for t in u]
    scales = [[torch.rand(-(-n // 256), generator=gen, device="cuda") * s + s for n in sizes] for s in (1e-4, 3e-4)]
    return p, g, m, u, *scales


def want(p, g, m, v, t, clip=1.0, lr=LR, b1=B1, b2=B2, eps=EPS, wd=WD):
    """(p, m, v, and the magnitudes their 32-bit errors go by), in 64 bits."""
    p, g, m, v = (np.asarray(x, dtype=np.float64) for x in (p, g, m, v))
    g = g * clip
    m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
    m_terms = b1 * np.abs(m) + (1 - b1) * np.abs(g)
    under = np.sqrt(v1 / (1 - b2 ** t)) + eps
    return p * (1 - lr * wd) - lr / (1 - b1 ** t) * m1 / under, m1, v1, m_terms, lr / (1 - b1 ** t) * m_terms / under


def check_step(before, after, t, dtype, clip=1.0, **more):
    """m: four roundoffs of its terms (constants, products, sum), v: six of itself.  p: of itself four; of the step 32: m 4,
    sqrt(v) 5, the corrections' exponentials 8 and the division 4, the products."""
    w, m1, v1, m_terms, step = want(*before, t, clip, **more)
    ref.check(after[1], m1, m_terms, 6 * U, what="m")
    ref.check(after[2], v1, v1, 8 * U, what="v")
    ref.check(after[0], w, 4 * U * np.abs(w) + 32 * U * step, 1.0, dtype, "p")


@pytest.mark.gpu
@pytest.mark.parametrize("apart", [0, 1, 8])
@pytest.mark.parametrize("dtype,gdtype", [("fp32", "fp32"), ("fp32", "bf16"), ("bf16", "bf16"), ("fp16", "fp32")])
def test_32_bits(cuda_device, dtype, gdtype, apart):
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    p, g, m, v, _, _ = make(SIZES, dtype, gdtype, 1, apart)
    copies = [torch.full_like(x, float("nan"), dtype=torch.bfloat16) if i % 2 else None for i, x in enumerate(p)]
    state = AdamWState(m, v)
    for t in (1, 2, 1000):
        before = [[ref.f64(x) for x in (p[i], g[i], m[i], v[i])] for i in range(len(p))]
        adamw_step(p, g, state, t, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, copies=copies)
        for i, b in enumerate(before):
            check_step(b, (p[i], m[i], v[i]), t, dtype)
            if copies[i] is not None and dtype == "fp32":
                assert torch.equal(copies[i], p[i].to(torch.bfloat16))


def neighbours(x):
    """The e4m3 values at or below and at or above x >= 0."""
    e = np.where(x < 2.0 ** -6, -6.0, np.floor(np.log2(np.maximum(x, 2.0 ** -6))))
    unit = 2.0 ** (e - 3)
    return np.floor(x / unit) * unit, np.minimum(np.ceil(x / unit) * unit, 448.0)


def check_8_bits(value, error, q, scale, positive):
    """q is one of the neighbours of what 32 bits make of value / scale: value within `error`, the quotient and the sum
    with the random bits within eight roundoffs of it."""
    n = value.size
    each = np.arange(n) // 256
    scale, q = ref.f64(scale), ref.f64(q)
    least, most = (np.array([s[i * 256:(i + 1) * 256].max() for i in range(len(scale))]) / 448.0
                   for s in (np.abs(value) - error, np.abs(value) + error))
    assert (scale >= np.maximum(least, 2.0 ** -126) * (1 - 4 * U)).all()
    assert (scale <= np.maximum(most, 2.0 ** -126) * (1 + 4 * U)).all()
    x, off = np.abs(value) / scale[each], error / scale[each]
    lo, hi = (neighbours(np.clip(s, 0, 448.0))[k] for k, s in enumerate(((x - off) * (1 - 8 * U), (x + off) * (1 + 8 * U))))
    if positive:
        lo, hi = (np.where(value > 0, np.maximum(s, 2.0 ** -9), s) for s in (lo, hi))
    a = np.abs(q)
    assert ((a >= lo) & (a <= hi)).all()
    assert (np.signbit(q) == np.signbit(value))[np.abs(value) > error].all()


@pytest.mark.gpu
@pytest.mark.parametrize("apart", [0, 1, 8])
@pytest.mark.parametrize("dtype,gdtype", [("fp32", "bf16"), ("bf16", "bf16"), ("fp16", "fp16")])
def test_8_bits(cuda_device, dtype, gdtype, apart):
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    p, g, m, u, ms, us = make(SIZES, dtype, gdtype, 2, apart, bits=8)
    clip = torch.tensor([0.5], device="cuda")
    for i, n in enumerate(SIZES):  # a block of zeros, an average of zero beside others
        if n > 256:
            m[i][:256], u[i][:256], g[i][:256] = 0, 0, 0
            u[i][256], g[i][256] = 0, 0
    before = []
    for i in range(len(p)):
        each = torch.arange(SIZES[i], device="cuda") // 256
        before.append([ref.f64(p[i]), ref.f64(g[i]), ref.f64(m[i]) * ref.f64(ms[i][each]),
                       (ref.f64(u[i]) * ref.f64(us[i][each])) ** 2])
    adamw_step(p, g, AdamWState(m, u, ms, us), 3, lr=LR, betas=(B1, B2), eps=EPS, weight_decay=WD, grad_scale=clip, seed=5)
    for i, b in enumerate(before):
        if SIZES[i] == 0:
            continue
        w, m1, v1, m_terms, step = want(*b, 3, 0.5)
        if dtype == "fp16":  # a step over a v of zero (m / eps) is beyond the type: from 65520 on it rounds to infinity
            w = np.where(np.abs(w) >= 65520, np.copysign(np.inf, w), w)
        ref.check(p[i], w, 4 * U * np.abs(np.nan_to_num(w)) + 40 * U * step, 1.0, dtype, "p")
        check_8_bits(m1, 6 * U * m_terms, m[i], ms[i], False)
        check_8_bits(np.sqrt(v1), 6 * U * np.sqrt(v1), u[i], us[i], True)


@pytest.mark.gpu
def test_8_bit_averages_move_as_they_should(cuda_device):
    """A value that lies between two 8-bit ones becomes the upper one as often as its place says: over n trials of variance
    under 1/4 the mean is within 5 / (2 sqrt(n)) of it; another seed or step rounds others.  So an average whose steps are
    small against 8 bits still gets where it should."""
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    n = 1 << 18
    target = torch.linspace(0.1, 1.0, 256, device="cuda").repeat(n // 256)
    target[::256] = 1.0
    first = {}
    for key in ((1, 1), (1, 2), (2, 1), (1, 1)):
        p, state = [torch.zeros(n, device="cuda")], AdamWState.zeros([torch.zeros(n, device="cuda")], 8)
        adamw_step(p, [target], state, key[0], lr=0.0, betas=(0.0, 0.0), weight_decay=0.0, seed=key[1])
        for which, (q, s) in enumerate(((state.exp_avg, state.exp_avg_scale), (state.exp_avg_sq, state.exp_avg_sq_scale))):
            q, s = ref.f64(q[0]).reshape(-1, 256), ref.f64(s[0])
            x = ref.f64(target)[:256] / s[0]
            lo, hi = neighbours(x)
            unit = np.where(hi > lo, hi - lo, 1.0)
            up = (q - lo) / unit
            assert np.isin(up, (0.0, 1.0)).all()
            chance = np.where(hi > lo, (x - lo) / unit, 0.0)
            assert (np.abs(up.mean(0) - chance) <= 2.5 / np.sqrt(n / 256) + 2.0 ** -16).all()
            assert abs((up - chance).mean()) <= 2.5 / np.sqrt(n) + 2.0 ** -16
            if (key, which) in first:
                np.testing.assert_array_equal(first[key, which], up)
            else:
                assert all((v != up).any() for (k, w), v in first.items() if w == which)
            first[key, which] = up
        assert (first[key, 0] != first[key, 1]).any()
    # 1000 steps of a constant gradient: the average of squares reaches 1 - 0.999^1000 = 0.632 of its square; its root as
    # stored wanders by at most 2^-4 of itself a step, and the mean over 2048 values by far less
    p, g = [torch.zeros(2048, device="cuda")], [torch.ones(2048, device="cuda")]
    state = AdamWState.zeros(p, 8)
    for t in range(1, 1001):
        adamw_step(p, g, state, t, lr=0.0)
    u = ref.f64(state.exp_avg_sq[0]) * ref.f64(state.exp_avg_sq_scale[0]).repeat(256)
    assert abs((u ** 2).mean() - 0.632) < 0.05
    m = ref.f64(state.exp_avg[0]) * ref.f64(state.exp_avg_scale[0]).repeat(256)
    assert abs(m.mean() - 1.0) < 0.02


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_many_tensors(cuda_device, bits):
    """More tensors than one launch takes, of unlike types, some without a gradient: the bits of a call for each (with 8 bits
    a position counts from the list's beginning, so there only the 32-bit results are)."""
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    sizes = [int(n) for n in np.random.default_rng(3).integers(0, 700, 1000)]
    kinds = ["fp32", "bf16", "fp16"]
    per = [make([n], kinds[i % 3], kinds[i // 3 % 3], i, i % 5, bits) for i, n in enumerate(sizes)]
    p, g, m, v = ([x[k][0] for x in per] for k in range(4))
    ms, vs = ([x[k][0] for x in per] if bits == 8 else None for k in (4, 5))
    none = {5, 17, 380, 999}
    g = [None if i in none else x for i, x in enumerate(g)]
    single = [[t.clone() for t in x] for x in (p, m, v)]
    scales = [[t.clone() for t in x] if x else None for x in (ms, vs)]
    old = [p[i].clone() for i in none]
    adamw_step(p, g, AdamWState(m, v, ms, vs), 7, lr=LR)
    for i in range(1000):
        one = AdamWState([single[1][i]], [single[2][i]], *([x[i]] if x else None for x in scales))
        adamw_step([single[0][i]], [g[i]], one, 7, lr=LR)
        assert torch.equal(single[0][i], p[i]), i
        if bits == 32:
            assert torch.equal(single[1][i], m[i]) and torch.equal(single[2][i], v[i])
        else:
            assert torch.equal(scales[0][i], ms[i]) and torch.equal(scales[1][i], vs[i])
    assert all(torch.equal(a, p[i]) for a, i in zip(old, none))


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
def test_captured(cuda_device, bits):
    """A captured call with step, rate, scale and skip on the device gives the bits of plain ones."""
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    shape = (33, 70)
    p = [torch.randn(shape, device="cuda"), torch.randn(5, device="cuda")]
    g = [torch.randn_like(t) for t in p]
    state = AdamWState.zeros(p, bits)
    q = [t.clone() for t in p]
    other = AdamWState.zeros(q, bits)
    step, lr = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros((), device="cuda")
    skip, clip = torch.zeros(1, dtype=torch.bool, device="cuda"), torch.ones((), device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step += 1
        adamw_step(p, g, state, step, lr=lr, grad_scale=clip, skip=skip, seed=3)
    step.zero_()
    for t in range(1, 5):
        lr.fill_(0.1 / t)
        clip.fill_(1.0 / t)
        for x in g:
            x.normal_()
        skip.fill_(t == 3)
        graph.replay()
        if t != 3:
            adamw_step(q, g, other, t, lr=float(lr), grad_scale=clip, seed=3)
        for a, b in zip(p + state.exp_avg + state.exp_avg_sq, q + other.exp_avg + other.exp_avg_sq):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), t


@pytest.mark.gpu
def test_on_a_stream_and_not_finite(cuda_device):
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    for bits in (8, 32):
        p, g = [torch.ones(600, device="cuda")], [torch.full((600,), 0.5, device="cuda")]
        state = AdamWState.zeros(p, bits)
        side = torch.cuda.Stream()
        torch.cuda.synchronize()
        adamw_step(p, g, state, 1, lr=0.5, weight_decay=0.0, stream=side)
        side.synchronize()
        assert float((p[0] - 0.5).abs().max()) < 1e-5  # the first step has the rate's size
        g[0][300] = float("nan")  # its own value, and with 8 bits what shares its scale
        adamw_step(p, g, state, 2, lr=0.5)
        assert torch.isnan(p[0][300]) and int(torch.isnan(p[0]).sum()) == 1
        adamw_step(p, [torch.ones_like(p[0])], state, 3, lr=0.5)
        assert int(torch.isnan(p[0]).sum()) == (256 if bits == 8 else 1)
    # betas of zero, gradients of zero, nothing to do
    p = [torch.ones(10, device="cuda")]
    adamw_step(p, [torch.zeros(10, device="cuda")], AdamWState.zeros(p), 1, lr=0.1, betas=(0.0, 0.0), weight_decay=0.0)
    assert (p[0] == 1).all()
    adamw_step([], [], AdamWState([], []), 1, lr=0.1)


@pytest.mark.gpu
def test_refuses_tensors(cuda_device):
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    p, g = [torch.ones(300, device="cuda")], [torch.ones(300, device="cuda")]
    state, small = AdamWState.zeros(p), AdamWState.zeros(p, 8)
    for bits in (16, 0):
        with pytest.raises(ValueError):
            AdamWState.zeros(p, bits)
    with pytest.raises(ValueError):
        AdamWState(small.exp_avg, small.exp_avg_sq)
    with pytest.raises(ValueError):
        AdamWState(state.exp_avg, [])
    with pytest.raises(ValueError):
        AdamWState(small.exp_avg, small.exp_avg_sq, small.exp_avg_scale)
    bad = [dict(params=p + p), dict(grads=[]), dict(grads=[g[0][:299]]), dict(grads=[g[0].double()]), dict(grads=[g[0].cpu()]),
           dict(params=[p[0].cpu()]), dict(params=[torch.ones(600, device="cuda")[::2]]), dict(step=0), dict(step=2 ** 31),
           dict(step=torch.ones(1, device="cuda")), dict(lr=float("nan")), dict(betas=(1.0, 0.5)), dict(betas=(0.5, -0.1)),
           dict(betas=(0.5,)), dict(eps=-1.0), dict(copies=[]), dict(copies=[torch.ones(299, device="cuda")]),
           dict(grad_scale=torch.ones(2, device="cuda")), dict(skip=torch.ones(1, device="cuda")), dict(params=3),
           dict(state=AdamWState.zeros([torch.ones(299, device="cuda")])), dict(weight_decay=float("inf")),
           dict(state=AdamWState(small.exp_avg, small.exp_avg_sq, [torch.ones(1, device="cuda")], [torch.ones(2, device="cuda")]))]
    for change in bad:
        args = {**dict(params=p, grads=g, state=state, step=1, lr=0.1), **change}
        with pytest.raises((ValueError, RuntimeError)):
            adamw_step(**args)
    both = [torch.ones(400, device="cuda")]
    with pytest.raises(ValueError):  # parameters that overlap
        adamw_step([both[0][:300], both[0][299:]], [g[0], g[0][:101]],
                   AdamWState.zeros([both[0][:300], both[0][299:]]), 1, lr=0.1)
    assert (p[0] == 1).all() and (state.exp_avg[0] == 0).all()


def test_refusals(lib):
    class Tensor(ctypes.Structure):
        _fields_ = [(n, ctypes.c_void_p) for n in ("p", "m", "v", "copy", "g", "m_scale", "v_scale")] + \
                   [("n", ctypes.c_longlong)] + [(n, ctypes.c_int) for n in ("p_dtype", "g_dtype", "copy_dtype")]
    msg = ctypes.create_string_buffer(256)
    good = dict(p=256, m=256, v=256, copy=None, g=256, m_scale=256, v_scale=256, n=10, p_dtype=0, g_dtype=0, copy_dtype=0)

    def call(tensor={}, count=1, bits=8, step=1, step_at=None, lr=0.1, lr_at=None, b1=0.9, b2=0.99, eps=1e-8, wd=0.0):
        t = Tensor(**{**good, **tensor})
        return lib.lstm_approx_adamw_step(count, ctypes.byref(t), bits, step, step_at, lr, lr_at, b1, b2, eps, wd, None, None,
                                          0, None, msg, 256)
    for change in (dict(p=None), dict(m=None), dict(v=None), dict(m_scale=None), dict(v_scale=None), dict(n=-1),
                   dict(n=1 << 41), dict(p_dtype=3), dict(g_dtype=-1), dict(copy=256, copy_dtype=7), dict(p=258), dict(g=257),
                   dict(m_scale=257), dict(copy=257, copy_dtype=1)):
        assert call(change) == EINVAL, change
        assert msg.value
    assert call(dict(m=258), bits=32) == EINVAL
    for more in (dict(count=-1), dict(bits=16), dict(step=0), dict(b1=1.0), dict(b1=-0.1), dict(b2=float("nan")), dict(eps=-1.0),
                 dict(eps=float("inf")), dict(lr=float("inf")), dict(wd=float("nan")), dict(step_at=ctypes.c_void_p(2)),
                 dict(lr_at=ctypes.c_void_p(2))):
        assert call(**more) == EINVAL, more


@pytest.mark.gpu
@pytest.mark.parametrize("bits", [8, 32])
@pytest.mark.parametrize("dtype,gdtype", [("fp32", "fp32"), ("bf16", "fp16")])
def test_every_alignment(cuda_device, bits, dtype, gdtype):
    """Tensors that begin at any value of an allocation: the bits of the aligned ones, and nothing beside them is written."""
    import torch
    from paper_1905_00689_gb300 import AdamWState, adamw_step
    n = 1000
    base = make([n], dtype, gdtype, 11, 0, bits)
    base = [x[0] for x in base if x is not None]
    want = [t.clone() for t in base] + [torch.zeros(n, dtype=torch.float16, device="cuda")]
    scales = lambda t: ([[t[4]], [t[5]]] if bits == 8 else [None, None])  # noqa: E731
    adamw_step([want[0]], [want[1]], AdamWState([want[2]], [want[3]], *scales(want)), 3, lr=LR, copies=[want[-1]])
    for shift in range(1, 17):
        big = [torch.full((n + 40,), 1.0, device="cuda").to(t.dtype) for t in base[:4]] + \
              [torch.ones(n + 40, dtype=torch.float16, device="cuda")]
        # each of the five at a place of its own
        at = [(shift * k) % 17 for k in (1, 3, 5, 7, 11)]
        part = [b[a:a + n] for b, a in zip(big, at)]
        for x, t in zip(part, base[:4]):
            x.copy_(t)
        own = [t.clone() for t in base[4:]]
        adamw_step([part[0]], [part[1]], AdamWState([part[2]], [part[3]], *([[t] for t in own] if bits == 8 else [None, None])), 3,
                   lr=LR, copies=[part[4]])
        for k, (x, w) in enumerate(zip(part, want[:4] + want[-1:])):
            assert torch.equal(x.view(torch.uint8), w.view(torch.uint8)), (shift, k)
        for b, a in zip(big, at):
            assert (b[:a].float() == 1).all() and (b[a + n:].float() == 1).all()
