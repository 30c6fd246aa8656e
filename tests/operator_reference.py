"""64-bit references of the block's operators, written from their formulas
(NumPy; loops over timesteps and groups), and the comparison the tests use."""
import numpy as np

U32 = 2.0 ** -24  # unit roundoff of fp32
HALF_ULP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}  # 2^-p, p bits of significand
TINY = {"fp32": 1e-38, "bf16": 1e-38, "fp16": 2.0 ** -25}  # half the spacing of the smallest values


def torch_dtype(name):
    import torch
    return {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}[name]


def f64(t):
    return t.detach().double().cpu().numpy()


def check(got, want, scale, tol, dtype="fp32", what=""):
    """|got - want| <= tol scale + the rounding of want to `dtype`, element by element; not finite values
    where, and as, `want` has them.  scale: a number or an array of magnitudes that the errors of 32-bit
    arithmetic go by."""
    got = np.asarray(got if isinstance(got, np.ndarray) else f64(got), dtype=np.float64)
    want = np.asarray(want, dtype=np.float64)
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(np.isfinite(got), fine), what
    np.testing.assert_array_equal(got[~fine], want[~fine], err_msg=what)
    allowed = np.broadcast_to(tol * np.asarray(scale, dtype=np.float64), want.shape)
    allowed = allowed + (HALF_ULP[dtype] * (np.abs(want) + allowed) + TINY[dtype] if dtype != "fp32" else 0.0)
    bad = fine & (np.abs(got - want) > allowed)
    assert not bad.any(), (what, int(bad.sum()), float(np.abs(got - want)[bad].max()),
                           float(allowed[bad].min()), np.argwhere(bad)[:4].tolist())


# ---- norm -------------------------------------------------------------------

def norm(x, w, residual=None, eps=1e-6):
    s = x if residual is None else x + residual
    rstd = 1.0 / np.sqrt((s * s).mean(-1) + eps)
    return s, rstd, s * rstd[..., None] * w


def norm_backward(dy, s, w, dsum=None, eps=1e-6):
    """By the quotient rule on y_j = w_j s_j / sqrt(mean s^2 + eps)."""
    D = s.shape[-1]
    rms = np.sqrt((s * s).mean(-1, keepdims=True) + eps)
    along = (dy * w * s).sum(-1, keepdims=True)
    ds = dy * w / rms - s * along / (D * rms ** 3)
    return ds + (0.0 if dsum is None else dsum), (dy * s / rms).reshape(-1, D).sum(0)


# ---- recurrence -------------------------------------------------------------

def sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0, e) / (1.0 + e)


def softplus(z):
    return np.maximum(z, 0.0) + np.log1p(np.exp(-np.abs(z)))


def gates(r, i, decay, c):
    sr, si = sigmoid(r), sigmoid(i)
    la = -c * softplus(decay) * sr
    return sr, si, la, np.exp(la), np.sqrt(-np.expm1(2.0 * la))


def scan(x, r, i, decay, c=8.0, h0=None, lengths=None, reset=None):
    """(y, h_last, h [T + 1, B, D]): the recurrence, stream by stream and timestep by timestep."""
    T, B, D = x.shape
    y = np.zeros((T, B, D))
    hs = np.zeros((T + 1, B, D))
    last = np.zeros((B, D))
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        h = np.zeros(D) if h0 is None else h0[b].copy()
        hs[0, b] = h
        for t in range(n):
            _, si, _, a, m = gates(r[t, b], i[t, b], decay, c)
            u = m * si * x[t, b]
            h = u if reset is not None and reset[t, b] else a * h + u
            y[t, b] = hs[t + 1, b] = h
        hs[n + 1:, b] = h
        last[b] = h
    return y, last, hs


def scan_backward(dy, x, r, i, decay, c=8.0, h0=None, lengths=None, reset=None, dh_last=None):
    """(dx, dr, di, ddecay, dh0, sum of |terms| of ddecay), timestep by timestep from the end, in the chain
    rule's own terms (dL/da, dL/dm)."""
    T, B, D = x.shape
    _, _, hs = scan(x, r, i, decay, c, h0, lengths, reset)
    dx, dr, di = np.zeros((3, T, B, D))
    ddecay, terms, dh0 = np.zeros(D), np.zeros(D), np.zeros((B, D))
    sp = softplus(decay)
    for b in range(B):
        n = T if lengths is None else min(max(int(lengths[b]), 0), T)
        g = np.zeros(D) if dh_last is None else dh_last[b].copy()
        for t in range(n - 1, -1, -1):
            sr, si, la, a, m = gates(r[t, b], i[t, b], decay, c)
            cut = reset is not None and reset[t, b]
            g = g + dy[t, b]
            before = np.zeros(D) if cut else hs[t, b]
            with np.errstate(divide="ignore", invalid="ignore"):
                dm = np.where(m > 0, -a * a / m, 0.0)
            dla = g * before * a + g * si * x[t, b] * dm
            dx[t, b] = g * m * si
            di[t, b] = g * m * x[t, b] * si * (1.0 - si)
            dr[t, b] = dla * -c * sp * sr * (1.0 - sr)
            term = dla * -c * sr * sigmoid(decay)
            ddecay += term
            terms += np.abs(term)
            g = np.zeros(D) if cut else g * a
        dh0[b] = g
    return dx, dr, di, ddecay, dh0, terms


# ---- 4-bit matrices ---------------------------------------------------------

def w4_unpack(q, K):
    q = np.asarray(q)
    return np.stack([q & 15, q >> 4], -1).reshape(q.shape[0], 2 * q.shape[1])[:, :K]


def w4_matrix(q, scale, zero, K, group):
    each = np.arange(K) // group
    z = 8.0 if zero is None else np.asarray(zero, dtype=np.float64)[:, each]
    return (w4_unpack(q, K) - z) * np.asarray(scale, dtype=np.float64)[:, each]


def w4_quantize(w, group, round_scale):
    """The stated rule in fp32; round_scale: fp32 -> the scale's type -> fp32."""
    N, K = w.shape
    G = -(-K // group)
    q = np.zeros((N, -(-K // 32) * 16), np.uint8)
    scale, zero = np.zeros((N, G), np.float32), np.zeros((N, G), np.uint8)
    for g in range(G):
        part = w[:, g * group:min(K, (g + 1) * group)].astype(np.float32)
        lo = np.minimum(part.min(1), np.float32(0))
        hi = np.maximum(part.max(1), np.float32(0))
        s = round_scale((hi - lo) / np.float32(15))
        s = np.where(s == 0, np.float32(1), s)
        z = np.clip(np.rint(-lo / s), 0, 15)
        v = np.clip(np.rint(part / s[:, None]) + z[:, None], 0, 15).astype(np.uint8)
        for k in range(part.shape[1]):
            col = g * group + k
            q[:, col // 2] |= v[:, k] << (4 * (col % 2))
        scale[:, g], zero[:, g] = s, z
    return q, scale, zero
