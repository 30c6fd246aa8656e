"""64-bit reference of the gated delta rule, written from its formula timestep by timestep (NumPy), and inputs for it."""
import numpy as np

import operator_reference as ref


def tensors(lead, H, Hk, Dk, Dv, dtype, seed, fused=False):
    """q, k of length 1, v, g in (-0.7, 0), beta in (0, 1); lead: (T, B) or (B,)."""
    import torch
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = ref.torch_dtype(dtype)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")
    if fused:
        z = normal(*lead, 2 * Hk * Dk + H * Dv).to(dt)
        q, k, v = z.split((Hk * Dk, Hk * Dk, H * Dv), -1)
        q, k, v = q.unflatten(-1, (Hk, Dk)), k.unflatten(-1, (Hk, Dk)), v.unflatten(-1, (H, Dv))
    else:
        q, k, v = (normal(*lead, *s).to(dt) for s in ((Hk, Dk), (Hk, Dk), (H, Dv)))
    for t in (q, k):
        t.copy_(t.float() / t.float().norm(dim=-1, keepdim=True))
    g = -torch.rand(*lead, H, generator=gen, device="cuda") ** 3 * 0.7
    beta = torch.sigmoid(normal(*lead, H))
    return q, k, v, g, beta


def scan(q, k, v, g, beta, h0=None, scale=None, lengths=None, reset=None, kept=None):
    """(o, h_last); kept: a list that receives, for every timestep, the state before it."""
    T, B, H, Dv = v.shape
    Hk, Dk = q.shape[2:]
    scale = Dk ** -0.5 if scale is None else scale
    n = [T] * B if lengths is None else [min(max(int(x), 0), T) for x in lengths]
    o = np.zeros((T, B, H, Dv))
    last = np.zeros((B, H, Dk, Dv)) if h0 is None else h0.copy()
    states = np.zeros((T, B, H, Dk, Dv)) if kept is not None else None
    for b in range(B):
        for h in range(H):
            S, c = last[b, h], h // (H // Hk)
            for t in range(n[b]):
                if kept is not None:
                    states[t, b, h] = S
                W = np.zeros_like(S) if reset is not None and reset[t, b] else S * np.exp(max(g[t, b, h], -200.0))
                u = beta[t, b, h] * (v[t, b, h] - W.T @ k[t, b, c])
                S = W + np.outer(k[t, b, c], u)
                o[t, b, h] = scale * S.T @ q[t, b, c]
            last[b, h] = S
    if kept is not None:
        kept.append(states)
    return o, last


def scan_backward(do, q, k, v, g, beta, h0=None, scale=None, lengths=None, reset=None, dh_last=None):
    """(dq, dk, dv, dg, dbeta, dh0) by the chain rule, from the end."""
    T, B, H, Dv = v.shape
    Hk, Dk = q.shape[2:]
    scale = Dk ** -0.5 if scale is None else scale
    n = [T] * B if lengths is None else [min(max(int(x), 0), T) for x in lengths]
    kept = []
    scan(q, k, v, g, beta, h0, scale, lengths, reset, kept)
    dq, dk, dv, dg, dbeta = (np.zeros_like(x) for x in (q, k, v, g, beta))
    dh0 = np.zeros((B, H, Dk, Dv))
    for b in range(B):
        for h in range(H):
            c = h // (H // Hk)
            dS = np.zeros((Dk, Dv)) if dh_last is None else dh_last[b, h].copy()
            for t in range(n[b] - 1, -1, -1):
                cut = reset is not None and reset[t, b]
                a = np.exp(max(g[t, b, h], -200.0))
                W = np.zeros((Dk, Dv)) if cut else kept[0][t, b, h] * a
                kt, qt, bt = k[t, b, c], q[t, b, c], beta[t, b, h]
                r = v[t, b, h] - W.T @ kt
                S = W + np.outer(kt, bt * r)
                dq[t, b, c] += scale * S @ do[t, b, h]
                dS = dS + scale * np.outer(qt, do[t, b, h])
                du = dS.T @ kt
                dk[t, b, c] += dS @ (bt * r) - W @ (bt * du)
                dv[t, b, h] = bt * du
                dbeta[t, b, h] = du @ r
                dW = dS - np.outer(kt, bt * du)
                dg[t, b, h] = (dW * W).sum()
                dS = np.zeros((Dk, Dv)) if cut else dW * a
            dh0[b, h] = dS
    return dq, dk, dv, dg, dbeta, dh0
