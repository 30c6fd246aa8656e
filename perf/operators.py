"""The operators of a gated-linear-recurrence block, as plain cases.

A recurrent language model whose gates do not see h_{t-1} is built of blocks
norm -> projections -> recurrence -> projection.  It is trained on whole
sequences and then serves single tokens of many streams.  The operators:

- norm: root-mean-square norm with the residual's addition; the output in the
  input's type, or as 8-bit floats (e4m3) with a scale for each group of
  columns; its backward pass;
- scan: h_t = a_t h_{t-1} + sqrt(1 - a_t^2) sigma(i_t) x_t with
  a_t = exp(-c softplus(decay) sigma(r_t)) over a sequence, with resets (packed
  documents), lengths (ragged batches) and an initial state; its backward pass;
- step: one timestep of it on a pool of states;
- w4: matrix-vector products y = x W^T with 4-bit weights, a scale and a zero
  point for each group of columns, x in 32 or 16 bits or as the norm's 8-bit
  output.

Sequences are time-major, [T][B][D], as everywhere in this package.  The plain
forms below are elementary torch operations in 32 bits, rounded once at the end.
"""
import math

import torch

own = False

C = 8.0            # the constant of the decay's exponent
EPS = 1e-6
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------
# cases

def _norm(name, dtype, rows, D, group=0, residual=True, train=False):
    return {"name": name, "kind": "norm", "dtype": dtype, "rows": rows, "D": D, "group": group,
            "residual": residual, "train": train}


def _scan(name, dtype, T, B, D, train=False, fused=False, ragged=False, resets=0.0, state=False):
    return {"name": name, "kind": "scan", "dtype": dtype, "T": T, "B": B, "D": D, "train": train, "fused": fused,
            "ragged": ragged, "resets": resets, "state": state}


def _step(name, dtype, B, D, pool=0, fused=False):
    return {"name": name, "kind": "step", "dtype": dtype, "B": B, "D": D, "pool": pool, "fused": fused}


def _w4(name, dtype, M, N, K, group, x8=False, bias=False):
    return {"name": name, "kind": "w4", "dtype": dtype, "M": M, "N": N, "K": K, "group": group, "x8": x8,
            "bias": bias}


def listed():
    return [
        # one token of one stream: the norm before 8-bit projections
        _norm("norm-one-token-8bit", "bf16", 1, 2048, group=128),
        # a prompt of 8192 tokens, or 8 x 1024, at the widest model
        _norm("norm-prompt", "bf16", 8192, 4096),
        # a training step (forward and backward) in 32 bits at odd sizes
        _norm("norm-train-odd", "fp32", 5001, 1531, train=True),
        # one token for each of 64 streams, gates as slices of one projection's output
        _step("step-64-streams", "bf16", 64, 1024, fused=True),
        # one token for each of 1000 streams whose states lie scattered in a pool
        _step("step-pool", "fp16", 1000, 2048, pool=1500),
        # the prompt of one stream, an odd length, gates as slices of one projection's output
        _scan("scan-prompt", "bf16", 8191, 1, 2048, fused=True),
        # prompts of unlike lengths, padded, resumed from states
        _scan("scan-ragged", "fp16", 700, 13, 1000, ragged=True, state=True),
        # a training step (forward and backward) on packed documents
        _scan("scan-train", "bf16", 2048, 8, 2048, train=True, resets=1 / 500),
        # a training step on one long sequence in 32 bits
        _scan("scan-train-long", "fp32", 20000, 1, 512, train=True, state=True),
        # one token of one stream
        _w4("w4-one-token", "bf16", 1, 8192, 2048, 128),
        # 16 streams on the norm's 8-bit output, a wide matrix
        _w4("w4-16-streams-8bit", "bf16", 16, 16384, 4096, 64, x8=True),
        # a small matrix of odd sizes in 32 bits, three streams
        _w4("w4-odd", "fp32", 3, 3001, 1000, 32, bias=True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("norm", "norm", "step", "scan", "scan", "w4", "w4"))
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    odd = rng.random() < 0.4

    def width(lo, hi):
        n = _log(rng, lo, hi)
        return n if odd else max(lo, n // 64 * 64)

    if kind == "norm":
        D = width(64, 8192)
        rows = _log(rng, 1, max(1, min(20000, 32_000_000 // D)))
        train = rng.random() < 0.4
        group = 0 if train or rng.random() < 0.5 else rng.choice((128, D))
        case = _norm("", dtype, rows, D, group=group, residual=rng.random() < 0.7, train=train)
    elif kind == "step":
        D = width(64, 4096)
        B = _log(rng, 1, max(1, min(1024, 4_000_000 // D)))
        case = _step("", dtype, B, D, pool=rng.choice((0, B + _log(rng, 1, 500))), fused=rng.random() < 0.5)
    elif kind == "scan":
        D = width(64, 4096)
        B = _log(rng, 1, 16)
        train = rng.random() < 0.5
        T = _log(rng, 1, max(2, min(20000, 30_000_000 // (B * D))))
        case = _scan("", dtype, T, B, D, train=train, fused=rng.random() < 0.5, ragged=rng.random() < 0.3,
                     resets=rng.choice((0.0, 0.0, 0.002, 0.1)), state=rng.random() < 0.5)
    else:
        K, N = width(64, 8192), width(64, 16384)
        N = min(N, 64_000_000 // K)
        case = _w4("", dtype, _log(rng, 1, 16), N, K, rng.choice((32, 64, 128)), bias=rng.random() < 0.3,
                   x8=rng.random() < 0.3)
    del case["name"]
    return case


def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "norm":
        n, rows, D = case["rows"] * case["D"], case["rows"], case["D"]
        ins = n * e * (2 if case["residual"] else 1) + D * 4
        outs = n * e if case["residual"] else 0
        outs += n + 4 * rows * -(-D // case["group"]) if case["group"] else n * e
        flops = 6 * n
        if case["train"]:  # rstd kept; backward reads dy, the sum and its gradient, writes the gradient and dw
            outs += 4 * rows
            ins += n * e * 3 + 4 * rows + 4 * D
            outs += n * e + 4 * D
            flops += 12 * n
        return {"bytes": ins + outs, "flops": flops}
    if case["kind"] == "step":
        n = case["B"] * case["D"]
        return {"bytes": n * (4 * e + 8) + 4 * case["D"] + (4 * case["B"] if case["pool"] else 0), "flops": 30 * n}
    if case["kind"] == "scan":
        T, B, D = case["T"], case["B"], case["D"]
        n = T * B * D
        small = 4 * D + 4 * B * D * (2 if case["state"] else 1)
        small += T * B if case["resets"] else 0
        total, flops = 4 * n * e + small, 30 * n
        if case["train"]:
            total += 7 * n * e + 2 * small + 8 * D
            flops += 60 * n
        return {"bytes": total, "flops": flops}
    M, N, K = case["M"], case["N"], case["K"]
    G = -(-K // case["group"])
    xbytes = M * K + 4 * M * -(-K // 128) if case["x8"] else M * K * e
    return {"bytes": N * -(-K // 2) + 3 * N * G + xbytes + M * N * e + (4 * N if case["bias"] else 0),
            "flops": 2 * M * N * K}


# ---------------------------------------------------------------------------
# inputs

def _packed(v, pitch):
    """4-bit values [N][K] as bytes [N][pitch], the even column in the low half."""
    N, K = v.shape
    full = torch.zeros(N, 2 * pitch, dtype=torch.uint8, device=v.device)
    full[:, :K] = v
    return full[:, 0::2] | (full[:, 1::2] << 4)


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0, dtype=dt):
        return (torch.randn(*shape, generator=gen, device="cuda") * std + mean).to(dtype)

    def uniform(*shape, lo=0.0, hi=1.0):
        return torch.rand(*shape, generator=gen, device="cuda") * (hi - lo) + lo

    def decays(D):  # a_t between 0.9 and 0.999 where the recurrence gate is open
        a = uniform(D, lo=0.9, hi=0.999)
        return torch.log(torch.expm1(-torch.log(a) / C))

    st = {"case": case}
    if case["kind"] == "norm":
        rows, D = case["rows"], case["D"]
        st["x"] = normal(rows, D)
        st["residual"] = normal(rows, D, std=3.0) if case["residual"] else None
        st["weight"] = normal(D, std=0.2, mean=1.0, dtype=torch.float32)
        if case["train"]:
            st["dy"] = normal(rows, D)
            st["dsum"] = normal(rows, D)
    elif case["kind"] in ("scan", "step"):
        D = case["D"]
        lead = (case["T"], case["B"]) if case["kind"] == "scan" else (case["B"],)
        if case["fused"]:  # slices of one projection's output
            z = normal(*lead, 3 * D)
            z[..., D:2 * D] *= 1.5
            st["x"], st["r"], st["i"] = z[..., :D], z[..., D:2 * D], z[..., 2 * D:]
        else:
            st["x"], st["r"], st["i"] = normal(*lead, D), normal(*lead, D, std=1.5), normal(*lead, D)
        st["decay"] = decays(D)
        if case["kind"] == "step":
            n = case["pool"] or case["B"]
            st["state"] = normal(n, D, dtype=torch.float32)
            st["slots"] = None
            if case["pool"]:
                st["slots"] = torch.randperm(n, generator=gen, device="cuda")[:case["B"]].to(torch.int32)
        else:
            T, B = lead
            st["h0"] = normal(B, D, dtype=torch.float32) if case["state"] else None
            st["lengths"] = None
            if case["ragged"]:
                st["lengths"] = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
            st["reset"] = uniform(T, B) < case["resets"] if case["resets"] else None
            if case["train"]:
                st["dy"] = normal(T, B, D)
                st["dh_last"] = normal(B, D, dtype=torch.float32) if case["state"] else None
    else:
        M, N, K, G = case["M"], case["N"], case["K"], -(-case["K"] // case["group"])
        q = torch.randint(0, 16, (N, K), generator=gen, device="cuda", dtype=torch.uint8)
        st["q"] = _packed(q, -(-K // 32) * 16)
        st["scale"] = (uniform(N, G, lo=0.5, hi=1.5) / (4.0 * math.sqrt(K))).to(torch.float16)
        st["zero"] = torch.randint(6, 10, (N, G), generator=gen, device="cuda", dtype=torch.uint8)
        st["bias"] = normal(N, dtype=torch.float32) if case["bias"] else None
        st["x"], st["x_scale"] = normal(M, K), None
        if case["x8"]:
            x, gx = normal(M, K, dtype=torch.float32), -(-K // 128)
            pad = torch.nn.functional.pad(x, (0, gx * 128 - K)).reshape(M, gx, 128)
            st["x_scale"] = pad.abs().amax(2) / E4M3_MAX
            st["x"] = (pad / st["x_scale"][..., None]).reshape(M, -1)[:, :K].contiguous().to(E4M3)
        if own:
            from paper_1905_00689_gb300 import W4Weight
            st["w"] = W4Weight(st["q"], st["scale"], st["zero"], K, case["group"])
    return st


# ---------------------------------------------------------------------------
# one pass

def run(st):
    kind = st["case"]["kind"]
    if own:
        return {"norm": _own_norm, "scan": _own_scan, "step": _own_step, "w4": _own_w4}[kind](st)
    return {"norm": _plain_norm, "scan": _plain_scan, "step": _plain_step, "w4": _plain_w4}[kind](st)


def _own_norm(st):
    import paper_1905_00689_gb300 as g
    case = st["case"]
    if case["group"]:
        q, scale, total = g.rms_norm_quant(st["x"], st["weight"], st["residual"], eps=EPS, group=case["group"])
        return (q, scale, total) if case["residual"] else (q, scale)
    if not case["train"]:
        y, total = g.rms_norm(st["x"], st["weight"], st["residual"], eps=EPS)
        return (y, total) if case["residual"] else (y,)
    rstd = torch.empty(case["rows"], dtype=torch.float32, device="cuda")
    y, total = g.rms_norm(st["x"], st["weight"], st["residual"], eps=EPS, rstd=rstd)
    total = st["x"] if total is None else total
    dx, dw = g.rms_norm_backward(st["dy"], total, st["weight"], rstd, st["dsum"])
    return (y, total, dx, dw) if case["residual"] else (y, dx, dw)


def _own_scan(st):
    import paper_1905_00689_gb300 as g
    case = st["case"]
    x, more = st["x"], {"c": C, "lengths": st["lengths"], "reset": st["reset"]}
    if not case["train"]:
        return g.gated_scan(x, st["r"], st["i"], st["decay"], st["h0"], **more)
    states = g.gated_scan_states(*x.shape)
    y, last = g.gated_scan(x, st["r"], st["i"], st["decay"], st["h0"], states=states, **more)
    dx, dr, di, ddecay, dh0 = g.gated_scan_backward(st["dy"], x, st["r"], st["i"], st["decay"], states,
                                                    st["dh_last"], **more)
    out = (y, last, dx, dr, di, ddecay)
    return out + (dh0,) if case["state"] else out


def _own_step(st):
    import paper_1905_00689_gb300 as g
    y = g.gated_step(st["x"], st["r"], st["i"], st["decay"], st["state"], c=C, slots=st["slots"])
    return y, st["state"]


def _own_w4(st):
    import paper_1905_00689_gb300 as g
    return g.w4_matvec(st["x"], st["w"], x_scale=st["x_scale"], bias=st["bias"],
                       out_dtype=DTYPES[st["case"]["dtype"]])


def _plain_norm(st):
    case, dt = st["case"], st["x"].dtype
    s = st["x"].float()
    if case["residual"]:
        s = s + st["residual"].float()
    rstd = torch.rsqrt((s * s).mean(1, keepdim=True) + EPS)
    y = s * rstd * st["weight"]
    if case["group"]:
        rows, D, G = case["rows"], case["D"], case["group"]
        n = -(-D // G)
        pad = torch.nn.functional.pad(y, (0, n * G - D)).reshape(rows, n, G)
        amax = pad.abs().amax(2)
        scale = torch.where(amax == 0, torch.ones_like(amax), amax / E4M3_MAX)
        q = (pad / scale[..., None]).reshape(rows, n * G)[:, :D].contiguous().to(E4M3)
        return (q, scale, s.to(dt)) if case["residual"] else (q, scale)
    if not case["train"]:
        return (y.to(dt), s.to(dt)) if case["residual"] else (y.to(dt),)
    dy = st["dy"].float()
    wdy = dy * st["weight"]
    xhat = s * rstd
    dx = rstd * (wdy - xhat * (wdy * xhat).mean(1, keepdim=True)) + st["dsum"].float()
    dw = (dy * xhat).sum(0)
    return (y.to(dt), s.to(dt), dx.to(dt), dw) if case["residual"] else (y.to(dt), dx.to(dt), dw)


def _gates(x, r, i, decay):
    """sigma(r), sigma(i), log a, a and sqrt(1 - a^2) in 32 bits."""
    sr, si = torch.sigmoid(r.float()), torch.sigmoid(i.float())
    la = -C * torch.nn.functional.softplus(decay) * sr
    return x.float(), sr, si, la, torch.exp(la), torch.sqrt(-torch.expm1(2 * la))


def _linear_scan(A, U):
    """h_t = A_t h_{t-1} + U_t along the first axis, by doubling the span of each sum."""
    span, T = 1, U.shape[0]
    while span < T:
        U = torch.cat([U[:span], torch.addcmul(U[span:], A[span:], U[:-span])])
        A = torch.cat([A[:span], A[span:] * A[:-span]])
        span *= 2
    return U


def _plain_scan(st):
    case, dt = st["case"], st["x"].dtype
    T, B, D = st["x"].shape
    x, sr, si, la, a, m = _gates(st["x"], st["r"], st["i"], st["decay"])
    t = torch.arange(T, device="cuda")[:, None, None]
    live = None if st["lengths"] is None else t < st["lengths"][None, :, None]
    keep = a if st["reset"] is None else a.masked_fill(st["reset"][..., None], 0.0)
    h0 = st["h0"] if st["h0"] is not None else torch.zeros(B, D, device="cuda")
    u = m * si * x
    u[0] += keep[0] * h0
    h = _linear_scan(keep, u)
    y = h if live is None else h.masked_fill(~live, 0.0)
    if live is None:
        last = h[-1]
    else:
        at = (st["lengths"].long() - 1).clamp(min=0)
        last = torch.where(st["lengths"][:, None] > 0, h[at, torch.arange(B, device="cuda")], h0)
    if not case["train"]:
        return y.to(dt), last
    dy = st["dy"].float()
    carry = torch.cat([keep[1:], torch.zeros_like(keep[:1])])      # a_{t+1}
    if live is not None:
        dy = dy.masked_fill(~live, 0.0)
        carry = carry.masked_fill(t + 1 >= st["lengths"][None, :, None], 0.0)
    dh_last = st["dh_last"] if st["dh_last"] is not None else torch.zeros(B, D, device="cuda")
    n = torch.full((B,), T, device="cuda") if st["lengths"] is None else st["lengths"]
    dy = torch.where(t == n[None, :, None] - 1, dy + dh_last, dy)
    g = _linear_scan(carry.flip(0), dy.flip(0)).flip(0)
    before = torch.cat([h0[None], h[:-1]])
    q = torch.where(la == 0, torch.zeros_like(la), -la / m)
    e = g * (keep * la * before + si * x * a * a * q)
    if live is not None:
        e = e.masked_fill(~live, 0.0)
    ratio = torch.sigmoid(st["decay"]) / torch.nn.functional.softplus(st["decay"])
    dx, dr, di = g * m * si, e * (1 - sr), g * m * x * si * (1 - si)
    dh0 = torch.where(n[:, None] > 0, keep[0] * g[0], dh_last)
    out = (y.to(dt), last, dx.to(dt), dr.to(dt), di.to(dt), ratio * e.sum((0, 1)))
    return out + (dh0,) if case["state"] else out


def _plain_step(st):
    x, sr, si, la, a, m = _gates(st["x"], st["r"], st["i"], st["decay"])
    if st["slots"] is None:
        h = st["state"].mul_(a).add_(m * si * x)
    else:
        slots = st["slots"].long()
        h = a * st["state"][slots] + m * si * x
        st["state"][slots] = h
    return h.to(st["x"].dtype), st["state"]


def _plain_w4(st):
    case = st["case"]
    K, G = case["K"], case["group"]
    q = torch.stack([st["q"] & 15, st["q"] >> 4], 2).reshape(case["N"], -1)[:, :K].float()
    each = torch.arange(K, device="cuda") // G
    w = (q - st["zero"].float()[:, each]) * st["scale"].float()[:, each]
    x = st["x"].float()
    if case["x8"]:
        x = x * st["x_scale"][:, torch.arange(K, device="cuda") // 128]
    y = x @ w.t()
    if case["bias"]:
        y = y + st["bias"]
    return y.to(DTYPES[case["dtype"]])


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions

def exact(case, seed):
    st = prepare(case, seed)
    f64 = {k: v.double() if torch.is_tensor(v) and v.is_floating_point() or k == "x" else v for k, v in st.items()}
    return {"norm": _exact_norm, "scan": _exact_scan, "step": _exact_step, "w4": _exact_w4}[case["kind"]](case, f64)


def _exact_norm(case, st):
    s = st["x"] + st["residual"] if case["residual"] else st["x"]
    rms = (s.pow(2).sum(1) / case["D"] + EPS).sqrt()
    y = s / rms[:, None] * st["weight"]
    if case["group"]:
        q, scales = torch.empty_like(y), []
        for at in range(0, case["D"], case["group"]):
            part = y[:, at:at + case["group"]]
            scales.append(part.abs().max(1).values / E4M3_MAX)
            q[:, at:at + case["group"]] = part / scales[-1][:, None]
        return (q, torch.stack(scales, 1), s) if case["residual"] else (q, torch.stack(scales, 1))
    if not case["train"]:
        return (y, s) if case["residual"] else (y,)
    # y_j = w_j s_j / rms: dy_j/ds_k = w_j (delta_jk / rms - s_j s_k / (D rms^3))
    along = (st["dy"] * st["weight"] * s).sum(1)
    dx = st["dy"] * st["weight"] / rms[:, None] - s * (along / (case["D"] * rms.pow(3)))[:, None] + st["dsum"]
    dw = (st["dy"] * s / rms[:, None]).sum(0)
    return (y, s, dx, dw) if case["residual"] else (y, dx, dw)


def _exact_gates(x, r, i, decay):
    sr, si = 1 / (1 + torch.exp(-r)), 1 / (1 + torch.exp(-i))
    la = -C * torch.log1p(torch.exp(decay)) * sr
    return sr, si, la, torch.exp(la), torch.sqrt(-torch.expm1(2 * la))


def _exact_scan(case, st):
    T, B, D = case["T"], case["B"], case["D"]
    lengths = [T] * B if st["lengths"] is None else st["lengths"].tolist()
    zeros = torch.zeros(B, D, dtype=torch.float64, device="cuda")
    ends = torch.tensor(lengths, device="cuda")[:, None]
    h0 = zeros if st["h0"] is None else st["h0"]
    hs = torch.zeros(T + 1, B, D, dtype=torch.float64, device="cuda")
    hs[0] = h0

    def at(t):
        sr, si, la, a, m = _exact_gates(st["x"][t], st["r"][t], st["i"][t], st["decay"])
        return sr, si, la, a, m, None if st["reset"] is None else st["reset"][t][:, None]

    for t in range(T):
        sr, si, la, a, m, cut = at(t)
        before = hs[t] if cut is None else torch.where(cut, zeros, hs[t])
        hs[t + 1] = torch.where(ends > t, a * before + m * si * st["x"][t], hs[t])
    y = torch.where(torch.arange(T, device="cuda")[:, None, None] < ends[None], hs[1:], zeros[None])
    if not case["train"]:
        return y, hs[T]
    g = zeros if st["dh_last"] is None else st["dh_last"]
    dx, dr, di = (torch.zeros(T, B, D, dtype=torch.float64, device="cuda") for _ in range(3))
    dsp = torch.zeros(D, dtype=torch.float64, device="cuda")
    sp = torch.log1p(torch.exp(st["decay"]))
    for t in range(T - 1, -1, -1):
        sr, si, la, a, m, cut = at(t)
        live = ends > t
        g = torch.where(live, g + st["dy"][t], g)
        before = hs[t] if cut is None else torch.where(cut, zeros, hs[t])
        dla = torch.where(live, g * (before * a - si * st["x"][t] * a * a / m), zeros)
        dx[t] = torch.where(live, g * m * si, zeros)
        di[t] = torch.where(live, g * m * st["x"][t] * si * (1 - si), zeros)
        dr[t] = dla * -C * sp * sr * (1 - sr)
        dsp += (dla * -C * sr).sum(0)
        back = a * g if cut is None else torch.where(cut, zeros, a * g)
        g = torch.where(live, back, g)
    out = (y, hs[T], dx, dr, di, dsp / (1 + torch.exp(-st["decay"])))
    return out + (g,) if case["state"] else out


def _exact_step(case, st):
    sr, si, la, a, m = _exact_gates(st["x"], st["r"], st["i"], st["decay"])
    rows = torch.arange(case["B"], device="cuda") if st["slots"] is None else st["slots"].long()
    h = a * st["state"].index_select(0, rows) + m * si * st["x"]
    return h, st["state"].index_copy(0, rows, h)


def _exact_w4(case, st):
    N, K, G = case["N"], case["K"], case["group"]
    x = st["x"]
    y = torch.zeros(case["M"], N, dtype=torch.float64, device="cuda")
    for g, at in enumerate(range(0, K, G)):
        to = min(K, at + G)
        cols = torch.arange(at, to, device="cuda")
        q = (st["q"][:, cols // 2] >> (4 * (cols % 2)).to(torch.uint8)) & 15
        part = (q.double() - st["zero"][:, g, None].double()) * st["scale"][:, g, None]
        xs = x[:, at:to] if not case["x8"] else x[:, at:to] * st["x_scale"][:, cols // 128]
        y += xs @ part.t()
    return y if st["bias"] is None else y + st["bias"]
