"""A recurrence with matrix states (the gated delta rule) and the AdamW step
that trains a model of it, as plain cases.

- delta: for every stream and head a state S [Dk, Dv],

      u_t = beta_t (v_t - e^{g_t} S_{t-1}^T k_t)
      S_t = e^{g_t} S_{t-1} + k_t u_t^T;   o_t = scale S_t^T q_t

  over a sequence, with resets (packed documents), lengths (ragged batches),
  first states and value heads that share query and key heads; its backward pass;
- delta_step: one timestep of it on a pool of states;
- adamw: one update of many tensors at once, with its two moving averages in 32
  bits, or in 8 bits (e4m3, a scale for each 256 values, rounded at random).

Sequences are time-major, [T][B][H][D], as everywhere in this package.  The
plain forms below are elementary torch operations in 32 bits, rounded once at
the end.  The plain delta rule goes by chunks of 64 timesteps: inside a chunk
the u_t solve a triangular system, between chunks the state is carried on.
"""
import math

import torch

own = False

CHUNK = 64
BLOCK = 256        # values to a scale of the 8-bit averages
BETAS, EPS, DECAY, RATE = (0.9, 0.999), 1e-8, 0.1, 3e-4
DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
E4M3 = torch.float8_e4m3fn
E4M3_MAX = 448.0


# ---------------------------------------------------------------------------
# cases

def _delta(name, dtype, T, B, H, Hk, Dk, Dv, train=False, ragged=False, resets=0.0, state=False, fused=False):
    return {"name": name, "kind": "delta", "dtype": dtype, "T": T, "B": B, "H": H, "Hk": Hk, "Dk": Dk, "Dv": Dv,
            "train": train, "ragged": ragged, "resets": resets, "state": state, "fused": fused}


def _step(name, dtype, B, H, Hk, Dk, Dv, pool=0, fused=False):
    return {"name": name, "kind": "step", "dtype": dtype, "B": B, "H": H, "Hk": Hk, "Dk": Dk, "Dv": Dv, "pool": pool,
            "fused": fused}


def _adamw(name, dtype, gdtype, layers, D, bits, copies=False, clip=False, apart=0):
    return {"name": name, "kind": "adamw", "dtype": dtype, "gdtype": gdtype, "layers": layers, "D": D, "bits": bits,
            "copies": copies, "clip": clip, "apart": apart}


def listed():
    return [
        # the prompt of one stream, an odd length, q, k and v as slices of one projection's output
        _delta("delta-prompt", "bf16", 8191, 1, 16, 16, 128, 128, fused=True),
        # prompts of unlike lengths, padded, resumed from states; value heads share key heads
        _delta("delta-ragged", "fp16", 700, 13, 6, 3, 64, 100, ragged=True, state=True),
        # a short prompt of a small model
        _delta("delta-short", "bf16", 100, 2, 4, 4, 64, 64),
        # a training step (forward and backward) on packed documents
        _delta("delta-train", "bf16", 2048, 4, 8, 8, 128, 128, train=True, resets=1 / 500),
        # a training step on a long sequence in 32 bits, odd widths, shared key heads
        _delta("delta-train-odd", "fp32", 4001, 1, 6, 2, 48, 80, train=True, state=True),
        # one token of one stream
        _step("delta-step-one", "bf16", 1, 16, 16, 128, 128),
        # one token for each of 64 streams whose states lie scattered in a pool, slices of one projection's output
        _step("delta-step-pool", "bf16", 64, 16, 8, 128, 128, pool=100, fused=True),
        # odd widths in 32 bits
        _step("delta-step-odd", "fp32", 33, 5, 5, 72, 100),
        # one block of a small model in 32 bits
        _adamw("adamw-block", "fp32", "fp32", 1, 512, 32),
        # a model of 24 blocks: 32-bit parameters, 16-bit gradients, clipped, and the 16-bit copies that the next step computes with
        _adamw("adamw-model", "fp32", "bf16", 24, 2048, 32, copies=True, clip=True),
        # the same model with the averages in 8 bits
        _adamw("adamw-model-8bit", "fp32", "bf16", 24, 2048, 8, copies=True, clip=True),
        # 40 blocks of odd width in 16 bits, tensors one after the other at any address
        _adamw("adamw-odd-8bit", "bf16", "bf16", 40, 333, 8, apart=1),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(("delta", "delta", "delta", "step", "adamw", "adamw"))
    dtype = rng.choice(("bf16", "bf16", "fp16", "fp32"))
    if kind == "adamw":
        D = _log(rng, 32, 2048)
        if rng.random() < 0.6:
            D = max(32, D // 32 * 32)
        layers = _log(rng, 1, max(1, min(100, 100_000_000 // (3 * D * D))))
        case = _adamw("", dtype, dtype if dtype != "fp32" else rng.choice(("fp32", "bf16")), layers, D, rng.choice((8, 32)),
                      copies=dtype == "fp32" and rng.random() < 0.5, clip=rng.random() < 0.5, apart=rng.choice((0, 0, 1)))
    else:
        Dk, Dv = rng.choice((32, 64, 64, 96, 128, 128)), rng.choice((32, 64, 64, 128, 128, 192))
        if rng.random() < 0.3:
            Dk, Dv = rng.randint(8, 128), rng.randint(8, 200)
        Hk = _log(rng, 1, 16)
        H = Hk * rng.choice((1, 1, 2, 3)) if Hk <= 8 else Hk
        if kind == "step":
            B = _log(rng, 1, max(1, min(512, 16_000_000 // (H * Dk * Dv))))
            case = _step("", dtype, B, H, Hk, Dk, Dv, pool=rng.choice((0, B + _log(rng, 1, 100))), fused=rng.random() < 0.5)
        else:
            B = _log(rng, 1, 16)
            train = rng.random() < 0.5
            most = (2_000_000 if train else 4_000_000) // (B * H)    # values of one channel
            T = _log(rng, 1, max(2, min(3000 if train else 8000, most * 4 // (Dk + Dv))))
            case = _delta("", dtype, T, B, H, Hk, Dk, Dv, train=train, ragged=rng.random() < 0.3,
                          resets=rng.choice((0.0, 0.0, 0.002, 0.05)), state=rng.random() < 0.5, fused=rng.random() < 0.5)
    del case["name"]
    return case


def _sizes(case):
    """Of the tensors of an adamw case: each block has a norm's weight, a projection and decays."""
    D = case["D"]
    return [n for _ in range(case["layers"]) for n in (D, 3 * D * D, D)]


def work(case):
    e = 4 if case["dtype"] == "fp32" else 2
    if case["kind"] == "adamw":
        n = sum(_sizes(case))
        each = 2 * e + (4 if case["gdtype"] == "fp32" else 2) + (2 if case["copies"] else 0)
        each += 16 if case["bits"] == 32 else 4 + 16 / BLOCK
        return {"bytes": n * each, "flops": 16 * n}
    H, Hk, Dk, Dv = case["H"], case["Hk"], case["Dk"], case["Dv"]
    n = case["B"] * (case["T"] if case["kind"] == "delta" else 1)
    values = n * (2 * Hk * Dk + 2 * H * Dv) * e + n * H * 8
    states = case["B"] * H * Dk * Dv * 4
    flops = 7 * n * H * Dk * Dv
    if case["kind"] == "step":
        return {"bytes": values + 2 * states + (4 * case["B"] if case["pool"] else 0), "flops": flops}
    small = (n if case["resets"] else 0) + (4 * case["B"] if case["ragged"] else 0)
    moved = values + states * (2 if case["state"] else 1) + small
    if case["train"]:  # reads do and the last state's gradient as well, writes the inputs' gradients
        moved += n * (2 * Hk * Dk + 2 * H * Dv) * e + n * H * 8 + (2 * states if case["state"] else 0)
        flops *= 3
    return {"bytes": moved, "flops": flops}


# ---------------------------------------------------------------------------
# inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0, dtype=dt):
        return (torch.randn(*shape, generator=gen, device="cuda") * std + mean).to(dtype)

    def uniform(*shape, lo=0.0, hi=1.0):
        return torch.rand(*shape, generator=gen, device="cuda") * (hi - lo) + lo

    st = {"case": case}
    if case["kind"] == "adamw":
        # tensors are views of one allocation for each purpose, 16 bytes apart or one after the other
        sizes, at, where = _sizes(case), 0, []
        for n in sizes:
            where.append(at)
            at += n + case["apart"] if case["apart"] else -(-n // 16) * 16
        blocks = [-(-n // BLOCK) for n in sizes]

        def views(flat):
            return [flat[a:a + n] for a, n in zip(where, sizes)]

        st["flat"] = {"p": normal(at, std=0.02), "g": normal(at, std=1e-3, dtype=DTYPES[case["gdtype"]])}
        if case["bits"] == 32:
            st["flat"]["m"] = normal(at, std=3e-4, dtype=torch.float32)
            st["flat"]["v"] = normal(at, std=1e-3, dtype=torch.float32).square()
        else:
            st["flat"]["m"] = normal(at, std=100.0, dtype=torch.float32).clamp(-E4M3_MAX, E4M3_MAX).to(E4M3)
            st["flat"]["v"] = normal(at, std=100.0, dtype=torch.float32).abs().clamp(2 ** -9, E4M3_MAX).to(E4M3)
            st["flat"]["ms"], st["flat"]["vs"] = uniform(sum(blocks), lo=2e-6, hi=4e-6), uniform(sum(blocks), lo=5e-6, hi=2e-5)
            st["ms"], st["vs"] = (list(st["flat"][k].split(blocks)) for k in ("ms", "vs"))
        if case["copies"]:
            st["flat"]["c"] = torch.zeros(at, dtype=torch.bfloat16, device="cuda")
        for k in ("p", "g", "m", "v", "c"):
            if k in st["flat"]:
                st[k] = views(st["flat"][k])
        st["clip"] = uniform(1, lo=0.3, hi=1.0) if case["clip"] else None
        st["t"] = 100
        if own:
            from paper_1905_00689_gb300 import AdamWState
            st["state"] = AdamWState(st["m"], st["v"], st.get("ms"), st.get("vs"))
        return st

    H, Hk, Dk, Dv = case["H"], case["Hk"], case["Dk"], case["Dv"]
    lead = (case["T"], case["B"]) if case["kind"] == "delta" else (case["B"],)
    if case["fused"]:  # slices of one projection's output; keys and queries get their norm in place, as a program has them
        z = normal(*lead, 2 * Hk * Dk + H * Dv)
        q, k, v = z.split((Hk * Dk, Hk * Dk, H * Dv), -1)
        q, k, v = q.unflatten(-1, (Hk, Dk)), k.unflatten(-1, (Hk, Dk)), v.unflatten(-1, (H, Dv))
    else:
        q, k, v = normal(*lead, Hk, Dk), normal(*lead, Hk, Dk), normal(*lead, H, Dv)
    for t in (q, k):
        t.copy_(t.float() / t.float().norm(dim=-1, keepdim=True))
    st["q"], st["k"], st["v"] = q, k, v
    # heads that forget after some tens to some thousands of timesteps
    rate = torch.exp(uniform(H, lo=math.log(1e-3), hi=math.log(0.2)))
    st["g"] = -rate * torch.nn.functional.softplus(normal(*lead, H, dtype=torch.float32) + 1.0)
    st["beta"] = torch.sigmoid(normal(*lead, H, dtype=torch.float32))
    if case["kind"] == "step":
        n = case["pool"] or case["B"]
        st["state"] = normal(n, H, Dk, Dv, std=0.3, dtype=torch.float32)
        st["slots"] = None
        if case["pool"]:
            st["slots"] = torch.randperm(n, generator=gen, device="cuda")[:case["B"]].to(torch.int32)
        return st
    T, B = lead
    st["h0"] = normal(B, H, Dk, Dv, std=0.3, dtype=torch.float32) if case["state"] else None
    st["lengths"] = None
    if case["ragged"]:
        st["lengths"] = torch.randint(0, T + 1, (B,), generator=gen, device="cuda", dtype=torch.int32)
    st["reset"] = uniform(T, B) < case["resets"] if case["resets"] else None
    if case["train"]:
        st["do"] = normal(T, B, H, Dv)
        st["dh_last"] = normal(B, H, Dk, Dv, std=0.1, dtype=torch.float32) if case["state"] else None
    return st


# ---------------------------------------------------------------------------
# one pass

def run(st):
    kind = st["case"]["kind"]
    if own:
        return {"delta": _own_delta, "step": _own_step, "adamw": _own_adamw}[kind](st)
    return {"delta": _plain_delta, "step": _plain_step, "adamw": _plain_adamw}[kind](st)


def _own_delta(st):
    import paper_1905_00689_gb300 as g
    case = st["case"]
    q, k, v, more = st["q"], st["k"], st["v"], {"lengths": st["lengths"], "reset": st["reset"]}
    if not case["train"]:
        return g.delta_scan(q, k, v, st["g"], st["beta"], st["h0"], **more)
    states = g.delta_scan_states(q, v)
    o, last = g.delta_scan(q, k, v, st["g"], st["beta"], st["h0"], states=states, **more)
    grads = g.delta_scan_backward(st["do"], q, k, v, st["g"], st["beta"], states, st["dh_last"], **more)
    return (o, last) + (tuple(grads) if case["state"] else tuple(grads)[:5])


def _own_step(st):
    import paper_1905_00689_gb300 as g
    o = g.delta_step(st["q"], st["k"], st["v"], st["g"], st["beta"], st["state"], slots=st["slots"])
    return o, st["state"]


def _own_adamw(st):
    import paper_1905_00689_gb300 as g
    st["t"] += 1
    g.adamw_step(st["p"], st["g"], st["state"], st["t"], lr=RATE, betas=BETAS, eps=EPS, weight_decay=DECAY,
                 copies=st.get("c"), grad_scale=st["clip"], seed=7)
    return {k: t for k, t in st["flat"].items() if k != "g"}


def _spread(x, H):
    """[..., Hk, D] in 32 bits, each head as often as value heads share it: [..., H, D]."""
    return x.float().repeat_interleave(H // x.shape[-2], -2)


def _plain_delta(st):
    """Chunk by chunk; x with a bar is x of a whole chunk.  i, j: rows (timesteps) of a chunk."""
    case, dt = st["case"], st["q"].dtype
    T, B, H, Hk, Dk, Dv = (case[x] for x in ("T", "B", "H", "Hk", "Dk", "Dv"))
    N, C = -(-T // CHUNK), CHUNK
    scale = Dk ** -0.5
    t = torch.arange(N * C, device="cuda")
    live = (t[:, None] < (torch.full((B,), T, device="cuda") if st["lengths"] is None else st["lengths"])[None]) & (t < T)[:, None]

    def chunks(x):  # [T, B, H, ...] as [N, B, H, C, ...]; nothing past a stream's length
        x = torch.nn.functional.pad(x.float(), (0, 0) * (x.dim() - 1) + (0, N * C - T))
        x = x.masked_fill(~live[(...,) + (None,) * (x.dim() - 2)], 0.0)
        return x.unflatten(0, (N, C)).movedim(1, 3)

    def whole(x):   # and back
        return x.movedim(3, 1).flatten(0, 1)[:T]

    q, k, v = chunks(_spread(st["q"], H)), chunks(_spread(st["k"], H)), chunks(st["v"])
    g, beta = chunks(st["g"]).double().cumsum(-1), chunks(st["beta"])
    cut = torch.zeros(N * C, B, dtype=torch.bool, device="cuda")
    if st["reset"] is not None:
        cut[:T] = st["reset"]
    docs = (cut & live).unflatten(0, (N, C)).movedim(1, 2).cumsum(-1)[:, :, None]    # [N, B, 1, C]: resets up to here
    at = torch.arange(C, device="cuda")
    D = torch.exp(torch.where((at[:, None] >= at) & (docs[..., :, None] == docs[..., None, :]),
                              g[..., :, None] - g[..., None, :], -torch.inf)).float()
    strict = D * (at[:, None] > at)
    gam = torch.exp(g).float() * (docs == 0)                      # decay of the chunk's first state up to row i
    dec = torch.exp(g[..., -1:] - g).float() * (docs == docs[..., -1:])    # decay from row j to the chunk's end
    gend = gam[..., -1]
    kk, qk = k @ k.mT, q @ k.mT
    P = -beta[..., None] * strict * kk
    inv = P + torch.eye(C, device="cuda")                         # (I - P)^-1 = (I + P) (I + P^2) (I + P^4) ...
    for _ in range(5):
        P = P @ P
        inv = inv + P @ inv
    M = D * qk
    S = st["h0"] if st["h0"] is not None else torch.zeros(B, H, Dk, Dv, device="cuda")
    starts, us, os = [], [], []
    for n in range(N):
        starts.append(S)
        X = v[n] - gam[n][..., None] * (k[n] @ S)
        U = inv[n] @ (beta[n][..., None] * X)
        os.append(scale * (gam[n][..., None] * (q[n] @ S) + M[n] @ U))
        S = gend[n][..., None, None] * S + (dec[n][..., None] * k[n]).mT @ U
        us.append(U)
    last = S
    o = whole(torch.stack(os)).masked_fill(~live[:T, :, None, None], 0.0).to(dt)
    if not case["train"]:
        return o, last
    do, U, S0 = chunks(st["do"]), torch.stack(us), torch.stack(starts)
    dS = st["dh_last"] if st["dh_last"] is not None else torch.zeros(B, H, Dk, Dv, device="cuda")
    local = scale * (M.mT @ do)
    ends, rs = [None] * N, [None] * N
    for n in range(N - 1, -1, -1):
        ends[n] = dS
        rs[n] = inv[n].mT @ (local[n] + dec[n][..., None] * (k[n] @ dS))
        dS = gend[n][..., None, None] * dS + q[n].mT @ (scale * gam[n][..., None] * do[n])
        dS = dS - k[n].mT @ ((beta[n] * gam[n])[..., None] * rs[n])
    dS1, R = torch.stack(ends), torch.stack(rs)
    X = v - gam[..., None] * (k @ S0)
    dP = scale * D * (do @ U.mT)
    ru = strict * (R @ U.mT)
    dB = -beta[..., None] * ru
    dbeta = (R * X).sum(-1) - (ru * kk).sum(-1)
    dq = dP @ k + scale * gam[..., None] * (do @ S0.mT)
    t1 = dB @ k - (beta * gam)[..., None] * (R @ S0.mT)
    far = dec[..., None] * (U @ dS1.mT)
    t2 = dP.mT @ q + dB.mT @ k + far
    dG = (q * dq).sum(-1) + (k * (t1 - t2)).sum(-1)
    dG[..., -1] += gend * (dS1 * S0).sum((-1, -2)) + (k * far).sum((-1, -2))
    dg = dG.flip(-1).cumsum(-1).flip(-1)

    def shared(x):  # summed over the value heads of each key head
        return whole(x).unflatten(2, (Hk, H // Hk)).sum(3).masked_fill(~live[:T, :, None, None], 0.0).to(dt)

    dv = (whole(beta[..., None] * R).masked_fill(~live[:T, :, None, None], 0.0)).to(dt)
    none = ~live[:T, :, None]
    out = (o, last, shared(dq), shared(t1 + t2), dv, whole(dg).masked_fill(none, 0.0), whole(dbeta).masked_fill(none, 0.0))
    return out + (dS,) if case["state"] else out


def _plain_step(st):
    H = st["v"].shape[1]
    q, k, v = _spread(st["q"], H), _spread(st["k"], H), st["v"].float()
    S = st["state"] if st["slots"] is None else st["state"][st["slots"].long()]
    S = S * torch.exp(st["g"])[..., None, None]
    u = st["beta"][..., None] * (v - (S * k[..., None]).sum(-2))
    S = S + k[..., None] * u[..., None, :]
    o = q.shape[-1] ** -0.5 * (S * q[..., None]).sum(-2)
    if st["slots"] is None:
        st["state"].copy_(S)
    else:
        st["state"][st["slots"].long()] = S
    return o.to(st["q"].dtype), st["state"]


def _mix(h):
    """A hash of 32 bits, in whole numbers of 64.  The factors are the odd numbers next to 2^32 / 1.618... and to the
    fraction of e = 2.718..."""
    h = h ^ (h >> 16)
    h = (h * 0x9E3779B1) & 0xFFFFFFFF
    h = h ^ (h >> 13)
    h = (h * 0xB7E15163) & 0xFFFFFFFF
    return h ^ (h >> 16)


def _chance(seed, step, first, n):
    """32 random bits for each of n values of a tensor whose first is the `first`-th of all."""
    at = torch.arange(first, first + n, device="cuda")
    key = _mix(_mix((seed + 1) & 0xFFFFFFFF) ^ step)
    return _mix(((at & 0xFFFFFFFF) + (key ^ (at >> 32))) & 0xFFFFFFFF)


def _to_e4m3(x, bits16):
    """x in [0, 448] to a neighbouring e4m3 value: the upper one with the chance of where x lies between them."""
    small = x < 2 ** -6
    b = torch.where(small, x + 2 ** -6, x).view(torch.int32)
    b = (b + (bits16 << 4).to(torch.int32) + 8) & ~0xFFFFF
    y = b.view(torch.float32)
    return torch.where(small, y - 2 ** -6, y).clamp(max=E4M3_MAX)


def _blocks(x):
    return torch.nn.functional.pad(x, (0, -x.numel() % BLOCK)).view(-1, BLOCK)


def _plain_adamw(st):
    st["t"] += 1
    t, (b1, b2), first = st["t"], BETAS, 0
    far1, far2 = 1 - b1 ** t, 1 - b2 ** t
    for n, p in enumerate(st["p"]):
        g, w = st["g"][n].float(), p.float()
        if st["clip"] is not None:
            g = g * st["clip"]
        m, v, size = st["m"][n], st["v"][n], p.numel()
        if st["case"]["bits"] == 8:
            ms, vs = st["ms"][n], st["vs"][n]
            m = (_blocks(m.float()) * ms[:, None]).view(-1)[:size]
            v = (_blocks(v.float()) * vs[:, None]).view(-1)[:size].square()
        m = m * b1 + g * (1 - b1)
        v = v * b2 + g * g * (1 - b2)
        u = torch.sqrt(v)
        w = w * (1 - RATE * DECAY) - (RATE / far1) * m / (u / math.sqrt(far2) + EPS)
        p.copy_(w.to(p.dtype))
        if "c" in st:
            st["c"][n].copy_(w.to(torch.bfloat16))
        if st["case"]["bits"] == 32:
            st["m"][n].copy_(m)
            st["v"][n].copy_(v)
            continue
        chance = _chance(7, t, first, size)
        first += size
        for x, bits, q, s in ((m, chance & 0xFFFF, st["m"][n], ms), (u, chance >> 16, st["v"][n], vs)):
            s.copy_((_blocks(x.abs()).amax(1) / E4M3_MAX).clamp(min=2 ** -126))
            y = _blocks(x.abs()) * (1 / s)[:, None]
            y = _to_e4m3(y.view(-1)[:size].clamp(max=E4M3_MAX), bits)
            y = torch.copysign(y, x) if x is m else torch.where(x > 0, y.clamp(min=2 ** -9), y)
            q.copy_(y.to(E4M3))
    return {k: x for k, x in st["flat"].items() if k != "g"}


# ---------------------------------------------------------------------------
# the same in 64 bits, from the definitions

def exact(case, seed):
    st = prepare(case, seed)
    return {"delta": _exact_delta, "step": _exact_step, "adamw": _exact_adamw}[case["kind"]](case, st)


def _exact_delta(case, st):
    """Timestep by timestep; the gradients by the chain rule, from the end."""
    T, B, H, Hk, Dk, Dv = (case[x] for x in ("T", "B", "H", "Hk", "Dk", "Dv"))
    if case["train"] and T * B * H * Dk * Dv > 2 ** 32:
        return None
    share = torch.arange(H, device="cuda") // (H // Hk)
    q, k, v, g, beta = (st[x].double() for x in ("q", "k", "v", "g", "beta"))
    n = torch.full((B,), T, device="cuda") if st["lengths"] is None else st["lengths"]
    zero = torch.zeros(B, H, Dk, Dv, dtype=torch.float64, device="cuda")
    S = zero if st["h0"] is None else st["h0"].double()
    o = torch.zeros(T, B, H, Dv, dtype=torch.float64, device="cuda")
    kept = torch.empty(T + 1, B, H, Dk, Dv, dtype=torch.float64, device="cuda") if case["train"] else None
    scale = 1 / math.sqrt(Dk)

    def before(S, t):  # what the state counts as at timestep t, decayed
        if st["reset"] is not None:
            S = torch.where(st["reset"][t][:, None, None, None], zero, S)
        return S * g[t].exp()[..., None, None]

    def at(t):
        return q[t][:, share], k[t][:, share], (n > t)[:, None, None]

    for t in range(T):
        if kept is not None:
            kept[t] = S
        qt, kt, live = at(t)
        W = before(S, t)
        u = beta[t][..., None] * (v[t] - torch.einsum("bhkv,bhk->bhv", W, kt))
        new = W + torch.einsum("bhk,bhv->bhkv", kt, u)
        S = torch.where(live[..., None], new, S)
        o[t] = torch.where(live, scale * torch.einsum("bhkv,bhk->bhv", new, qt), o[t])
    if not case["train"]:
        return o, S
    last = S
    dS = zero if st["dh_last"] is None else st["dh_last"].double()
    dq, dk, dv, dg, dbeta = (torch.zeros_like(x) for x in (q, k, v, g, beta))
    do = st["do"].double()
    for t in range(T - 1, -1, -1):
        qt, kt, live = at(t)
        W = before(kept[t], t)
        r = v[t] - torch.einsum("bhkv,bhk->bhv", W, kt)
        u = beta[t][..., None] * r
        S = W + torch.einsum("bhk,bhv->bhkv", kt, u)
        dot = torch.where(live, do[t], torch.zeros_like(do[t]))
        dqt = scale * torch.einsum("bhkv,bhv->bhk", S, dot)
        G = dS + scale * torch.einsum("bhk,bhv->bhkv", qt, dot)
        du = torch.einsum("bhkv,bhk->bhv", G, kt)
        dr = beta[t][..., None] * du
        dkt = torch.einsum("bhkv,bhv->bhk", G, u) - torch.einsum("bhkv,bhv->bhk", W, dr)
        dW = G - torch.einsum("bhk,bhv->bhkv", kt, dr)
        for into, x in ((dq, dqt), (dk, dkt)):
            into[t] = torch.where(live, x, torch.zeros_like(x)).unflatten(1, (Hk, H // Hk)).sum(2)
        dv[t] = torch.where(live, dr, dv[t])
        dbeta[t] = torch.where(live[..., 0], (du * r).sum(-1), dbeta[t])
        dg[t] = torch.where(live[..., 0], (dW * W).sum((-1, -2)), dg[t])
        dS = torch.where(live[..., None], before(dW, t), dS)
    out = (o, last, dq, dk, dv, dg, dbeta)
    return out + (dS,) if case["state"] else out


def _exact_step(case, st):
    share = torch.arange(case["H"], device="cuda") // (case["H"] // case["Hk"])
    q, k, v, g, beta, state = (st[x].double() for x in ("q", "k", "v", "g", "beta", "state"))
    rows = torch.arange(case["B"], device="cuda") if st["slots"] is None else st["slots"].long()
    W = state.index_select(0, rows) * g.exp()[..., None, None]
    u = beta[..., None] * (v - torch.einsum("bhkv,bhk->bhv", W, k[:, share]))
    S = W + torch.einsum("bhk,bhv->bhkv", k[:, share], u)
    o = torch.einsum("bhkv,bhk->bhv", S, q[:, share]) / math.sqrt(case["Dk"])
    return o, state.index_copy(0, rows, S)


def _exact_adamw(case, st):
    """The parameters and 32-bit averages; the 8-bit ones are rounded at random."""
    flat = {k: x.clone() if k in ("p", "m", "v") and case["bits"] == 32 else x for k, x in st["flat"].items()}
    out = {k: flat[k].double() for k in ("p", "m", "v")}
    if "c" in flat:
        out["c"] = flat["c"].double()
    clip = 1.0 if st["clip"] is None else st["clip"].double()
    start = st["p"][0].storage_offset()
    for n, p in enumerate(st["p"]):
        at = slice(p.storage_offset() - start, p.storage_offset() - start + p.numel())
        g = st["g"][n].double() * clip
        if case["bits"] == 8:
            each = torch.arange(p.numel(), device="cuda") // BLOCK
            m, v = st["m"][n].double() * st["ms"][n].double()[each], (st["v"][n].double() * st["vs"][n].double()[each]) ** 2
        else:
            m, v = st["m"][n].double(), st["v"][n].double()
        m = BETAS[0] * m + (1 - BETAS[0]) * g
        v = BETAS[1] * v + (1 - BETAS[1]) * g ** 2
        step = (m / (1 - BETAS[0] ** 101)) / ((v / (1 - BETAS[1] ** 101)).sqrt() + EPS)
        out["p"][at] = p.double() - RATE * (DECAY * p.double() + step)
        out["m"][at], out["v"][at] = m, v
        if "c" in out:
            out["c"][at] = out["p"][at]
    if case["bits"] == 8:
        out.update(m=None, v=None, ms=None, vs=None)
    return out
