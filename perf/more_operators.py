"""The operators of a block that learns by the gated delta rule: the rule itself over packed sequences, the gated norm of its heads, and the norms before and
after the block with its gate and the residual's scale; for training steps, for prompts and for single tokens.

A case is one operator with everything that its descriptor takes.  `op` names the operator ("delta", "heads", "block"), `does` what the program runs: "fwd"
(inference), "bwd" (the backward pass), "train" (forward and backward pass) or "step" (one new token of each row, the carried states updated in place).
Tokens are packed: T of them in `sequences` sequences, of equal lengths or, where `ragged`, of any (one of them empty).
"""
import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


# ---- the cases -------------------------------------------------------------------------------------------------

def _delta(name, does, T, Hk, H, K, V, dtype, sequences=1, ragged=False, carry=False, wide=False, unit=False):
    """Hk key heads, each shared by H / Hk value heads; states of K x V a value head.  carry: the sequences continue earlier ones, whose states are given and
    whose new ones come back.  wide: q, k and v are parts of the convolution's rows, a and b of a projection's.  unit: q and k come with length one and are
    not normalised by the call.  A step has T rows whose states lie in 2 T slots, in any order."""
    return {"name": name, "op": "delta", "does": does, "T": T, "Hk": Hk, "H": H, "K": K, "V": V, "dtype": dtype, "sequences": sequences,
            "ragged": ragged, "carry": carry, "wide": wide, "unit": unit}


def _heads(name, does, T, H, D, dtype, gate=True, wide=False):
    """wide: the gate is one half of a projection's rows."""
    return {"name": name, "op": "heads", "does": does, "T": T, "H": H, "D": D, "dtype": dtype, "gate": gate, "wide": wide}


def _block(name, does, T, C, dtype, post=True, gate=False, scale=False, residual=True, pre=True):
    """post: the block's output is normalised; gate: and gated; scale: a factor for each channel; residual: what it is added to; pre: the sum is normalised
    for the next block."""
    return {"name": name, "op": "block", "does": does, "T": T, "C": C, "dtype": dtype, "post": post, "gate": gate, "scale": scale,
            "residual": residual, "pre": pre}


def listed():
    return [
        # generation: one token of 64 rows, whose states are most of what moves
        _delta("delta_tokens", "step", 64, 4, 8, 128, 128, "bf16", wide=True),
        # one short prompt, small heads: latency
        _delta("delta_short_prompt", "fwd", 301, 8, 8, 64, 64, "bf16"),
        # a long prompt alone on the card, that continues an earlier one
        _delta("delta_long_prompt", "fwd", 16384, 8, 16, 128, 128, "bf16", carry=True, wide=True),
        # many prompts, packed, of any lengths
        _delta("delta_prompts", "fwd", 16383, 16, 16, 64, 128, "bf16", sequences=24, ragged=True, wide=True),
        # a training step, bf16
        _delta("delta_training", "train", 8192, 8, 8, 128, 128, "bf16", sequences=8, wide=True),
        # a small training step in fp32: heads that are no multiple of a tile, shared keys, packed
        _delta("delta_training_odd", "train", 1501, 3, 6, 40, 56, "f32", sequences=5, ragged=True),
        # the heads of a few new tokens in generation: the latency of one small call
        _heads("heads_tokens", "fwd", 64, 16, 128, "bf16", wide=True),
        # the heads of a training batch, backward
        _heads("heads_gradients", "bwd", 16384, 8, 128, "bf16", wide=True),
        # heads of an odd width in fp32, without a gate
        _heads("heads_odd", "fwd", 9999, 12, 100, "f32", gate=False),
        # a few new tokens between two blocks, all parts of it
        _block("block_tokens", "fwd", 8, 1024, "bf16", gate=True, scale=True),
        # a long prompt or a training batch between two blocks
        _block("block_batch", "fwd", 32768, 1024, "bf16", scale=True),
        # the backward pass of a training step, all parts of it: a row count that is no multiple of anything
        _block("block_gradients", "bwd", 9999, 1536, "bf16", gate=True, scale=True),
    ]


def _between(rng, least, most):
    return int(round(math.exp(rng.uniform(math.log(least), math.log(most)))))


def draw(rng):
    """One case of the listed ones' ranges: 1 to 32768 tokens, 1 to 16 heads of 16 to 256 by 16 to 256 (odd ones among them), 1 to 64 sequences, 32 to 2048 channels, both
    types, each direction; at most what the largest listed case of its kind has."""
    op = rng.choice(["delta", "delta", "heads", "block"])
    does = rng.choice({"delta": ["fwd", "train", "step"], "heads": ["fwd", "bwd"], "block": ["fwd", "bwd"]}[op])
    dtype = rng.choice(sorted(TORCH))
    if op == "delta":
        sizes = [_between(rng, 16, 256) for _ in range(2)]
        if rng.random() < 0.6:
            sizes = [rng.choice([32, 64, 64, 128, 128, 256]) for _ in range(2)]
        K, V = sizes
        H = _between(rng, 1, 16)
        Hk = rng.choice([n for n in range(1, H + 1) if H % n == 0 and n * 4 >= H])
        cells = H * K * V
        if does == "step":
            T = max(1, min(_between(rng, 1, 128), (1 << 23) // cells))
            case = _delta("", does, T, Hk, H, K, V, dtype, wide=rng.random() < 0.5, unit=rng.random() < 0.2)
        else:
            T = _between(rng, 1, 16384)
            T = max(1, min(T, ((1 << 32) if does == "fwd" else (1 << 30)) // cells // (1 if dtype == "bf16" else 4)))
            sequences, ragged = 1, False
            if rng.random() < 0.7:
                sequences = _between(rng, 1, min(64, T))
                ragged = rng.random() < 0.6
            if not ragged:
                T = T // sequences * sequences
            case = _delta("", does, T, Hk, H, K, V, dtype, sequences, ragged, does == "fwd" and rng.random() < 0.5, rng.random() < 0.5,
                          rng.random() < 0.2)
    elif op == "heads":
        H = _between(rng, 1, 32)
        D = rng.choice([32, 64, 128, 128, 256]) if rng.random() < 0.6 else _between(rng, 16, 256)
        T = max(1, min(_between(rng, 1, 32768), (1 << 24) // (H * D)))
        case = _heads("", does, T, H, D, dtype, rng.random() < 0.7, rng.random() < 0.5)
    else:
        C = _between(rng, 32, 2048)
        if rng.random() < 0.75:
            C = max(32, C // 16 * 16)
        T = max(1, min(_between(rng, 1, 32768), (1 << 24) // C))
        post, gate = rng.random() < 0.7, rng.random() < 0.5
        case = _block("", does, T, C, dtype, post, gate, rng.random() < 0.5, rng.random() < 0.8, rng.random() < 0.8)
    del case["name"]
    return case


# ---- inputs ----------------------------------------------------------------------------------------------------

def _lengths(case, rng):
    """How long the packed sequences are: equal lengths, or any, one of them zero."""
    T, S = case["T"], case["sequences"]
    if not case["ragged"]:
        return [T // S] * S
    cuts = sorted(rng.randint(0, T) for _ in range(S - 1))
    if S > 2:
        cuts[1] = cuts[0]
    return [b - a for a, b in zip([0] + cuts, cuts + [T])]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    stored = TORCH[case["dtype"]]

    def normal(*shape, scale=1.0, mean=0.0, dtype=stored):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale + mean).to(dtype)

    def uniform(lo, hi, *shape):
        return torch.rand(*shape, generator=gen, device="cuda") * (hi - lo) + lo

    T, does = case["T"], case["does"]
    s = {"case": dict(case)}
    if case["op"] == "heads":
        H, D = case["H"], case["D"]
        s |= {"x": normal(T, H * D, scale=0.7), "w": normal(D, scale=0.2, mean=1.0)}
        if case["gate"]:
            s["z"] = normal(T, 2 * H * D)[:, H * D:] if case["wide"] else normal(T, H * D)
        if does == "bwd":
            s["rstd"] = (s["x"].float().view(T, H, D).square().mean(2) + EPS).rsqrt()
            s["dy"] = normal(T, H * D)
        return s
    if case["op"] == "block":
        C = case["C"]
        s |= {"x": normal(T, C, scale=0.8), "alpha": 0.7}
        if case["post"]:
            s["w1"] = normal(C, scale=0.2, mean=1.0)
        if case["gate"]:
            s["z"] = normal(T, C)
        if case["scale"]:
            s["scale"] = normal(C, scale=0.1, mean=0.5)
        if case["pre"]:
            s["w2"] = normal(C, scale=0.2, mean=1.0)
        if case["residual"]:
            s["residual"] = normal(T, C, scale=1.5)
        if does == "bwd":  # what a program has kept of its forward pass
            out = _plain_block(dict(s, case=dict(case, does="fwd")))
            s |= {"total": out["total"], "dtotal": normal(T, C)} | {k: out[k] for k in ("rstd1", "rstd2") if k in out}
            if case["pre"]:
                s["dy"] = normal(T, C)
        return s

    Hk, H, K, V, S = case["Hk"], case["H"], case["K"], case["V"], case["sequences"]
    rng = random.Random(seed)
    if does == "step":  # rows of a running batch: their states lie anywhere in a larger table
        s["slots"] = torch.tensor(rng.sample(range(2 * T), T), dtype=torch.int32, device="cuda")
        S = 2 * T
    else:
        lengths = _lengths(case, rng)
        starts = [0]
        for n in lengths:
            starts.append(starts[-1] + n)
        s["lengths"] = lengths
        s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    widths = [Hk * K, Hk * K, H * V]
    parts = [normal(T, n) for n in widths]
    if case["unit"]:
        parts[:2] = [torch.nn.functional.normalize(p.float().view(T, Hk, K), dim=2).view(T, Hk * K).to(stored) for p in parts[:2]]
    gates = [normal(T, H, scale=0.5), normal(T, H)]
    if case["wide"]:  # beside each other, as the convolution and the projection leave them
        parts = torch.cat(parts, 1).split(widths, 1)
        gates = torch.cat(gates, 1).split([H, H], 1)
    s["q"], s["k"], s["v"] = parts
    s["a"], s["b"] = gates
    # steps of 0.001 to 0.1 about which the tokens vary, and rates of 1 to 16 a unit of time
    dt = torch.exp(uniform(math.log(1e-3), math.log(0.1), H))
    s["a_bias"] = dt + torch.log(-torch.expm1(-dt))
    s["A"] = -torch.exp(uniform(0.0, math.log(16.0), H))
    if does == "step" or case["carry"]:
        s["state"] = normal(S, H, K, V, scale=0.3, dtype=torch.float32)
    if does == "train":
        s["dy"] = normal(T, H * V)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------

def _gate(z, silu):
    q = torch.sigmoid(z)
    return (z * q, q * (1 + z * (1 - q))) if silu else (q, q * (1 - q))


def _plain_heads(s):
    c = s["case"]
    T, H, D, stored = c["T"], c["H"], c["D"], s["x"].dtype
    x, w = s["x"].float().view(T, H, D), s["w"].float()
    z = s["z"].float().view(T, H, D) if c["gate"] else None
    g, dg = _gate(z, True) if c["gate"] else (1.0, None)
    if c["does"] == "fwd":
        rstd = (x.square().mean(2) + EPS).rsqrt()
        return {"y": (x * rstd[..., None] * w * g).to(stored).view(T, H * D), "rstd": rstd}
    rstd, dy = s["rstd"][..., None], s["dy"].float().view(T, H, D)
    n = x * rstd
    dn = dy * g * w
    out = {"dx": (rstd * (dn - n * (dn * n).mean(2, keepdim=True))).to(stored).view(T, H * D), "dw": (dy * g * n).sum((0, 1))}
    return out | ({"dz": (dy * n * w * dg).to(stored).view(T, H * D)} if c["gate"] else {})


def _plain_block(s):
    c, alpha, stored = s["case"], s["alpha"], s["x"].dtype

    def part(k):
        return s[k].float() if k in s else None

    x, w1, z, scale, w2 = (part(k) for k in ("x", "w1", "z", "scale", "w2"))
    factor = alpha * scale if c["scale"] else alpha
    g, dg = _gate(z, False) if c["gate"] else (1.0, None)
    if c["does"] == "fwd":
        out, p = {}, x
        if c["post"]:
            out["rstd1"] = (x.square().mean(1) + EPS).rsqrt()
            p = x * out["rstd1"][:, None] * w1
        total = p * g * factor
        if c["residual"]:
            total = total + s["residual"].float()
        out["total"] = total.to(stored)
        if c["pre"]:
            out["rstd2"] = (total.square().mean(1) + EPS).rsqrt()
            out["y"] = (total * out["rstd2"][:, None] * w2).to(stored)
        return out
    out, dt = {}, s["dtotal"].float()
    if c["pre"]:
        n2, dy = s["total"].float() * s["rstd2"][:, None], s["dy"].float()
        g2 = dy * w2
        dt = dt + s["rstd2"][:, None] * (g2 - n2 * (g2 * n2).mean(1, keepdim=True))
        out["dw2"] = (dy * n2).sum(0)
    if c["residual"]:
        out["dresidual"] = dt.to(stored)
    n1 = x * s["rstd1"][:, None] if c["post"] else x
    p = n1 * w1 if c["post"] else x
    dv = dt * factor
    if c["scale"]:
        out["dscale"] = (dt * alpha * p * g).sum(0)
    if c["gate"]:
        out["dz"] = (dv * p * dg).to(stored)
    dp = dv * g
    if c["post"]:
        out["dw1"] = (dp * n1).sum(0)
        g1 = dp * w1
        dp = s["rstd1"][:, None] * (g1 - n1 * (g1 * n1).mean(1, keepdim=True))
    out["dx"] = dp.to(stored)
    return out


CHUNK = 32


def _chunks(s):
    """Of the chunks of all sequences, the first ones first: the tokens of each and whether they are there; for each place in a sequence the range of its
    chunks and their sequences; and where each token lies among them.  Made at the first pass."""
    if "chunks" not in s:
        lengths = s["lengths"]
        starts = [sum(lengths[:i]) for i in range(len(lengths))]
        rows, there, ranges, lies = [], [], [], [0] * s["case"]["T"]
        for lo in range(0, max(lengths), CHUNK):
            now = [i for i, n in enumerate(lengths) if n > lo]
            ranges.append((len(rows), len(rows) + len(now), torch.tensor(now, device="cuda")))
            for i in now:
                n, first = min(CHUNK, lengths[i] - lo), starts[i] + lo
                lies[first:first + n] = range(len(rows) * CHUNK, len(rows) * CHUNK + n)
                rows.append([first + min(j, n - 1) for j in range(CHUNK)])
                there.append([j < n for j in range(CHUNK)])
        s["chunks"] = torch.tensor(rows, device="cuda"), torch.tensor(there, device="cuda"), ranges, torch.tensor(lies, device="cuda")
    return s["chunks"]


def _rule(s, q, k, v, a, b, A, a_bias):
    """(y, states after each sequence): chunk by chunk, and within a chunk by the inverse of a triangular matrix, all in 32 bits."""
    c = s["case"]
    T, Hk, H, K, V, S = c["T"], c["Hk"], c["H"], c["K"], c["V"], c["sequences"]
    rows, mask, ranges, lies = _chunks(s)

    def heads(t, n, size, share):  # [chunks, H, CHUNK, size], zeros where there is no token
        return ((t.view(T, n, size)[rows] * mask[..., None, None]).transpose(1, 2)).repeat_interleave(share, 1)

    def unit(t, n):
        t = t.view(T, n, K)
        return t if c["unit"] else t * (t.square().sum(2, keepdim=True) + EPS).rsqrt()

    qc, kc = heads(unit(q, Hk) * K ** -0.5, Hk, K, H // Hk), heads(unit(k, Hk), Hk, K, H // Hk)
    vc = heads(v, H, V, 1)
    raw = a + a_bias
    g = A * torch.where(raw > 20, raw, torch.log1p(torch.exp(raw.clamp(max=20))))
    g = (g[rows] * mask[..., None]).transpose(1, 2).double().cumsum(2)  # far sums of small numbers
    beta = (torch.sigmoid(b)[rows] * mask[..., None]).transpose(1, 2)[..., None]
    low = torch.ones(CHUNK, CHUNK, device="cuda").tril()
    decay = torch.exp((g[..., :, None] - g[..., None, :]).masked_fill(low == 0, 0.0)).float() * low
    lam, end = torch.exp(g).float()[..., None], torch.exp(g[..., -1:] - g).float()[..., None]
    L = beta * decay * (kc @ kc.transpose(2, 3).contiguous()) * low.tril(-1)
    inverse = torch.eye(CHUNK, device="cuda") - L
    power = L
    for _ in range(int(math.log2(CHUNK)) - 1):
        power = power @ power
        inverse = inverse + inverse @ power
    P = decay * (qc @ kc.transpose(2, 3).contiguous())
    state = s["state"] if "state" in s else torch.zeros(S, H, K, V, device="cuda")
    ys = []
    for lo, hi, of in ranges:
        h, kn, ln = state[of], kc[lo:hi], lam[lo:hi]
        U = inverse[lo:hi] @ (beta[lo:hi] * (vc[lo:hi] - ln * (kn @ h)))
        ys.append(ln * (qc[lo:hi] @ h) + P[lo:hi] @ U)
        state = state.index_copy(0, of, ln[:, :, -1:] * h + (end[lo:hi] * kn).transpose(2, 3).contiguous() @ U)
    return torch.cat(ys).transpose(1, 2).reshape(-1, H * V)[lies], state


NAMES = ("q", "k", "v", "a", "b", "A", "a_bias")


def _plain_delta(s):
    c, stored = s["case"], s["q"].dtype
    T, Hk, H, K, V = c["T"], c["Hk"], c["H"], c["K"], c["V"]
    leaves = [s[n].float().clone() for n in NAMES]
    if c["does"] == "step":
        q, k, v, a, b, A, a_bias = leaves
        q, k, v = q.view(T, Hk, K), k.view(T, Hk, K), v.view(T, H, V)
        if not c["unit"]:
            q, k = (t * (t.square().sum(2, keepdim=True) + EPS).rsqrt() for t in (q, k))
        q, k = (t.repeat_interleave(H // Hk, 1) for t in (q * K ** -0.5, k))
        raw = a + a_bias
        g = A * torch.where(raw > 20, raw, torch.log1p(torch.exp(raw.clamp(max=20))))
        at = s["slots"].long()
        h = torch.exp(g)[..., None, None] * s["state"][at]
        u = torch.sigmoid(b)[..., None] * (v - (h * k[..., None]).sum(2))
        h = h + k[..., None] * u[:, :, None]
        s["state"][at] = h
        return {"y": (h * q[..., None]).sum(2).to(stored).view(T, H * V), "state": s["state"]}
    if c["does"] == "fwd":
        y, state = _rule(s, *leaves)
        return {"y": y.to(stored)} | ({"state": state} if c["carry"] else {})
    with torch.enable_grad():
        for t in leaves:
            t.requires_grad_(True)
        y, _ = _rule(s, *leaves)
        grads = torch.autograd.grad(y, leaves, s["dy"].float())
    out = {"d" + n: (t if n in ("A", "a_bias") else t.to(stored)) for n, t in zip(NAMES, grads)}
    return {"y": y.detach().to(stored)} | out


# ---- the framework's calls -------------------------------------------------------------------------------------

def _plan(s):
    """The descriptor, outputs and workspaces that a program keeps for its layer, made at the first pass."""
    import paper_1803_09926_amd as dw
    c = s["case"]
    T, does = c["T"], c["does"]
    dtype = {"f32": dw.F32, "bf16": dw.BF16}[c["dtype"]]

    def f32(*shape):
        return torch.empty(*shape, device="cuda")

    def like(t):
        return torch.empty(t.shape, device="cuda", dtype=t.dtype)

    def same_rows(t):  # a gradient's rows lie as its tensor's do
        return torch.empty_strided(t.shape, t.stride(), device="cuda", dtype=t.dtype)

    def space(n):
        return torch.empty(max(n, 16), device="cuda", dtype=torch.uint8)

    if c["op"] == "heads":
        H, D = c["H"], c["D"]
        d = dw.hnorm_desc(T, H, D, dtype, EPS, z_stride=s["z"].stride(0) if c["gate"] else None)
        p = {"dw": dw, "d": d}
        if does == "fwd":
            return p | {"out": {"y": like(s["x"]), "rstd": f32(T, H)}}
        return p | {"out": {"dx": like(s["x"]), "dw": f32(D)} | ({"dz": same_rows(s["z"])} if c["gate"] else {}), "space": space(dw.hnorm_bwd_workspace_bytes(d))}
    if c["op"] == "block":
        C, x = c["C"], s["x"]
        d = dw.rnorm_desc(T, C, dtype, EPS, post=c["post"], alpha=s["alpha"])
        p = {"dw": dw, "d": d}
        if does == "fwd":
            out = ({"rstd1": f32(T)} if c["post"] else {}) | {"total": like(x)} | ({"rstd2": f32(T), "y": like(x)} if c["pre"] else {})
            return p | {"out": out}
        out = {"dx": like(x)}
        out |= {"d" + k: like(x) for k in ("z", "residual") if k in s}
        out |= {"d" + k: f32(C) for k in ("w1", "scale", "w2") if k in s}
        return p | {"out": out, "space": space(dw.rnorm_bwd_workspace_bytes(d))}
    H, K, V = c["H"], c["K"], c["V"]
    strides = {k + "_stride": s[k].stride(0) if T > 1 else None for k in ("q", "k", "v", "a", "b")}
    d = dw.gdelta_desc(T, H, K, V, key_heads=c["Hk"], sequences=2 * T if does == "step" else c["sequences"], dtype=dtype, norm=not c["unit"], eps=EPS, **strides)
    p = {"dw": dw, "d": d}
    y = torch.empty(T, H * V, device="cuda", dtype=s["v"].dtype)
    if does == "step":
        return p | {"out": {"y": y}}
    p |= {"out": {"y": y} | ({"state": like(s["state"])} if c["carry"] else {}), "space": space(dw.gdelta_fwd_workspace_bytes(d))}
    if does == "train":
        p |= {"kept": space(dw.gdelta_kept_bytes(d)), "back": space(dw.gdelta_bwd_workspace_bytes(d))}
        p["out"] |= {"d" + k: same_rows(s[k]) for k in ("q", "k", "v", "a", "b")} | {"dA": f32(H), "da_bias": f32(H)}
    return p


def _own(s):
    p = s.get("plan")
    if p is None:
        p = s["plan"] = _plan(s)
    dw, d, o, c = p["dw"], p["d"], p["out"], s["case"]
    does = c["does"]
    if c["op"] == "heads":
        if does == "fwd":
            dw.hnorm_fwd(d, s["x"], s["w"], o["y"], z=s.get("z"), rstd=o["rstd"])
        else:
            dw.hnorm_bwd(d, s["x"], s["w"], s["rstd"], s["dy"], o["dx"], o["dw"], p["space"], z=s.get("z"), dz=o.get("dz"))
        return o
    if c["op"] == "block":
        given = {k: s.get(k) for k in ("w1", "z", "scale", "w2")}
        if does == "fwd":
            dw.rnorm_fwd(d, s["x"], o["total"], y=o.get("y"), residual=s.get("residual"), rstd1=o.get("rstd1"), rstd2=o.get("rstd2"), **given)
        else:
            dw.rnorm_bwd(d, s["x"], s["total"], o["dx"], p["space"], dy=s.get("dy"), dtotal=s["dtotal"], rstd1=s.get("rstd1"), rstd2=s.get("rstd2"),
                         dz=o.get("dz"), dresidual=o.get("dresidual"), dw1=o.get("dw1"), dscale=o.get("dscale"), dw2=o.get("dw2"), **given)
        return o
    q, k, v, a, b = (s[n] for n in ("q", "k", "v", "a", "b"))
    more = {"A": s["A"], "a_bias": s["a_bias"]}
    if does == "step":
        dw.gdelta_step(d, q, k, v, a, b, s["state"], o["y"], slots=s["slots"], **more)
        return o | {"state": s["state"]}
    more["starts"] = s["starts"] if c["ragged"] else None
    dw.gdelta_fwd(d, q, k, v, a, b, o["y"], p["space"], init=s.get("state"), final=o.get("state"), kept=p.get("kept"), **more)
    if does == "train":
        dw.gdelta_bwd(d, q, k, v, a, b, p["kept"], s["dy"], o["dq"], o["dk"], o["dv"], o["da"], o["db"], p["back"], dA=o["dA"], da_bias=o["da_bias"], **more)
    return o


def run(state):
    if own:
        return _own(state)
    return {"heads": _plain_heads, "block": _plain_block, "delta": _plain_delta}[state["case"]["op"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def work(case):
    """Each input read once, each output written once; the operations of the formulas token by token, an exponential counted as one."""
    size, does, T = 4 if case["dtype"] == "f32" else 2, case["does"], case["T"]
    if case["op"] == "heads":
        n, D = T * case["H"] * case["D"], case["D"]
        gate = 1 if case["gate"] else 0
        if does == "fwd":
            return {"bytes": (2 + gate) * n * size + 4 * T * case["H"] + D * size, "flops": (5 + 4 * gate) * n}
        return {"bytes": (3 + 2 * gate) * n * size + 4 * T * case["H"] + D * (size + 4), "flops": (9 + 10 * gate) * n}
    if case["op"] == "block":
        C = case["C"]
        n = T * C
        post, gate, scale, residual, pre = (1 if case[k] else 0 for k in ("post", "gate", "scale", "residual", "pre"))
        vectors = (post + scale + pre) * C
        if does == "fwd":
            return {"bytes": (2 + gate + residual + pre) * n * size + 4 * T * (post + pre) + vectors * size,
                    "flops": (1 + 4 * post + 4 * gate + scale + residual + 4 * pre) * n}
        read = 1 if post or gate or scale else 0  # the block's output itself
        return {"bytes": (2 + read + 2 * gate + residual + 2 * pre) * n * size + 4 * T * (post + pre) + vectors * (size + 4),
                "flops": (1 + 10 * post + 9 * gate + 4 * scale + 10 * pre) * n}
    Hk, H, K, V, S = case["Hk"], case["H"], case["K"], case["V"], case["sequences"]
    rows = T * (2 * Hk * K + H * V + 2 * H) * size
    y = T * H * V * size
    params, cells = 8 * H, T * H * K * V
    if does == "step":
        return {"bytes": rows + y + 8 * cells + params, "flops": 7 * cells}
    carried = 8 * S * H * K * V if case["carry"] else 0
    if does == "fwd":
        return {"bytes": rows + y + params + carried, "flops": 7 * cells}
    return {"bytes": 3 * rows + 2 * y + 3 * params, "flops": 23 * cells}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------

def _exact_act(z, silu):
    sig = 1 / (1 + torch.exp(-z))
    return (z * sig, sig + z * sig * (1 - sig)) if silu else (sig, sig * (1 - sig))


def _exact_rms_back(x, rstd, dn):
    """The gradient of x where n = x rstd, from that of n."""
    return rstd * dn - x * rstd ** 3 * (dn * x).sum(-1, keepdim=True) / x.shape[-1]


def _exact_heads(s):
    c = s["case"]
    shape = (c["T"], c["H"], c["D"])
    x, w = s["x"].double().view(shape), s["w"].double()
    act, slope = _exact_act(s["z"].double().reshape(shape), True) if c["gate"] else (torch.ones_like(x), None)
    if c["does"] == "fwd":
        rstd = 1 / torch.sqrt((x ** 2).sum(2) / c["D"] + EPS)
        return {"y": (w * act * x * rstd[..., None]).reshape(c["T"], -1), "rstd": rstd}
    rstd, dy = s["rstd"].double()[..., None], s["dy"].double().view(shape)
    out = {"dx": _exact_rms_back(x, rstd, dy * act * w).reshape(c["T"], -1), "dw": (dy * act * x * rstd).sum(0).sum(0)}
    if c["gate"]:
        out["dz"] = (dy * slope * w * x * rstd).reshape(c["T"], -1)
    return out


def _exact_block(s):
    c = s["case"]
    x = s["x"].double()
    ones = torch.ones(c["C"], dtype=torch.float64, device=x.device)
    w1, w2, scale = (s[k].double() if k in s else ones for k in ("w1", "w2", "scale"))
    act, slope = _exact_act(s["z"].double(), False) if c["gate"] else (torch.ones_like(x), None)
    if c["does"] == "fwd":
        rstd1 = 1 / torch.sqrt((x ** 2).sum(1) / c["C"] + EPS)
        v = act * (x * rstd1[:, None] * w1 if c["post"] else x)
        total = s["alpha"] * scale * v + (s["residual"].double() if c["residual"] else 0.0)
        rstd2 = 1 / torch.sqrt((total ** 2).sum(1) / c["C"] + EPS)
        out = ({"rstd1": rstd1} if c["post"] else {}) | {"total": total}
        return out | ({"rstd2": rstd2, "y": total * rstd2[:, None] * w2} if c["pre"] else {})
    out, dt = {}, s["dtotal"].double()
    if c["pre"]:
        total, dy, rstd2 = s["total"].double(), s["dy"].double(), s["rstd2"].double()[:, None]
        out["dw2"] = (dy * total * rstd2).sum(0)
        dt = dt + _exact_rms_back(total, rstd2, dy * w2)
    if c["residual"]:
        out["dresidual"] = dt
    n1 = x * s["rstd1"].double()[:, None] if c["post"] else x
    dv = s["alpha"] * dt
    if c["scale"]:
        out["dscale"] = (dv * n1 * w1 * act).sum(0)
    dv = dv * scale
    if c["gate"]:
        out["dz"] = dv * n1 * w1 * slope
    if c["post"]:
        out["dw1"] = (dv * act * n1).sum(0)
        out["dx"] = _exact_rms_back(x, s["rstd1"].double()[:, None], dv * act * w1)
    else:
        out["dx"] = dv * act
    return out


def _exact_delta(s):
    """Token by token, all sequences beside each other."""
    c = s["case"]
    T, Hk, H, K, V, does = c["T"], c["Hk"], c["H"], c["K"], c["V"], c["does"]
    share = torch.arange(H, device="cuda") // (H // Hk)
    q, k = (s[n].double().reshape(T, Hk, K) for n in ("q", "k"))
    v = s["v"].double().reshape(T, H, V)
    rq, rk = ((1.0 if c["unit"] else 1 / torch.sqrt((t ** 2).sum(2, keepdim=True) + EPS)) for t in (q, k))
    qn, kn, scale = q * rq, k * rk, 1 / math.sqrt(K)
    raw = s["a"].double() + s["a_bias"].double()
    soft = torch.logaddexp(raw, torch.zeros_like(raw))
    A = s["A"].double()
    decay, beta = torch.exp(A * soft), 1 / (1 + torch.exp(-s["b"].double()))
    train = does == "train"
    if does == "step":
        first, lengths, slots = list(range(T)), [1] * T, s["slots"].tolist()
    else:
        first, lengths = s["starts"].tolist()[:-1], s["lengths"]
        slots = list(range(len(lengths)))
    state = s["state"].double() if "state" in s else None
    order = sorted(range(len(lengths)), key=lambda i: -lengths[i])  # the longest first: those still running are the first ones
    at = torch.tensor([first[i] for i in order], device="cuda")
    slot = torch.tensor([slots[i] for i in order], device="cuda")
    h = state[slot] if state is not None else torch.zeros(len(order), H, K, V, dtype=torch.float64, device="cuda")
    y, u = torch.zeros_like(v), torch.zeros_like(v)
    kept = torch.zeros(T, H, K, V, dtype=torch.float64, device="cuda") if train else None  # the decayed states that a token meets
    running = []
    for p in range(max(lengths)):
        running.append(sum(1 for n in lengths if n > p) if p == 0 or running[-1] > 1 else 1)
    for p, m in enumerate(running):
        t = at[:m] + p
        kt, qt = kn[t][:, share], qn[t][:, share]
        h[:m] *= decay[t][..., None, None]
        if train:
            kept[t] = h[:m]
        u[t] = beta[t][..., None] * (v[t] - (h[:m] * kt[..., None]).sum(2))
        h[:m] += kt[..., None] * u[t][:, :, None]
        y[t] = scale * (h[:m] * qt[..., None]).sum(2)
    out = {"y": y.reshape(T, H * V)}
    if state is not None:
        state[slot] = h
        out["state"] = state
    if not train:
        return out
    dy = s["dy"].double().view(T, H, V) * scale
    dq, dk = torch.zeros(T, H, K, dtype=torch.float64, device="cuda"), torch.zeros(T, H, K, dtype=torch.float64, device="cuda")
    dv, dbeta, dlog = torch.zeros_like(v), torch.zeros_like(beta), torch.zeros_like(beta)
    g = torch.zeros_like(h)
    for p in reversed(range(len(running))):
        m = running[p]
        t = at[:m] + p
        kt, qt = kn[t][:, share], qn[t][:, share]
        met, ut = kept[t], u[t][:, :, None]
        dq[t] = ((met + kt[..., None] * ut) * dy[t][:, :, None]).sum(3)
        g[:m] += qt[..., None] * dy[t][:, :, None]
        du = (g[:m] * kt[..., None]).sum(2)
        read = (met * kt[..., None]).sum(2)
        dbeta[t] = (du * (v[t] - read)).sum(2)
        dv[t] = du * beta[t][..., None]
        dk[t] = (g[:m] * ut).sum(3) - (met * dv[t][:, :, None]).sum(3)
        g[:m] -= kt[..., None] * dv[t][:, :, None]
        dlog[t] = (g[:m] * met).sum((2, 3))
        g[:m] *= decay[t][..., None, None]
    sig = 1 / (1 + torch.exp(-raw))
    da = dlog * A * sig
    dq, dk = (t.view(T, Hk, H // Hk, K).sum(2) for t in (dq, dk))
    if not c["unit"]:
        dq, dk = (r * (d - n * (d * n).sum(2, keepdim=True)) for d, n, r in ((dq, qn, rq), (dk, kn, rk)))
    return out | {"dq": dq.reshape(T, Hk * K), "dk": dk.reshape(T, Hk * K), "dv": dv.reshape(T, H * V), "da": da, "db": dbeta * beta * (1 - beta),
                  "dA": (dlog * soft).sum(0), "da_bias": da.sum(0)}


def exact(case, seed):
    return {"heads": _exact_heads, "block": _exact_block, "delta": _exact_delta}[case["op"]](prepare(case, seed))
