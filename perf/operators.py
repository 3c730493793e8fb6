"""The operators of a token sequence's block whose speed counts: the layer norm in front of it, the short causal depthwise
convolution over its tokens, and the selective state space scan that reads the convolution's output; for training steps, for prompts and
for single tokens.

A case is one operator with everything that its descriptor takes.  `op` names the operator ("norm", "conv", "scan"), `does` what the
program runs: "fwd" (inference), "bwd" (the backward pass), "train" (forward and backward pass) or "step" (one new token of each row, the carried states
updated in place).  Tokens are packed: T of them in `sequences` sequences, of equal lengths or, where `ragged`, of any (one of them empty).
"""
import math
import random

import torch

own = False

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-5


# ---- the cases -------------------------------------------------------------------------------------------------

def _norm(name, does, T, C, dtype, residual):
    return {"name": name, "op": "norm", "does": does, "T": T, "C": C, "dtype": dtype, "residual": residual}


def _conv(name, does, T, C, dtype, K=4, sequences=1, ragged=False, carry=False, wide=False):
    """carry: the sequences continue earlier ones, whose last inputs are given and whose new last inputs come back.  wide: the input is one half
    of a projection's rows.  A step has T rows whose states lie in 2 T slots, in any order."""
    return {"name": name, "op": "conv", "does": does, "T": T, "C": C, "dtype": dtype, "K": K, "sequences": sequences, "ragged": ragged,
            "carry": carry, "wide": wide}


def _scan(name, does, T, C, dtype, N=16, groups=1, sequences=1, ragged=False, carry=False, wide=False):
    """carry, wide and the slots of a step as for the convolution; wide is here the gate's half of the projection, and the rows that hold B and C
    beside each other."""
    return {"name": name, "op": "scan", "does": does, "T": T, "C": C, "dtype": dtype, "N": N, "groups": groups, "sequences": sequences,
            "ragged": ragged, "carry": carry, "wide": wide}


def listed():
    return [
        # the norm of a few new tokens with the residual's sum, as each step of generation has it: the latency of one small call
        _norm("norm_tokens", "fwd", 8, 1024, "bf16", True),
        # the norm of a long prompt or a training batch, with the residual's sum
        _norm("norm_batch", "fwd", 32768, 1024, "bf16", True),
        # the norm's backward pass in a training step: a row count that is no multiple of anything, fp32
        _norm("norm_gradients", "bwd", 9999, 1536, "f32", False),
        # generation: one token of 64 rows through the convolution
        _conv("conv_tokens", "step", 64, 2048, "bf16", wide=True),
        # prompts of several users, packed, that continue earlier ones
        _conv("conv_prompts", "fwd", 8191, 1536, "bf16", sequences=6, ragged=True, carry=True, wide=True),
        # the convolution's backward pass over a training batch
        _conv("conv_gradients", "bwd", 16384, 1024, "f32", sequences=8),
        # generation: one token of 64 rows through the scan, whose states are most of what moves
        _scan("scan_tokens", "step", 64, 2048, "bf16", wide=True),
        # one short prompt: few channels in flight, and a chain of 300 tokens
        _scan("scan_short_prompt", "fwd", 301, 1024, "bf16"),
        # a long prompt alone on the card
        _scan("scan_long_prompt", "fwd", 16384, 1024, "bf16", carry=True, wide=True),
        # many prompts, packed, of any lengths
        _scan("scan_prompts", "fwd", 16383, 2048, "bf16", sequences=24, ragged=True, wide=True),
        # a training step, bf16
        _scan("scan_training", "train", 8192, 1536, "bf16", sequences=8, wide=True),
        # a small training step in fp32: channels that are no multiple of a tile, two groups of B and C, packed
        _scan("scan_training_odd", "train", 1501, 728, "f32", N=8, groups=2, sequences=5, ragged=True),
    ]


def _between(rng, least, most):
    return int(round(math.exp(rng.uniform(math.log(least), math.log(most)))))


def draw(rng):
    """One case of the listed ones' ranges: 1 to 32768 tokens, 32 to 2048 channels (odd ones among them), 1 to 64 sequences, filters of 2 to 8 taps, 1 to 64
    states, both types, each direction; at most what the largest listed case of its kind has."""
    op = rng.choice(["norm", "conv", "scan", "scan"])
    does = rng.choice({"norm": ["fwd", "bwd"], "conv": ["fwd", "bwd", "step"], "scan": ["fwd", "train", "step"]}[op])
    dtype = rng.choice(sorted(TORCH))
    C = _between(rng, 32, 2048)
    if rng.random() < 0.75:
        C = max(32, C // 16 * 16)
    if does == "step":
        T = _between(rng, 1, 128)
    else:
        T = _between(rng, 1, 32768)
    if op == "norm":
        T = max(1, min(T, (1 << 25) // C))
        case = _norm("", does, T, C, dtype, rng.random() < 0.5)
    else:
        sequences, ragged = 1, False
        if does != "step" and rng.random() < 0.7:
            sequences = _between(rng, 1, min(64, T))
            ragged = rng.random() < 0.6
        carry, wide = does == "fwd" and rng.random() < 0.5, rng.random() < 0.5
        if op == "conv":
            T = max(1, min(T, (1 << 24) // C))
            K = rng.choice([2, 3, 4, 4, 4, 5, 7, 8])
        else:
            N = rng.choice([1, 3, 4, 8, 16, 16, 16, 24, 32, 64])
            groups = rng.choice([1, 1, 1, 2, 4])
            C = C // groups * groups
            T = max(1, min(T, ((1 << 29) if does == "fwd" else (1 << 27)) // (C * max(N, 8))))
        sequences = min(sequences, T)
        if not ragged and does != "step":
            T = T // sequences * sequences
        if op == "conv":
            case = _conv("", does, T, C, dtype, K, sequences, ragged, carry, wide)
        else:
            case = _scan("", does, T, C, dtype, N, groups, sequences, ragged, carry, wide)
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

    T, C = case["T"], case["C"]
    s = {"case": dict(case)}
    if case["op"] == "norm":
        s |= {"x": normal(T, C, scale=1.5, mean=0.4), "w": normal(C, scale=0.2, mean=1.0), "b": normal(C, scale=0.2)}
        if case["residual"]:
            s["dtotal" if case["does"] == "bwd" else "residual"] = normal(T, C)
        if case["does"] == "bwd":
            x = s["x"].float()
            s["mean"] = x.mean(1)
            s["rstd"] = ((x - s["mean"][:, None]).square().mean(1) + EPS).rsqrt()
            s["dy"] = normal(T, C)
        return s

    step, S = case["does"] == "step", case["sequences"]
    rng = random.Random(seed)
    if step:  # rows of a running batch: their states lie anywhere in a larger table
        slots = rng.sample(range(2 * T), T)
        s["slots"] = torch.tensor(slots, dtype=torch.int32, device="cuda")
        S = 2 * T
    else:
        lengths = _lengths(case, rng)
        starts = [0]
        for n in lengths:
            starts.append(starts[-1] + n)
        s["lengths"] = lengths
        s["starts"] = torch.tensor(starts, dtype=torch.int32, device="cuda")
    both = normal(T, 2 * C) if case["wide"] else None  # what a projection gives: the input and the gate beside each other
    if case["op"] == "conv":
        K = case["K"]
        s |= {"x": both[:, :C] if case["wide"] else normal(T, C), "w": normal(K, C, scale=K ** -0.5), "b": normal(C, scale=0.1)}
        if step or case["carry"]:
            s["state"] = normal(S, K - 1, C)
        if case["does"] == "bwd":
            s["dy"] = normal(T, C)
        return s

    N, G = case["N"], case["groups"]
    s["x"] = normal(T, C)
    s["z"] = both[:, C:] if case["wide"] else normal(T, C)
    if case["wide"]:
        bc = normal(T, 2 * G * N)
        s["B"], s["C"] = bc[:, :G * N], bc[:, G * N:]
    else:
        s["B"], s["C"] = normal(T, G * N), normal(T, G * N)
    # steps of 0.001 to 0.1 about which the tokens vary, and decays of 1 to N a unit of time: the usual start of training
    dt = torch.exp(uniform(math.log(1e-3), math.log(0.1), C))
    s["dt_bias"] = dt + torch.log(-torch.expm1(-dt))
    s["dt"] = normal(T, C, scale=0.5)
    s["A"] = -torch.arange(1, N + 1, device="cuda", dtype=torch.float32).repeat(C, 1) * torch.exp(uniform(-0.1, 0.1, C, N))
    s["D"] = normal(C, scale=0.2, mean=1.0, dtype=torch.float32)
    if step or case["carry"]:
        s["state"] = normal(S, C, N, dtype=torch.float32)
    if case["does"] == "train":
        s["dy"] = normal(T, C)
    return s


# ---- the plain forms -------------------------------------------------------------------------------------------

def _plain_norm(s):
    stored, x, w, b = s["x"].dtype, s["x"].float(), s["w"].float(), s["b"].float()
    if s["case"]["does"] == "fwd":
        total = x + s["residual"].float() if "residual" in s else x
        mean = total.mean(1)
        centred = total - mean[:, None]
        rstd = (centred.square().mean(1) + EPS).rsqrt()
        out = {"y": (centred * rstd[:, None] * w + b).to(stored), "mean": mean, "rstd": rstd}
        return out | ({"total": total.to(stored)} if "residual" in s else {})
    dy, rstd = s["dy"].float(), s["rstd"][:, None]
    xhat = (x - s["mean"][:, None]) * rstd
    g = dy * w
    dx = rstd * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    if "dtotal" in s:
        dx = dx + s["dtotal"].float()
    return {"dx": dx.to(stored), "dw": (dy * xhat).sum(0), "db": dy.sum(0)}


def _places(s):
    """The sequence of each token, and the token's place in it."""
    t = torch.arange(s["case"]["T"], device="cuda")
    seq = torch.searchsorted(s["starts"][1:].long(), t, right=True)
    return seq, t - s["starts"][seq]


def _plain_conv(s):
    c = s["case"]
    stored, T, C, K, S = s["x"].dtype, c["T"], c["C"], c["K"], c["sequences"]
    x, w, b = s["x"].float(), s["w"].float(), s["b"].float()
    if c["does"] == "step":
        at = s["slots"].long()
        taps = torch.cat([s["state"][at].float(), x[:, None]], 1)
        s["state"][at] = taps[:, 1:].to(stored)
        p = (taps * w).sum(1) + b
        return {"y": (p * torch.sigmoid(p)).to(stored), "state": s["state"]}
    seq, place = _places(s)
    before = s["state"].float().reshape(-1, C) if "state" in s else torch.zeros(S * (K - 1), C, device="cuda")
    table = torch.cat([before, x])  # the rows before each sequence, then the tokens

    def row(seq, place):  # the table's row of a place in a sequence, K - 1 places before its first among them
        return torch.where(place < 0, seq * (K - 1) + K - 1 + place, S * (K - 1) + s["starts"][seq] + place)

    back = torch.arange(K - 1, -1, -1, device="cuda")
    taps = table[row(seq[:, None], place[:, None] - back)]
    p = (taps * w).sum(1) + b
    q = torch.sigmoid(p)
    if c["does"] == "fwd":
        out = {"y": (p * q).to(stored)}
        if c["carry"]:
            every = torch.arange(S, device="cuda")
            ends = s["starts"][1:] - s["starts"][:-1]
            out["state"] = table[row(every[:, None], ends[:, None] - back[:-1])].to(stored)
        return out
    dp = s["dy"].float() * (q + p * q * (1 - q))
    t = torch.arange(T, device="cuda")[:, None] + back  # the outputs that a token is a tap of
    inside = t < s["starts"][seq + 1][:, None]
    dx = (dp[t.clamp(max=T - 1)] * inside[..., None] * w).sum(1)
    return {"dx": dx.to(stored), "dw": (dp[:, None] * taps).sum(0), "db": dp.sum(0)}


def _recurrence(a, u, longest):
    """h[t] = a[t] h[t-1] + u[t] along the first axis, in place of u, by doubling: a is 0 at each sequence's first token."""
    a, k = a.clone(), 1
    while k < longest:
        u[k:] += a[k:] * u[:-k]
        a[k:] = a[k:] * a[:-k]
        k *= 2
    return u


def _plain_scan(s):
    c = s["case"]
    stored, T, C, N, G = s["x"].dtype, c["T"], c["C"], c["N"], c["groups"]
    x, z, A, D = s["x"].float(), s["z"].float(), s["A"], s["D"]
    raw = s["dt"].float() + s["dt_bias"]
    delta = torch.where(raw > 20, raw, torch.log1p(torch.exp(raw.clamp(max=20))))

    def wide(v):  # a group's values for each of its channels
        return v.float().view(T, G, 1, N).expand(T, G, C // G, N).reshape(T, C, N)

    B, Ct = wide(s["B"]), wide(s["C"])
    a = torch.exp(delta[..., None] * A)
    u = (delta * x)[..., None] * B
    q = torch.sigmoid(z)
    if c["does"] == "step":
        at = s["slots"].long()
        h = a * s["state"][at] + u
        s["state"][at] = h
        return {"y": (((h * Ct).sum(2) + D * x) * z * q).to(stored), "state": s["state"]}
    seq, place = _places(s)
    first = place == 0
    if "state" in s:
        u = torch.where(first[:, None, None], u + a * s["state"][seq], u)
    longest = max(s["lengths"])
    h = _recurrence(torch.where(first[:, None, None], 0.0, a), u, longest)
    y = (h * Ct).sum(2) + D * x
    out = {"y": (y * z * q).to(stored)}
    if c["carry"]:
        ends = s["starts"][1:].long()
        empty = ends == s["starts"][:-1]
        out["state"] = torch.where(empty[:, None, None], s["state"], h[(ends - 1).clamp(min=0)])
    if c["does"] == "fwd":
        return out
    dout = s["dy"].float()
    dz = dout * y * (q + z * q * (1 - q))
    dy = dout * z * q
    before = torch.where(first[:, None, None], 0.0, torch.cat([torch.zeros_like(h[:1]), h[:-1]]))
    after = torch.cat([torch.where(first[1:, None, None], 0.0, a[1:]), torch.zeros_like(a[:1])])
    g = _recurrence(after.flip(0), (dy[..., None] * Ct).flip(0), longest).flip(0)
    decay = g * a * before
    gB = (g * B).sum(2)
    ddelta = x * gB + (decay * A).sum(2)
    graw = ddelta * torch.sigmoid(raw)

    def narrow(v):  # the sum over a group's channels
        return v.view(T, G, C // G, N).sum(2).view(T, G * N).to(stored)

    return out | {"dx": (dy * D + delta * gB).to(stored), "dz": dz.to(stored), "ddt": graw.to(stored),
                  "dB": narrow(g * (delta * x)[..., None]), "dC": narrow(dy[..., None] * h),
                  "dA": (decay * delta[..., None]).sum(0), "dD": (dy * x).sum(0), "ddt_bias": graw.sum(0)}


# ---- the framework's calls -------------------------------------------------------------------------------------

def _plan(s):
    """The descriptor, outputs and workspaces that a program keeps for its layer, made at the first pass."""
    import paper_1803_09926_amd as dw
    c = s["case"]
    T, C, x = c["T"], c["C"], s["x"]
    dtype = {"f32": dw.F32, "bf16": dw.BF16}[c["dtype"]]

    def f32(*shape):
        return torch.empty(*shape, device="cuda")

    def like(t):
        return torch.empty(t.shape, device="cuda", dtype=t.dtype)

    def same_rows(t):  # a gradient's rows lie as its tensor's do
        return torch.empty_strided(t.shape, t.stride(), device="cuda", dtype=t.dtype)

    def space(n):
        return torch.empty(max(n, 16), device="cuda", dtype=torch.uint8)

    if c["op"] == "norm":
        d = dw.lnorm_desc(T, C, dtype, EPS)
        if c["does"] == "fwd":
            out = {"y": like(x), "mean": f32(T), "rstd": f32(T)} | ({"total": like(x)} if "residual" in s else {})
            return {"dw": dw, "d": d, "out": out}
        return {"dw": dw, "d": d, "out": {"dx": like(x), "dw": f32(C), "db": f32(C)}, "space": space(dw.lnorm_bwd_workspace_bytes(d))}
    slots = 2 * T if c["does"] == "step" else c["sequences"]
    if c["op"] == "conv":
        K = c["K"]
        d = dw.cconv_desc(T, C, K, slots, dtype, x_stride=x.stride(0))
        p = {"dw": dw, "d": d}
        if c["does"] == "bwd":
            return p | {"out": {"dx": same_rows(x), "dw": f32(K, C), "db": f32(C)}, "space": space(dw.cconv_bwd_workspace_bytes(d))}
        return p | {"out": {"y": like(x)} | ({"state": like(s["state"])} if c["carry"] else {})}
    N = c["N"]
    d = dw.sscan_desc(T, C, N, c["groups"], slots, dtype, z_stride=s["z"].stride(0), b_stride=s["B"].stride(0), c_stride=s["C"].stride(0))
    p = {"dw": dw, "d": d}
    if c["does"] == "step":
        return p | {"out": {"y": like(x)}}
    p |= {"out": {"y": like(x)} | ({"state": like(s["state"])} if c["carry"] else {}), "space": space(dw.sscan_fwd_workspace_bytes(d))}
    if c["does"] == "train":
        p["kept"] = space(dw.sscan_kept_bytes(d))
        p["back"] = space(dw.sscan_bwd_workspace_bytes(d))
        p["out"] |= {"dx": like(x), "dz": same_rows(s["z"]), "ddt": like(x), "dB": same_rows(s["B"]), "dC": same_rows(s["C"]),
                     "dA": f32(C, N), "dD": f32(C), "ddt_bias": f32(C)}
    return p


def _own(s):
    p = s.get("plan")
    if p is None:
        p = s["plan"] = _plan(s)
    dw, d, o, c = p["dw"], p["d"], p["out"], s["case"]
    if c["op"] == "norm":
        if c["does"] == "fwd":
            dw.lnorm_fwd(d, s["x"], s["w"], s["b"], o["y"], o["mean"], o["rstd"], residual=s.get("residual"), total=o.get("total"))
        else:
            dw.lnorm_bwd(d, s["x"], s["w"], s["mean"], s["rstd"], s["dy"], o["dx"], o["dw"], o["db"], p["space"], dtotal=s.get("dtotal"))
        return o
    if c["op"] == "conv":
        if c["does"] == "step":
            dw.cconv_step(d, s["x"], s["w"], s["b"], s["state"], o["y"], slots=s["slots"])
            return o | {"state": s["state"]}
        starts = s["starts"] if c["ragged"] else None
        if c["does"] == "fwd":
            dw.cconv_fwd(d, s["x"], s["w"], s["b"], o["y"], starts=starts, init=s.get("state"), final=o.get("state"))
        else:
            dw.cconv_bwd(d, s["x"], s["w"], s["b"], s["dy"], o["dx"], o["dw"], o["db"], p["space"], starts=starts)
        return o
    x, dt, A, B, C = s["x"], s["dt"], s["A"], s["B"], s["C"]
    more = {"D": s["D"], "z": s["z"], "dt_bias": s["dt_bias"]}
    if c["does"] == "step":
        dw.sscan_step(d, x, dt, A, B, C, s["state"], o["y"], slots=s["slots"], **more)
        return o | {"state": s["state"]}
    more["starts"] = s["starts"] if c["ragged"] else None
    dw.sscan_fwd(d, x, dt, A, B, C, o["y"], p["space"], init=s.get("state"), final=o.get("state"), kept=p.get("kept"), **more)
    if c["does"] == "train":
        dw.sscan_bwd(d, x, dt, A, B, C, p["kept"], s["dy"], o["dx"], o["ddt"], o["dA"], o["dB"], o["dC"], p["back"], dD=o["dD"], dz=o["dz"],
                     ddt_bias=o["ddt_bias"], **more)
    return o


def run(state):
    if own:
        return _own(state)
    return {"norm": _plain_norm, "conv": _plain_conv, "scan": _plain_scan}[state["case"]["op"]](state)


# ---- what a pass cannot do without -----------------------------------------------------------------------------

def work(case):
    """Each input read once, each output written once; the operations of the formulas, an exponential counted as one."""
    size, does = 4 if case["dtype"] == "f32" else 2, case["does"]
    T, C = case["T"], case["C"]
    if case["op"] == "norm":
        more = 1 if case["residual"] else 0
        if does == "fwd":
            return {"bytes": (2 + 2 * more) * T * C * size + 8 * T + 2 * C * size, "flops": (8 + more) * T * C}
        return {"bytes": (3 + more) * T * C * size + 8 * T + C * size + 8 * C, "flops": (13 + more) * T * C}
    if case["op"] == "conv":
        K, S = case["K"], case["sequences"]
        if does == "step":
            return {"bytes": (2 * T * C + 2 * T * (K - 1) * C + (K + 1) * C) * size, "flops": (2 * K + 5) * T * C}
        carried = 2 * S * (K - 1) * C * size if case["carry"] else 0
        if does == "fwd":
            return {"bytes": (2 * T * C + (K + 1) * C) * size + carried, "flops": (2 * K + 5) * T * C}
        return {"bytes": (3 * T * C + (K + 1) * C) * size + 4 * (K + 1) * C, "flops": (6 * K + 10) * T * C}
    N, G, S = case["N"], case["groups"], case["sequences"]
    params = 4 * (C * N + 2 * C)
    if does == "step":
        return {"bytes": (4 * T * C + 2 * T * G * N) * size + 8 * T * C * N + params, "flops": T * C * (7 * N + 12)}
    carried = 8 * S * C * N if case["carry"] else 0
    forward = {"bytes": (4 * T * C + 2 * T * G * N) * size + params + carried, "flops": T * C * (7 * N + 12)}
    if does == "fwd":
        return forward
    return {"bytes": forward["bytes"] + (7 * T * C + 4 * T * G * N) * size + 2 * params, "flops": forward["flops"] + T * C * (22 * N + 30)}


# ---- the definitions in 64 bits --------------------------------------------------------------------------------

def _exact_norm(s):
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    C = x.shape[1]
    if s["case"]["does"] == "fwd":
        if "residual" in s:
            x = x + s["residual"].double()
        mean = x.sum(1) / C
        rstd = 1 / torch.sqrt(((x - mean[:, None]) ** 2).sum(1) / C + EPS)
        out = {"y": w * (x - mean[:, None]) * rstd[:, None] + b, "mean": mean, "rstd": rstd}
        return out | ({"total": x} if "residual" in s else {})
    dy, rstd = s["dy"].double(), s["rstd"].double()[:, None]
    xhat = (x - s["mean"].double()[:, None]) * rstd
    dxhat = dy * w
    dx = (C * dxhat - dxhat.sum(1, keepdim=True) - xhat * (dxhat * xhat).sum(1, keepdim=True)) * rstd / C
    if "dtotal" in s:
        dx = dx + s["dtotal"].double()
    return {"dx": dx, "dw": (dy * xhat).sum(0), "db": dy.sum(0)}


def _exact_conv(s):
    """Sequence by sequence, each with its K - 1 rows before it."""
    c = s["case"]
    K, C, stored = c["K"], c["C"], TORCH[c["dtype"]]
    x, w, b = s["x"].double(), s["w"].double(), s["b"].double()
    back = c["does"] == "bwd"
    if c["does"] == "step":
        spans = [(i, i + 1) for i in range(c["T"])]
        where = s["slots"].tolist()
    else:
        bounds = s["starts"].tolist()
        spans = list(zip(bounds[:-1], bounds[1:]))
        where = range(len(spans))
    y, dx = torch.zeros_like(x), torch.zeros_like(x)
    dw, db = torch.zeros_like(w), torch.zeros_like(b)
    state = s["state"].double() if "state" in s else None
    for (lo, hi), slot in zip(spans, where):
        before = state[slot] if state is not None else torch.zeros(K - 1, C, dtype=torch.float64, device=x.device)
        line = torch.cat([before, x[lo:hi]])
        n = hi - lo
        p = b + sum(w[k] * line[k:k + n] for k in range(K))
        sig = 1 / (1 + torch.exp(-p))
        y[lo:hi] = p * sig
        if back:
            dp = s["dy"][lo:hi].double() * sig * (1 + p * (1 - sig))
            dline = torch.zeros_like(line)
            for k in range(K):
                dline[k:k + n] += w[k] * dp
                dw[k] += (dp * line[k:k + n]).sum(0)
            db += dp.sum(0)
            dx[lo:hi] = dline[K - 1:]
        if state is not None:
            state[slot] = line[n:]
    if back:
        return {"dx": dx, "dw": dw, "db": db}
    return {"y": y} | ({"state": state} if state is not None else {})


def _exact_scan(s):
    """Token by token, all sequences beside each other."""
    c = s["case"]
    T, C, N, G = c["T"], c["C"], c["N"], c["groups"]
    x, z, A, D = s["x"].double(), s["z"].double(), s["A"].double(), s["D"].double()
    raw = s["dt"].double() + s["dt_bias"].double()
    delta = torch.logaddexp(raw, torch.zeros_like(raw))
    group = torch.arange(C, device=x.device) // (C // G)
    B, Ct = s["B"].double().view(T, G, N), s["C"].double().view(T, G, N)
    sig = 1 / (1 + torch.exp(-z))
    train = c["does"] == "train"
    if c["does"] == "step":
        first, lengths, slots = list(range(T)), [1] * T, s["slots"].tolist()
    else:
        first, lengths = s["starts"].tolist()[:-1], s["lengths"]
        slots = list(range(len(lengths)))
    state = s["state"].double() if "state" in s else None
    order = sorted(range(len(lengths)), key=lambda i: -lengths[i])  # the longest first: those still running are the first ones
    at = torch.tensor([first[i] for i in order], device=x.device)
    slot = torch.tensor([slots[i] for i in order], device=x.device)
    h = state[slot] if state is not None else torch.zeros(len(order), C, N, dtype=torch.float64, device=x.device)
    y, kept = torch.zeros_like(x), torch.zeros(T, C, N, dtype=torch.float64, device=x.device) if train else None
    running = []  # how many sequences have a token at each place
    for p in range(max(lengths)):
        running.append(sum(1 for n in lengths if n > p) if p == 0 or running[-1] > 1 else 1)
    for p, m in enumerate(running):
        t = at[:m] + p
        h[:m] = torch.exp(delta[t][..., None] * A) * h[:m] + (delta[t] * x[t])[..., None] * B[t][:, group]
        y[t] = (h[:m] * Ct[t][:, group]).sum(2)
        if train:
            kept[t] = h[:m]
    y += D * x
    out = {"y": y * z * sig}
    if state is not None:
        state[slot] = h
        out["state"] = state
    if not train:
        return out
    dout = s["dy"].double()
    dy = dout * z * sig
    dx, ddelta = dy * D, torch.zeros_like(x)
    dA, dB, dC = torch.zeros_like(A), torch.zeros_like(B), torch.zeros_like(Ct)
    g = torch.zeros_like(h)
    for p in reversed(range(len(running))):
        m = running[p]
        t = at[:m] + p
        Bt, a = B[t][:, group], torch.exp(delta[t][..., None] * A)
        g[:m] += dy[t][..., None] * Ct[t][:, group]
        dC[t] = (dy[t][..., None] * kept[t]).view(m, G, C // G, N).sum(2)
        dB[t] = (g[:m] * (delta[t] * x[t])[..., None]).view(m, G, C // G, N).sum(2)
        gB = (g[:m] * Bt).sum(2)
        dx[t] += delta[t] * gB
        g[:m] *= a  # the gradient of the state before the token
        if p:
            ddelta[t] = (g[:m] * kept[t - 1] * A).sum(2)
            dA += (g[:m] * kept[t - 1] * delta[t][..., None]).sum(0)
        ddelta[t] += x[t] * gB
    ddt = ddelta / (1 + torch.exp(-raw))
    return out | {"dx": dx, "dz": dout * y * sig * (1 + z * (1 - sig)), "ddt": ddt, "dB": dB.view(T, G * N), "dC": dC.view(T, G * N),
                  "dA": dA, "dD": (dy * x).sum(0), "ddt_bias": ddt.sum(0)}


def exact(case, seed):
    return {"norm": _exact_norm, "conv": _exact_conv, "scan": _exact_scan}[case["op"]](prepare(case, seed))
