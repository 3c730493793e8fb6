"""A stack of blocks that learn by the gated delta rule, from this library's operators: a projection to queries, keys, values, gates and rates, the short causal
depthwise convolution over the first three, the delta rule, the gated norm of its heads, and the projection back; between blocks the norm of a block's output, its
scale, the residual's sum and the norm for the next block in one call.

The dense projections are plain matrix products (torch.mm, a library's); everything else runs on the kernels of this package.  A stack trains on packed sequences
(`forward` with keep=True, then `backward`), reads prompts (`forward` with `states`), and generates token by token (`step`).

Usage:  python -m paper_1803_09926_amd.delta_mixer [--width 1024] [--blocks 2] [--tokens 4096] [--steps 5] [--generate 32]
Trains a stack on synthetic sequences, then continues prompts and checks the tokens generated one at a time against the prompt read at once.
"""
from __future__ import annotations

import argparse
import json
import math
import time

import torch

import paper_1803_09926_amd as dw

ALPHA = 0.5                                      # of a block's normalised output beside the residual


class DeltaBlock:
    """The mixer between two norms: rows of `width` to rows of `width`."""

    def __init__(self, width, heads, key_heads, K, V, taps=4, dtype=torch.bfloat16, seed=0, device="cuda"):
        self.M, self.H, self.Hk, self.K, self.V, self.taps = width, heads, key_heads, K, V, taps
        self.dtype, self.kind = dtype, dw.F32 if dtype == torch.float32 else dw.BF16
        self.keys, self.values = key_heads * K, heads * V
        self.C = 2 * self.keys + self.values                     # channels of the convolution: queries, keys, values
        self.wide = self.C + self.values + 2 * heads             # and of the projection: the heads' gate, a and b behind them
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(*shape, generator=g) * scale).to(device=device, dtype=dtype)

        def ones(n):
            return torch.ones(n, device=device, dtype=dtype)

        dt = torch.exp(torch.rand(heads, generator=g) * (math.log(0.1) - math.log(1e-3)) + math.log(1e-3))
        self.p = {"w_in": normal(width, self.wide, scale=width ** -0.5), "conv_w": normal(taps, self.C, scale=taps ** -0.5), "head_w": ones(V),
                  "w_out": normal(self.values, width, scale=self.values ** -0.5), "post_w": ones(width), "scale": ones(width), "next_w": ones(width),
                  "A_log": torch.log(torch.rand(heads, generator=g) * 15 + 1).to(device), "a_bias": (dt + torch.log(-torch.expm1(-dt))).to(device)}

    def states(self, sequences):
        """Of sequences that start: the convolution's last rows, and the heads' states."""
        return (torch.zeros(sequences, self.taps - 1, self.C, device=self.p["A_log"].device, dtype=self.dtype),
                torch.zeros(sequences, self.H, self.K, self.V, device=self.p["A_log"].device))

    def _new(self, *shape, like=None):
        return torch.empty(*shape, device=self.p["A_log"].device, dtype=like or self.dtype)

    def _space(self, nbytes):
        """A workspace for one call (torch's allocator hands it out again behind that call on the same stream)."""
        return self._new(max(nbytes, 16), like=torch.uint8)

    def _descs(self, T, sequences):
        C, H = self.C, self.H
        return (dw.cconv_desc(T, C, self.taps, sequences, self.kind, x_stride=self.wide),
                dw.gdelta_desc(T, H, self.K, self.V, self.Hk, sequences, self.kind, q_stride=C, k_stride=C, v_stride=C, a_stride=self.wide, b_stride=self.wide),
                dw.hnorm_desc(T, H, self.V, self.kind, z_stride=self.wide), dw.rnorm_desc(T, self.M, self.kind, alpha=ALPHA))

    def _parts(self, proj, u):
        """(q, k, v of the convolution's rows; z, a, b of the projection's)"""
        n, v, C, H = self.keys, self.values, self.C, self.H
        return u[:, :n], u[:, n:2 * n], u[:, 2 * n:], proj[:, C:C + v], proj[:, C + v:C + v + H], proj[:, C + v + H:]

    def forward(self, normed, total, starts=None, sequences=1, states=None, keep=False):
        """(normed, total) for the next block.  states: continues these sequences, and moves them on.  keep: what `backward` needs is returned third."""
        p, T = self.p, normed.shape[0]
        cd, gd, hd, rd = self._descs(T, sequences)
        rows, S = states if states is not None else (None, None)
        proj = normed @ p["w_in"]
        u, y, o = self._new(T, self.C), self._new(T, self.values), self._new(T, self.values)
        new_rows, new_S = (None, None) if rows is None else (torch.empty_like(rows), torch.empty_like(S))
        dw.cconv_fwd(cd, proj[:, :self.C], p["conv_w"], None, u, starts=starts, init=rows, final=new_rows)
        q, k, v, z, a, b = self._parts(proj, u)
        kept = self._space(dw.gdelta_kept_bytes(gd)) if keep else None
        space = None if keep else self._space(dw.gdelta_fwd_workspace_bytes(gd))
        dw.gdelta_fwd(gd, q, k, v, a, b, y, space, A=-torch.exp(p["A_log"]), a_bias=p["a_bias"], starts=starts, init=S, final=new_S, kept=kept)
        rstd = self._new(T, self.H, like=torch.float32)
        dw.hnorm_fwd(hd, y, p["head_w"], o, z=z, rstd=rstd)
        began = None if rows is None or not keep else rows.clone()
        if rows is not None:
            rows.copy_(new_rows)
            S.copy_(new_S)
        out, following, summed = o @ p["w_out"], self._new(T, self.M), self._new(T, self.M)
        r1, r2 = self._new(T, like=torch.float32), self._new(T, like=torch.float32)
        dw.rnorm_fwd(rd, out, summed, y=following, w1=p["post_w"], scale=p["scale"], residual=total, w2=p["next_w"], rstd1=r1, rstd2=r2)
        return (following, summed) + (((normed, proj, u, kept, y, o, rstd, out, summed, r1, r2, starts, sequences, began),) if keep else ())

    def backward(self, dfollowing, dsummed, kept):
        """From the gradients of (normed, total) behind the block (the second may be None) to those before it, and the gradients by parameter.  The states that the
        sequences began with are constants."""
        p = self.p
        normed, proj, u, kept, y, o, rstd, out, summed, r1, r2, starts, sequences, rows = kept
        T = normed.shape[0]
        cd, gd, hd, rd = self._descs(T, sequences)
        g = {k: torch.empty(v.shape, device=v.device) for k, v in p.items() if not k.startswith("w_")}
        dout, dtotal = self._new(T, self.M), self._new(T, self.M)
        dw.rnorm_bwd(rd, out, summed, dout, self._space(dw.rnorm_bwd_workspace_bytes(rd)), dy=dfollowing, dtotal=dsummed, w1=p["post_w"], scale=p["scale"],
                     w2=p["next_w"], rstd1=r1, rstd2=r2, dresidual=dtotal, dw1=g["post_w"], dscale=g["scale"], dw2=g["next_w"])
        g["w_out"] = o.t() @ dout
        do, dy, dproj, du = dout @ p["w_out"].t(), self._new(T, self.values), torch.empty_like(proj), torch.empty_like(u)
        q, k, v, z, a, b = self._parts(proj, u)
        dq, dk, dv, dz, da, db = self._parts(dproj, du)
        dw.hnorm_bwd(hd, y, p["head_w"], rstd, do, dy, g["head_w"], self._space(dw.hnorm_bwd_workspace_bytes(hd)), z=z, dz=dz)
        A = -torch.exp(p["A_log"])
        dw.gdelta_bwd(gd, q, k, v, a, b, kept, dy, dq, dk, dv, da, db, self._space(dw.gdelta_bwd_workspace_bytes(gd)), A=A, a_bias=p["a_bias"], starts=starts,
                      dA=g["A_log"], da_bias=g["a_bias"])
        g["A_log"].mul_(A)
        dw.cconv_bwd(cd, proj[:, :self.C], p["conv_w"], None, du, dproj[:, :self.C], g["conv_w"], None, self._space(dw.cconv_bwd_workspace_bytes(cd)),
                     starts=starts, init=rows)
        g["w_in"] = normed.t() @ dproj
        return dproj @ p["w_in"].t(), dtotal, g

    def step(self, normed, total, states, slots=None):
        """(normed, total) for one new token of each row; the rows' states are moved on in place."""
        p, T = self.p, normed.shape[0]
        rows, S = states
        cd, gd, hd, rd = self._descs(T, rows.shape[0])
        proj = normed @ p["w_in"]
        u, y, o = self._new(T, self.C), self._new(T, self.values), self._new(T, self.values)
        dw.cconv_step(cd, proj[:, :self.C], p["conv_w"], None, rows, u, slots=slots)
        q, k, v, z, a, b = self._parts(proj, u)
        dw.gdelta_step(gd, q, k, v, a, b, S, y, A=-torch.exp(p["A_log"]), a_bias=p["a_bias"], slots=slots)
        dw.hnorm_fwd(hd, y, p["head_w"], o, z=z)
        following, summed = self._new(T, self.M), self._new(T, self.M)
        dw.rnorm_fwd(rd, o @ p["w_out"], summed, y=following, w1=p["post_w"], scale=p["scale"], residual=total, w2=p["next_w"])
        return following, summed


class DeltaMixer:
    """A stack of blocks, the norm in front of the first and, of each, the one behind it."""

    def __init__(self, width, blocks, heads, key_heads, K, V, taps=4, dtype=torch.bfloat16, seed=0, device="cuda"):
        self.blocks = [DeltaBlock(width, heads, key_heads, K, V, taps, dtype, seed + i, device) for i in range(blocks)]
        self.M, self.first_w = width, torch.ones(width, device=device, dtype=dtype)

    def states(self, sequences):
        return [b.states(sequences) for b in self.blocks]

    def _first(self, x):
        d, total, normed = dw.rnorm_desc(x.shape[0], self.M, self.blocks[0].kind, post=False), torch.empty_like(x), torch.empty_like(x)
        rstd = torch.empty(x.shape[0], device=x.device)
        dw.rnorm_fwd(d, x, total, y=normed, w2=self.first_w, rstd2=rstd)
        return d, total, normed, rstd

    def forward(self, x, starts=None, sequences=1, states=None, keep=False):
        """The normalised rows behind the last block, for T packed tokens; with keep (rows, what `backward` takes)."""
        d, total, normed, rstd = self._first(x)
        kept = [(d, x, total, rstd)]
        for i, block in enumerate(self.blocks):
            normed, total, *more = block.forward(normed, total, starts, sequences, None if states is None else states[i], keep)
            kept += more
        return (normed, kept) if keep else normed

    def backward(self, dy, kept):
        """(the gradient of x, that of the first norm's weight, the gradients of each block's parameters)"""
        dtotal, grads = None, []
        for block, k in zip(reversed(self.blocks), reversed(kept[1:])):
            dy, dtotal, g = block.backward(dy, dtotal, k)
            grads.insert(0, g)
        d, x, total, rstd = kept[0]
        dx, dfirst = torch.empty_like(x), torch.empty(self.M, device=x.device)
        space = torch.empty(max(dw.rnorm_bwd_workspace_bytes(d), 16), device=x.device, dtype=torch.uint8)
        dw.rnorm_bwd(d, x, total, dx, space, dy=dy, dtotal=dtotal, w2=self.first_w, rstd2=rstd, dw2=dfirst)
        return dx, dfirst, grads

    def step(self, x, states, slots=None):
        """The normalised rows behind the last block for one new token of each row of x."""
        _, total, normed, _ = self._first(x)
        for block, s in zip(self.blocks, states):
            normed, total = block.step(normed, total, s, slots)
        return normed


def train_step(stack, x, target, starts, sequences, rate):
    """One step of gradient descent, `rate` times the gradient's direction, on the mean square of the stack's output's distance from target; the loss."""
    y, kept = stack.forward(x, starts, sequences, keep=True)
    off = y.float() - target
    _, dfirst, grads = stack.backward((off * (2.0 / off.numel())).to(x.dtype), kept)
    found = [(stack.first_w, dfirst)] + [(b.p[k], g.float()) for b, gs in zip(stack.blocks, grads) for k, g in gs.items()]
    scale = -rate / torch.stack([g.square().sum() for _, g in found]).sum().sqrt()
    for v, g in found:
        v.add_((g * scale).to(v.dtype))
    return off.square().mean()


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--width", type=int, default=1024)
    ap.add_argument("--blocks", type=int, default=2)
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--steps", type=int, default=5)
    ap.add_argument("--generate", type=int, default=32)
    ap.add_argument("--rate", type=float, default=0.15)
    a = ap.parse_args(argv)
    dw.load()
    K = max(8, a.width // 8)
    stack = DeltaMixer(a.width, a.blocks, 8, 4, min(K, 128), min(K, 128))
    T, M = a.tokens, a.width
    bounds = [0, T // 5, T // 5, T // 2, T]                      # packed sequences, one of them empty
    starts = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, M, generator=gen, device="cuda").to(torch.bfloat16)
    target = torch.cumsum(x.float(), 0).mul_(T ** -0.5)          # something that needs what came before
    losses, ms = [], []
    for _ in range(a.steps):
        torch.cuda.synchronize()
        t = time.perf_counter()
        loss = train_step(stack, x, target, starts, len(bounds) - 1, a.rate)
        torch.cuda.synchronize()
        ms.append((time.perf_counter() - t) * 1e3)
        losses.append(float(loss))
        print("step %d: loss %.5f, %.2f ms" % (len(losses), losses[-1], ms[-1]), flush=True)

    # prompts, then tokens one at a time, against all of it read at once
    rows, length, new = 4, T // 8, a.generate
    seqs = torch.randn(rows, length + new, M, generator=gen, device="cuda").to(torch.bfloat16)

    def read(tokens, states):
        return stack.forward(tokens.reshape(-1, M), sequences=rows, states=states).float().reshape(rows, -1, M)

    whole = read(seqs.contiguous(), stack.states(rows))
    states = stack.states(rows)
    read(seqs[:, :length].contiguous(), states)
    off, spent = 0.0, []
    for t in range(new):
        torch.cuda.synchronize()
        began = time.perf_counter()
        y = stack.step(seqs[:, length + t].contiguous(), states)
        torch.cuda.synchronize()
        spent.append((time.perf_counter() - began) * 1e6)
        want = whole[:, length + t]
        diff = float((y.float() - want).abs().max() / want.abs().max())
        assert math.isfinite(diff), "not a number at token %d" % t
        off = max(off, diff)
    print(json.dumps({"width": M, "blocks": a.blocks, "tokens": T, "loss_first": round(losses[0], 5), "loss_last": round(losses[-1], 5),
                      "ms_per_training_step": round(sorted(ms)[len(ms) // 2], 3), "us_per_generated_token_of_%d_rows" % rows: round(sorted(spent)[len(spent) // 2], 1),
                      "generated_against_read_at_once": round(off, 5)}))
    return losses, off


if __name__ == "__main__":
    main()
