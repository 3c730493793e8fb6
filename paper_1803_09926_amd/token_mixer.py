"""A block over token sequences from this library's operators: layer norm, a projection to the input and its gate, the short causal depthwise convolution,
the projections that give the scan its step sizes, B and C, the selective state space scan, and the projection back.

The dense projections are plain matrix products (torch.mm, a library's); everything else runs on the kernels of this package.  A block trains on packed sequences
(`forward` with keep=True, then `backward`), reads prompts (`forward` with `states`), and generates token by token (`step`); it keeps the residual stream apart, so that its sum
is taken inside the next block's norm.

Usage:  python -m paper_1803_09926_amd.token_mixer [--width 1024] [--blocks 2] [--tokens 4096] [--steps 5] [--generate 32]
Trains a stack on synthetic sequences, then continues prompts and checks the tokens generated one at a time against the prompt read at once.
"""
from __future__ import annotations

import argparse
import json
import math
import time

import torch

import paper_1803_09926_amd as dw


class TokenMixer:
    """One block of `width` channels, 2 * width inside."""

    def __init__(self, width, states=16, taps=4, dtype=torch.bfloat16, seed=0, device="cuda"):
        self.M, self.C, self.N, self.K, self.R = width, 2 * width, states, taps, max(1, width // 16)
        self.dtype, self.kind = dtype, dw.F32 if dtype == torch.float32 else dw.BF16
        M, C, N, K, R = self.M, self.C, self.N, self.K, self.R
        g = torch.Generator().manual_seed(seed)

        def normal(*shape, scale):
            return (torch.randn(*shape, generator=g) * scale).to(device=device, dtype=dtype)

        dt = torch.exp(torch.rand(C, generator=g) * (math.log(0.1) - math.log(1e-3)) + math.log(1e-3))
        self.p = {"norm_w": torch.ones(M, device=device, dtype=dtype), "norm_b": torch.zeros(M, device=device, dtype=dtype),
                  "w_in": normal(M, 2 * C, scale=M ** -0.5), "conv_w": normal(K, C, scale=K ** -0.5), "conv_b": torch.zeros(C, device=device, dtype=dtype),
                  "w_x": normal(C, R + 2 * N, scale=C ** -0.5), "w_dt": normal(R, C, scale=R ** -0.5),
                  "dt_bias": (dt + torch.log(-torch.expm1(-dt))).to(device), "A_log": torch.log(torch.arange(1, N + 1, device=device, dtype=torch.float32)).repeat(C, 1),
                  "D": torch.ones(C, device=device), "w_out": normal(C, M, scale=0.5 * C ** -0.5)}
        self.kept, self._read, self._unread = None, False, 0         # of the last forward(keep=True): whether `backward` had it, and how many it has not had

    def _space(self, nbytes):
        """A workspace for one call.  torch's allocator hands it out again behind that call on the same stream; one that the block held would be written by calls on
        two streams at once."""
        return torch.empty(max(nbytes, 16), device=self.p["D"].device, dtype=torch.uint8)

    def _new(self, *shape, like=None):
        return torch.empty(*shape, device=self.p["D"].device, dtype=like or self.dtype)

    def states(self, sequences):
        """States of sequences that start: the convolution's last rows and the scan's states, as forward and step take them."""
        return (torch.zeros(sequences, self.K - 1, self.C, device=self.p["D"].device, dtype=self.dtype),
                torch.zeros(sequences, self.C, self.N, device=self.p["D"].device))

    def _descs(self, T, sequences):
        C, wide = self.C, self.R + 2 * self.N
        return (dw.lnorm_desc(T, self.M, self.kind), dw.cconv_desc(T, C, self.K, sequences, self.kind, x_stride=2 * C),
                dw.sscan_desc(T, C, self.N, 1, sequences, self.kind, z_stride=2 * C, b_stride=wide, c_stride=wide))

    def _decay(self):
        """A of the scan: below zero whatever is learnt."""
        return -torch.exp(self.p["A_log"])

    def _projected(self, u):
        """(all that w_x gives, dt, B, C)"""
        p = u @ self.p["w_x"]
        R, N = self.R, self.N
        return p, p[:, :R] @ self.p["w_dt"], p[:, R:R + N], p[:, R + N:]

    def forward(self, hidden, residual=None, starts=None, sequences=1, states=None, keep=False):
        """(hidden, residual) after the block, for T packed tokens.  states: continues these sequences, and moves them on.  keep: for `backward`, to which
        the states that the sequences began with are constants; what it needs is in `kept` until the next forward with keep."""
        p, T, C = self.p, hidden.shape[0], self.C
        nd, cd, sd = self._descs(T, sequences)
        normed, total = self._new(T, self.M), hidden if residual is None else self._new(T, self.M)
        mean, rstd = self._new(T, like=torch.float32), self._new(T, like=torch.float32)
        dw.lnorm_fwd(nd, hidden, p["norm_w"], p["norm_b"], normed, mean, rstd, residual=residual, total=None if residual is None else total)
        xz = normed @ p["w_in"]
        u, y = self._new(T, C), self._new(T, C)
        rows, h = states if states is not None else (None, None)
        new_rows, new_h = (torch.empty_like(rows), torch.empty_like(h)) if states is not None else (None, None)
        dw.cconv_fwd(cd, xz[:, :C], p["conv_w"], p["conv_b"], u, starts=starts, init=rows, final=new_rows)
        proj, dt, B, Cm = self._projected(u)
        kept = torch.empty(max(dw.sscan_kept_bytes(sd), 16), device=u.device, dtype=torch.uint8) if keep else None
        dw.sscan_fwd(sd, u, dt, self._decay(), B, Cm, y, self._space(dw.sscan_fwd_workspace_bytes(sd)), D=p["D"], z=xz[:, C:], dt_bias=p["dt_bias"],
                     starts=starts, init=h, final=new_h, kept=kept)
        began = (rows.clone(), h.clone()) if keep and states is not None else (None, None)
        if states is not None:
            rows.copy_(new_rows)
            h.copy_(new_h)
        if keep:
            self._read, self._unread = False, self._unread + 1
            self.kept = (total, normed, mean, rstd, xz, u, proj, dt, kept, y, starts, sequences, began)
        return y @ p["w_out"], total

    def backward(self, dhidden, dresidual=None, kept=None):
        """From the gradients of what `forward` gave to (the gradient of hidden and residual alike, the gradients by parameter).  kept: what the block's `kept` was
        behind that forward, where another one with keep has come since."""
        p, C, R, N = self.p, self.C, self.R, self.N
        if kept is None:
            if self.kept is None:
                raise RuntimeError("no forward(keep=True) came before")
            if self._read and self._unread:
                raise RuntimeError("an earlier forward's activations were replaced by a later one's: take `kept` behind each forward(keep=True) and hand it to backward")
            kept = self.kept
        self._read, self._unread = self._read or kept is self.kept, max(0, self._unread - 1)
        total, normed, mean, rstd, xz, u, proj, dt, kept, y, starts, sequences, (rows, h) = kept
        T = total.shape[0]
        nd, cd, sd = self._descs(T, sequences)
        g = {k: torch.empty(v.shape, device=v.device) for k, v in p.items() if not k.startswith("w_")}
        g["w_out"] = y.t() @ dhidden
        dy = dhidden @ p["w_out"].t()
        du, ddt, dproj, dxz = self._new(T, C), self._new(T, C), torch.empty_like(proj), torch.empty_like(xz)
        A = self._decay()
        dw.sscan_bwd(sd, u, dt, A, proj[:, R:R + N], proj[:, R + N:], kept, dy, du, ddt, g["A_log"], dproj[:, R:R + N], dproj[:, R + N:],
                     self._space(dw.sscan_bwd_workspace_bytes(sd)), D=p["D"], z=xz[:, C:], dt_bias=p["dt_bias"], starts=starts, init=h, dD=g["D"],
                     dz=dxz[:, C:], ddt_bias=g["dt_bias"])
        g["A_log"].mul_(A)
        g["w_dt"] = proj[:, :R].t() @ ddt
        dproj[:, :R] = ddt @ p["w_dt"].t()
        g["w_x"] = u.t() @ dproj
        du.addmm_(dproj, p["w_x"].t())
        dw.cconv_bwd(cd, xz[:, :C], p["conv_w"], p["conv_b"], du, dxz[:, :C], g["conv_w"], g["conv_b"],
                     self._space(dw.cconv_bwd_workspace_bytes(cd)), starts=starts, init=rows)
        g["w_in"] = normed.t() @ dxz
        dnormed, dx = dxz @ p["w_in"].t(), self._new(T, self.M)
        dw.lnorm_bwd(nd, total, p["norm_w"], mean, rstd, dnormed, dx, g["norm_w"], g["norm_b"], self._space(dw.lnorm_bwd_workspace_bytes(nd)),
                     dtotal=dresidual)
        return dx, g

    def step(self, hidden, residual, states, slots=None):
        """(hidden, residual) for one new token of each row; the rows' states are moved on in place."""
        p, T, C = self.p, hidden.shape[0], self.C
        rows, h = states
        nd, cd, sd = self._descs(T, rows.shape[0])
        normed, total = self._new(T, self.M), hidden if residual is None else self._new(T, self.M)
        dw.lnorm_fwd(nd, hidden, p["norm_w"], p["norm_b"], normed, residual=residual, total=None if residual is None else total)
        xz = normed @ p["w_in"]
        u, y = self._new(T, C), self._new(T, C)
        dw.cconv_step(cd, xz[:, :C], p["conv_w"], p["conv_b"], rows, u, slots=slots)
        _, dt, B, Cm = self._projected(u)
        dw.sscan_step(sd, u, dt, self._decay(), B, Cm, h, y, D=p["D"], z=xz[:, C:], dt_bias=p["dt_bias"], slots=slots)
        return y @ p["w_out"], total


def train_step(stack, x, target, starts, sequences, rate):
    """One step of gradient descent of the stack, `rate` times the gradient's direction, on the mean square of its output's distance from target; the loss."""
    hidden, residual = x, None
    for block in stack:
        hidden, residual = block.forward(hidden, residual, starts, sequences, keep=True)
    off = hidden.float() + residual.float() - target
    grad = (off * (2.0 / off.numel())).to(x.dtype)
    dhidden, dresidual, found = grad, grad, []
    for block in reversed(stack):
        dresidual, grads = block.backward(dhidden, dresidual)
        dhidden = dresidual
        found += [(block.p[k], g.float()) for k, g in grads.items()]
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
    stack = [TokenMixer(a.width, seed=i) for i in range(a.blocks)]
    T, M = a.tokens, a.width
    bounds = [0, T // 5, T // 5, T // 2, T]                          # packed sequences, one of them empty
    starts = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(T, M, generator=gen, device="cuda").to(torch.bfloat16)
    target = torch.cumsum(x.float(), 0).mul_(T ** -0.5)              # something that needs what came before
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
        hidden, residual = tokens.reshape(-1, M), None
        for block, s in zip(stack, states):
            hidden, residual = block.forward(hidden, residual, sequences=rows, states=s)
        return (hidden.float() + residual.float()).reshape(rows, -1, M)

    whole = read(seqs.contiguous(), [b.states(rows) for b in stack])
    states = [b.states(rows) for b in stack]
    read(seqs[:, :length].contiguous(), states)
    off, spent = 0.0, []
    for t in range(new):
        torch.cuda.synchronize()
        began = time.perf_counter()
        hidden, residual = seqs[:, length + t].contiguous(), None
        for block, s in zip(stack, states):
            hidden, residual = block.step(hidden, residual, s)
        torch.cuda.synchronize()
        spent.append((time.perf_counter() - began) * 1e6)
        want = whole[:, length + t]
        diff = float((hidden.float() + residual.float() - want).abs().max() / want.abs().max())
        assert math.isfinite(diff), "not a number at token %d" % t
        off = max(off, diff)
    print(json.dumps({"width": M, "blocks": a.blocks, "tokens": T, "loss_first": round(losses[0], 5), "loss_last": round(losses[-1], 5),
                      "ms_per_training_step": round(sorted(ms)[len(ms) // 2], 3), "us_per_generated_token_of_%d_rows" % rows: round(sorted(spent)[len(spent) // 2], 1),
                      "generated_against_read_at_once": round(off, 5)}))
    return losses, off


if __name__ == "__main__":
    main()
