"""Sizes that the descriptors of the sequence operators accept and that take more lanes than one launch has (2^32 - 1): nothing is refused, and the pieces meet without a gap.
Tolerances as in test_gpu_sequence.py."""
import numpy as np
import pytest
import torch

import paper_1803_09926_amd as dw
from oracle import sequence as seq

import gpu_util as gu

pytestmark = pytest.mark.gpu


def _space(n):
    return torch.empty(max(n, 16), device="cuda", dtype=torch.uint8)


@pytest.mark.parametrize("C", [8, 3])
def test_layer_norm_of_more_rows_than_lanes(gpu_lib, C):
    """A wavefront a row: 2^26 - 4 rows fill a launch."""
    T, most = (1 << 26) + 33, (1 << 26) - 4
    gen = torch.Generator(device="cuda").manual_seed(1)
    x, r = (torch.randint(-8, 9, (T, C), generator=gen, device="cuda", dtype=torch.int8).to(torch.bfloat16) for _ in range(2))
    w = torch.randn(C, generator=gen, device="cuda").to(torch.bfloat16)
    y, total = (torch.full_like(x, float("nan")) for _ in range(2))
    mean, rstd = (torch.full((T,), float("nan"), device="cuda") for _ in range(2))
    print("norm of", T, "rows", flush=True)
    dw.lnorm_fwd(dw.lnorm_desc(T, C, dw.BF16), x, w, None, y, mean, rstd, residual=r, total=total)
    assert torch.equal(total, x + r)                                  # (small whole numbers: exact)
    assert torch.isfinite(mean).all() and torch.isfinite(rstd).all()
    for lo in (0, most - 17, T - 40):
        rows = slice(lo, lo + 40)
        want = seq.layer_norm(gu.to_host(x[rows]), gu.to_host(w), None, 1e-5, gu.to_host(r[rows]))
        for got, ref, tol in ((y, want[0], 1e-2), (mean, want[1], 1e-5), (rstd, want[2], 1e-5)):
            gu.assert_close(gu.to_host(got[rows]), ref, tol, "rows from %d" % lo)
    dx, gw, gb = torch.full_like(x, float("nan")), torch.empty(C, device="cuda"), torch.empty(C, device="cuda")
    d = dw.lnorm_desc(T, C, dw.BF16)
    dw.lnorm_bwd(d, total, w, mean, rstd, x, dx, gw, gb, _space(dw.lnorm_bwd_workspace_bytes(d)), dtotal=r)
    rows = slice(T - 40, T)
    want = seq.layer_norm_bwd(gu.to_host(total[rows]), gu.to_host(w), gu.to_host(mean[rows]), gu.to_host(rstd[rows]), gu.to_host(x[rows]), gu.to_host(r[rows]))
    gu.assert_close(gu.to_host(dx[rows]), want[0], 1e-2, "dx")
    # whole numbers, whose sums a lane keeps in 32 bits over some 2^15 rows; against 64 bits
    assert float((gb.double() - x.double().sum(0)).abs().max()) <= 2e-5 * float(x.double().sum(0).abs().max().clamp(min=1.0)) + 1.0


def test_conv_step_of_more_rows_than_lanes(gpu_lib):
    """A block of 64 lanes a row: 2^26 - 1 rows fill a launch."""
    T, most = (1 << 26) + 70, (1 << 26) - 1
    gen = torch.Generator(device="cuda").manual_seed(2)
    x, state = torch.randn(T, 1, generator=gen, device="cuda"), torch.randn(T, 1, 1, generator=gen, device="cuda")
    w = torch.tensor([[0.5], [-1.5]], device="cuda")
    before, y = state.clone(), torch.full_like(x, float("nan"))
    print("convolution of", T, "rows", flush=True)
    dw.cconv_step(dw.cconv_desc(T, 1, 2, T, dw.F32, False), x, w, None, state, y)
    assert torch.equal(state.view(T, 1), x)
    off = (y - (0.5 * before.view(T, 1) - 1.5 * x)).abs()
    assert float(off.max()) <= 1e-5                                   # two products and a sum of numbers up to 12
    slots = torch.arange(T, device="cuda", dtype=torch.int32).flip(0)
    slots[most] = -1
    state.copy_(before)
    dw.cconv_step(dw.cconv_desc(T, 1, 2, T, dw.F32, False), x, w, None, state, y, slots=slots)
    keep = torch.ones(T, dtype=torch.bool, device="cuda")
    keep[most] = False
    want = 0.5 * before.view(T, 1).flip(0) - 1.5 * x
    assert float((y - want)[keep].abs().max()) <= 1e-5 and float(y[most]) == 0.0
    at = T - 1 - most
    assert float(state[at]) == float(before[at]) and torch.equal(state[at + 1:].view(-1), x[:most].flip(0).view(-1))


def test_scan_step_of_more_rows_than_lanes(gpu_lib):
    """A block of 256 lanes a row: 2^24 - 1 rows fill a launch."""
    T = (1 << 24) + 70
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, dt, B, C, z = (torch.randn(T, 1, generator=gen, device="cuda") for _ in range(5))
    state = torch.randn(T, 1, 1, generator=gen, device="cuda")
    A = torch.tensor([[-0.5]], device="cuda")
    before, y = state.clone(), torch.full_like(x, float("nan"))
    d = dw.sscan_desc(T, 1, 1, 1, T, dw.F32, False)
    print("scan of", T, "rows", flush=True)
    dt = dt.abs()
    dw.sscan_step(d, x, dt, A, B, C, state, y, z=z)
    h = torch.exp(dt.double() * -0.5) * before.view(T, 1).double() + (dt * x * B).double()
    want = h * C.double() * torch.nn.functional.silu(z.double())
    assert float((state.view(T, 1).double() - h).norm() / h.norm()) <= 2e-5 and float((y.double() - want).norm() / want.norm()) <= 2e-5
    assert float((state.view(T, 1).double() - h).abs().max() / h.abs().max()) <= 2e-5 and float((y.double() - want).abs().max() / want.abs().max()) <= 2e-5


def test_scan_gradients_of_more_shared_values_than_lanes(gpu_lib):
    """2^32 values of dB and dC, a lane each."""
    T, G, N, last, back = 1 << 21, 32, 32, 40, 300
    gen = torch.Generator(device="cuda").manual_seed(4)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    x, dt, dy, B, C = normal(T, G), normal(T, G), normal(T, G), normal(T, G * N), normal(T, G * N)
    A = -1.0 - torch.rand(G, N, generator=gen, device="cuda")
    d = dw.sscan_desc(T, G, N, G, 1, dw.BF16)
    y, dx, ddt = (torch.empty_like(x) for _ in range(3))
    kept = _space(dw.sscan_kept_bytes(d))
    print("scan of", T, "tokens", flush=True)
    dw.sscan_fwd(d, x, dt, A, B, C, y, _space(dw.sscan_fwd_workspace_bytes(d)), kept=kept)
    dA, dB, dC = torch.empty_like(A), torch.full_like(B, float("nan")), torch.full_like(C, float("nan"))
    dw.sscan_bwd(d, x, dt, A, B, C, kept, dy, dx, ddt, dA, dB, dC, _space(dw.sscan_bwd_workspace_bytes(d)))
    torch.cuda.synchronize()
    assert not torch.isnan(dB[T // 2 - 5:]).any() and not torch.isnan(dC[T // 2 - 5:]).any()
    # the last tokens depend on those far before them by less than exp(-0.8 * 260), as softplus(dt) is 0.8 on average
    rows = {k: gu.to_host(v[T - back:]) for k, v in (("x", x), ("dt", dt), ("dy", dy))}
    ref = seq.scan_bwd(rows["x"], rows["dt"], gu.to_host(A), gu.to_host(B[T - back:]).reshape(back, G, N), gu.to_host(C[T - back:]).reshape(back, G, N), [0, back],
                       rows["dy"])
    for got, k in ((dB, "dB"), (dC, "dC"), (dx, "dx"), (ddt, "ddt")):
        gu.assert_close(gu.to_host(got[T - last:]), ref[k][back - last:].reshape(last, -1), 1e-2, k)


def test_scan_gradients_of_more_parameters_than_lanes(gpu_lib):
    """2^30 + 2^25 sums over tokens, 64 of them a block."""
    C, N = 1 << 24, 64
    gen = torch.Generator(device="cuda").manual_seed(5)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda", dtype=torch.bfloat16)

    x, dt, dy, B, Cm = normal(1, C), normal(1, C), normal(1, C), normal(1, N), normal(1, N)
    A, D = torch.zeros(C, N, device="cuda"), torch.ones(C, device="cuda")
    d = dw.sscan_desc(1, C, N, 1, 1, dw.BF16, False)
    y, dx, ddt = (torch.full_like(x, float("nan")) for _ in range(3))
    kept = _space(dw.sscan_kept_bytes(d))
    print("scan of", C, "channels", flush=True)
    dw.sscan_fwd(d, x, dt, A, B, Cm, y, _space(dw.sscan_fwd_workspace_bytes(d)), D=D, kept=kept)
    nan = float("nan")
    dA, dD, db, dB, dC = torch.full_like(A, nan), torch.full_like(D, nan), torch.full_like(D, nan), torch.empty_like(B), torch.empty_like(Cm)
    dw.sscan_bwd(d, x, dt, A, B, Cm, kept, dy, dx, ddt, dA, dB, dC, _space(dw.sscan_bwd_workspace_bytes(d)), D=D, dD=dD, ddt_bias=db)
    torch.cuda.synchronize()
    assert torch.equal(dD, (dy.float() * x.float())[0])               # one token: one product
    assert not dA.any()                                               # and nothing before it that could decay
    bc = float((B.double() * Cm.double()).sum())
    want = dy.double() * x.double() * bc                              # of the step size
    assert float((db.double() - want[0]).abs().max() / want.abs().max()) <= 2e-5
