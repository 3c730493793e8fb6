"""GPU parity of the heads' norm and of the norms around a block with their oracle in 64 bits, forward and backward.

Tolerances as in test_gpu_sequence.py: bf16 outputs are rounded once, to 2^-9 of themselves (1e-2 in both norms); fp32: sums of at most 8192 terms in a tree twice over, 13 * 2^-24 each, and
an exponential and a reciprocal of 1 ulp: 1e-5; sums over tokens 2e-5."""
import numpy as np
import pytest
import torch

import paper_1803_09926_amd as dw
from oracle import delta as od

import gpu_util as gu
from test_gpu_sequence import Made, _close, _space

pytestmark = pytest.mark.gpu

TOL = {"f32": 1e-5, "bf16": 1e-2}
DTYPE = {"f32": dw.F32, "bf16": dw.BF16}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [1, 3, 8, 16, 31, 32, 33, 64, 100, 128, 129, 256, 257, 512, 513, 1000, 1024])
@pytest.mark.parametrize("T,H,gate,w,more,shift,silu", [(1, 1, True, True, 0, 0, True), (7, 3, True, True, 5, 1, False), (37, 2, False, True, 8, 0, True),
                                                        (6, 5, True, False, 0, 0, True)])
def test_heads(gpu_lib, dtype, D, T, H, gate, w, more, shift, silu):
    print("heads", dtype, D, T, H, gate, w, more, shift, silu, flush=True)
    m = Made(D * 100 + T, dtype, shift)
    x, z, wt = m.host((T, H, D), 0.7), (m.host((T, H, D)) if gate else None), (m.host((D,), 0.2, 1.0) if w else None)
    width = H * D
    d = dw.hnorm_desc(T, H, D, DTYPE[dtype], 1e-6, silu, width + more, width + 2 * more, width + more)
    rows = lambda v, n=1: None if v is None else m.dev(v.reshape(T, width), rows=width + n * more)  # noqa: E731
    y, rstd = m.out((T, width), rows=width + more), m.out((T, H), False)
    xt, zt, wd = rows(x), rows(z, 2), None if wt is None else m.dev(wt)
    dw.hnorm_fwd(d, xt, wd, y, z=zt, rstd=rstd)
    want = od.heads_norm(x, wt, z, 1e-6, silu)
    _close(y, want[0], TOL[dtype], "y")
    _close(rstd, want[1], 1e-5, "rstd")
    dy = m.host((T, H, D))
    dx, gw = m.out((T, width), rows=width + more), (m.out((D,), False) if w else None)
    dz = m.out((T, width), rows=width + 2 * more) if gate else None
    dw.hnorm_bwd(d, xt, wd, rstd, rows(dy), dx, gw, _space(dw.hnorm_bwd_workspace_bytes(d)), z=zt, dz=dz)
    ref = od.heads_norm_bwd(x, wt, z, gu.to_host(rstd), dy, silu)
    if D > 1:                                    # (of one channel the gradient is nearly zero: what is left is rounding)
        _close(dx, ref[0], TOL[dtype], "dx")
    if w:
        _close(gw, ref[1], 2e-5, "dw")
    if gate:
        _close(dz, ref[2], TOL[dtype], "dz")


def test_heads_many_runs_and_none(gpu_lib):
    m = Made(5, "bf16")
    T, H, D = 4001, 6, 48
    x, z, dy = m.host((T, H, D)), m.host((T, H, D)), m.host((T, H, D))
    d = dw.hnorm_desc(T, H, D, dw.BF16)
    y, rstd, dx, dz, gw = m.out((T, H * D)), m.out((T, H), False), m.out((T, H * D)), m.out((T, H * D)), m.out((D,), False)
    dev = [m.dev(v.reshape(T, -1)) for v in (x, z, dy)]
    dw.hnorm_fwd(d, dev[0], None, y, z=dev[1], rstd=rstd)
    _close(y, od.heads_norm(x, None, z, 1e-6)[0], 1e-2, "y")
    dw.hnorm_bwd(d, dev[0], None, rstd, dev[2], dx, gw, _space(dw.hnorm_bwd_workspace_bytes(d)), z=dev[1], dz=dz)
    ref = od.heads_norm_bwd(x, None, z, gu.to_host(rstd), dy)
    for got, r, tol in ((dx, ref[0], 1e-2), (gw, ref[1], 2e-5), (dz, ref[2], 1e-2)):
        _close(got, r, tol, "gradients")
    d = dw.hnorm_desc(0, H, D, dw.BF16)
    none = dev[0][:0]
    dw.hnorm_fwd(d, none, None, none)
    dw.hnorm_bwd(d, none, None, rstd[:0], none, none, gw, None)
    assert not gw.any()


@pytest.mark.parametrize("op", ["heads", "block"])
def test_offsets_beyond_32_bits(gpu_lib, op):
    T, C = (1 << 21) + 5, 1032                   # 2.16e9 elements
    x = torch.zeros(T, C, device="cuda", dtype=torch.bfloat16)
    tail = torch.randn(7, C, device="cuda").to(torch.bfloat16)
    x[-7:] = tail
    y, dx = torch.empty_like(x), torch.empty_like(x)
    if op == "heads":
        d = dw.hnorm_desc(T, 8, 129, dw.BF16)
        rstd = torch.empty(T, 8, device="cuda")
        dw.hnorm_fwd(d, x, None, y, rstd=rstd)
        dw.hnorm_bwd(d, x, None, rstd, x, dx, None, None)
        h = gu.to_host(tail).reshape(7, 8, 129)
        want, r = od.heads_norm(h, None, None, 1e-6)
        _close(y[-7:], want, 1e-2, "the last rows")
        # (the gradient along itself is nearly zero: rounding of rstd * x, 2^-8 of the largest)
        assert float(dx[-7:].abs().max()) < 2 ** -7 * float((r.max() * np.abs(h).max()))
    else:
        d, total = dw.rnorm_desc(T, C, dw.BF16, alpha=0.5), torch.empty_like(x)
        dw.rnorm_fwd(d, x, total, y=y)
        want = od.block_norm(gu.to_host(tail), 1e-6, alpha=0.5)
        _close(y[-7:], want["y"], 1e-2, "the last rows")
        _close(total[-7:], want["total"], 1e-2, "the last rows' sums")
    assert not y[:3].any() and not y[T // 2:T // 2 + 3].any()


PARTS = [dict(post=True, z=True, scale=True, residual=True, y=True, w=True, dtotal=True), dict(post=True, z=False, scale=False, residual=True, y=True, w=True, dtotal=False),
         dict(post=False, z=True, scale=False, residual=False, y=True, w=False, dtotal=True), dict(post=True, z=False, scale=True, residual=True, y=False, w=True, dtotal=True),
         dict(post=False, z=False, scale=False, residual=True, y=True, w=True, dtotal=True), dict(post=False, z=False, scale=True, residual=True, y=False, w=False, dtotal=True)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", [1, 2, 7, 64, 65, 512, 513, 728, 1024, 1025, 2048, 2050, 4096, 4099, 8191, 8192])
@pytest.mark.parametrize("T,parts,more,shift,silu", [(1, 0, 0, 0, False), (5, 0, 8, 1, True), (37, 1, 0, 0, False), (6, 2, 3, 0, True), (9, 3, 0, 1, False),
                                                     (6, 4, 0, 0, False), (600, 5, 8, 0, False)])
def test_block(gpu_lib, dtype, C, T, parts, more, shift, silu):
    has = PARTS[parts]
    print("block", dtype, C, T, parts, more, shift, silu, flush=True)
    m = Made(C * 100 + T, dtype, shift)
    x, z = m.host((T, C), 0.8), (m.host((T, C)) if has["z"] else None)
    w1 = m.host((C,), 0.2, 1.0) if has["w"] and has["post"] else None
    w2 = m.host((C,), 0.2, 1.0) if has["w"] and has["y"] else None
    scale, residual = m.host((C,), 0.1, 0.5) if has["scale"] else None, m.host((T, C), 1.5) if has["residual"] else None
    kw = dict(post=has["post"], silu=silu, alpha=0.7)
    d = dw.rnorm_desc(T, C, DTYPE[dtype], 1e-6, **kw, x_stride=C + more, z_stride=C + 2 * more)
    dev = lambda v, n=0: None if v is None else m.dev(v, rows=C + n * more if n else None)  # noqa: E731
    given = {"w1": dev(w1), "z": dev(z, 2), "scale": dev(scale), "w2": dev(w2)}
    xt, total, y = dev(x, 1), m.out((T, C)), m.out((T, C)) if has["y"] else None
    r1, r2 = m.out((T,), False) if has["post"] else None, m.out((T,), False) if has["y"] else None
    dw.rnorm_fwd(d, xt, total, y=y, residual=dev(residual), rstd1=r1, rstd2=r2, **given)
    want = od.block_norm(x, 1e-6, w1, z, scale, residual, w2, **kw)
    for name, got in (("total", total), ("y", y), ("rstd1", r1), ("rstd2", r2)):
        if got is not None:
            _close(got, want[name], TOL["f32"] if got.dtype == torch.float32 else TOL[dtype], name)
    dy, dt = m.host((T, C)) if has["y"] else None, m.host((T, C)) if has["dtotal"] else None
    out = {"dx": m.out((T, C), rows=C + more), "dresidual": m.out((T, C)) if has["residual"] else None,
           "dz": m.out((T, C), rows=C + 2 * more) if has["z"] else None}
    out |= {k: None if v is None else m.out((C,), False) for k, v in (("dw1", w1), ("dscale", scale), ("dw2", w2))}
    dw.rnorm_bwd(d, xt, total, workspace=_space(dw.rnorm_bwd_workspace_bytes(d)), dy=dev(dy), dtotal=dev(dt), rstd1=r1, rstd2=r2, **given, **out)
    host = lambda t: None if t is None else gu.to_host(t)  # noqa: E731
    ref = od.block_norm_bwd(x, gu.to_host(total).reshape(T, C), host(r1), host(r2), dy, dt, w1, z, scale, w2, **kw)
    for name, got in out.items():
        if got is None or (C == 1 and name in ("dx", "dw1")):     # (of one channel the norm's gradient is nearly zero: what is left is rounding)
            continue
        if C == 1 and name == "dresidual" and dt is None:
            continue
        _close(got, ref[name], 2e-5 if got.dtype == torch.float32 and name[1] in "ws" else TOL[dtype], name)


def test_block_of_no_rows(gpu_lib):
    d, none = dw.rnorm_desc(0, 64), torch.empty(0, 64, device="cuda")
    w, g = torch.ones(64, device="cuda"), torch.full((64,), 3.0, device="cuda")
    dw.rnorm_fwd(d, none, none, y=none, w1=w)
    dw.rnorm_bwd(d, none, none, none, None, dy=none, w1=w, rstd1=none[:, 0], rstd2=none[:, 0], dw1=g)
    assert not g.any()


@pytest.mark.parametrize("value", [np.nan, np.inf])
def test_rows_are_apart(gpu_lib, value):
    """What is not finite in a row leaves the others' bits alone; rows that share a block among them."""
    m = Made(71, "bf16")
    T, C = 40, 384
    x, z, r = m.host((T, C)), m.host((T, C)), m.host((T, C))

    def run(x):
        d, total, y = dw.rnorm_desc(T, C, dw.BF16), m.out((T, C)), m.out((T, C))
        dw.rnorm_fwd(d, m.dev(x), total, y=y, z=m.dev(z), residual=m.dev(r))
        h, hy = dw.hnorm_desc(T, 8, 48, dw.BF16), m.out((T, C))
        dw.hnorm_fwd(h, m.dev(x), None, hy, z=m.dev(z))
        return gu.to_host(total), gu.to_host(y), gu.to_host(hy).reshape(T * 8, 48)

    was = run(x)
    x[17, 50] = value
    got = run(x)
    for a, b, n in zip(got, was, (17, 17, 17 * 8 + 1)):
        assert np.array_equal(np.delete(a, n, 0), np.delete(b, n, 0)) and not np.isfinite(a[n]).all()


def test_captured_and_replayed(gpu_lib):
    m = Made(73, "bf16")
    T, H, D = 300, 4, 64
    C = H * D
    x, z, dy, r = (m.dev(m.host((T, C))) for _ in range(4))
    w, wd = m.dev(m.host((C,))), m.dev(m.host((D,)))
    hd, rd = dw.hnorm_desc(T, H, D, dw.BF16), dw.rnorm_desc(T, C, dw.BF16)
    o = {k: m.out((T, C)) for k in ("y", "dx", "dz", "total", "ry", "rdx", "dr")}
    f = {"rstd": m.out((T, H), False), "dw": m.out((D,), False), "r1": m.out((T,), False), "r2": m.out((T,), False), "dw1": m.out((C,), False), "dw2": m.out((C,), False)}
    hs, rs = _space(dw.hnorm_bwd_workspace_bytes(hd)), _space(dw.rnorm_bwd_workspace_bytes(rd))

    def run():
        dw.hnorm_fwd(hd, x, wd, o["y"], z=z, rstd=f["rstd"])
        dw.hnorm_bwd(hd, x, wd, f["rstd"], dy, o["dx"], f["dw"], hs, z=z, dz=o["dz"])
        dw.rnorm_fwd(rd, x, o["total"], y=o["ry"], w1=w, residual=r, w2=w, rstd1=f["r1"], rstd2=f["r2"])
        dw.rnorm_bwd(rd, x, o["total"], o["rdx"], rs, dy=dy, w1=w, w2=w, rstd1=f["r1"], rstd2=f["r2"], dresidual=o["dr"], dw1=f["dw1"], dw2=f["dw2"])

    outs = list(o.values()) + list(f.values())
    run()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for _ in range(3):
        x.copy_(torch.randn(T, C, device="cuda"))
        run()
        want = [t.clone() for t in outs]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b)
