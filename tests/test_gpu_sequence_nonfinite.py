"""Infinities in the selective scan: every output is infinite, not a number or finite where the formula in 64 bits is, whatever the number of states and channels leaves
of the kernels' lanes, and the finite ones are as near as without them."""
import numpy as np
import pytest
import torch

import paper_1803_09926_amd as dw
from oracle import sequence as seq

import gpu_util as gu

pytestmark = pytest.mark.gpu

TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}
TOL = {"f32": 2e-5, "bf16": 1e-2}      # as for finite inputs: 300 tokens whose state is rounded 3 times each, or one rounding to bf16


def _space(n):
    return torch.full((max(n, 16),), 0xFF, device="cuda", dtype=torch.uint8)


def _same(got, want, tol, what):
    got, want = gu.to_host(got).astype(np.float64).reshape(want.shape), np.asarray(want)
    assert np.array_equal(np.isnan(got), np.isnan(want)), what + ": not a number"
    assert np.array_equal(np.where(np.isinf(got), np.sign(got), 0), np.where(np.isinf(want), np.sign(want), 0)), what + ": infinite"
    there = np.isfinite(want)
    gu.assert_close(np.where(there, got, 0), np.where(there, want, 0), tol, what)


def _positive(seed, T, C, N, G, dtype):
    """Inputs of one sign, so that infinities of both do not meet in a sum: by name, rounded as the call has them."""
    r = np.random.default_rng(seed)

    def made(*shape, lo=0.1, hi=1.0, stored=True):
        t = torch.from_numpy(r.uniform(lo, hi, shape).astype(np.float32))
        return t.to(TORCH[dtype]).float().numpy() if stored else t.numpy()
    v = {"x": made(T, C), "dt": made(T, C, lo=-1.0), "B": made(T, G, N), "C": made(T, G, N), "A": -made(C, N, stored=False), "D": made(C, stored=False),
         "z": made(T, C), "dt_bias": made(C, stored=False)}
    return v, made(T, C)


def _both_ways(v, dy, bounds, G, dtype, softplus=True):
    """The kernels' outputs and the oracle's, by name."""
    T, C = v["x"].shape
    N, S = v["A"].shape[1], len(bounds) - 1
    d = dw.sscan_desc(T, C, N, G, S, {"f32": dw.F32, "bf16": dw.BF16}[dtype], softplus)
    on = {k: None if a is None else torch.from_numpy(np.ascontiguousarray(a)).cuda().to(TORCH[dtype] if k in ("x", "dt", "z", "B", "C") else torch.float32)
          for k, a in v.items()}
    starts = torch.tensor(bounds, dtype=torch.int32, device="cuda")
    call = (d, on["x"], on["dt"], on["A"], on["B"], on["C"])
    more = {"D": on["D"], "z": on["z"], "dt_bias": on["dt_bias"], "starts": starts}
    out = {"y": torch.empty_like(on["x"]), "final": torch.empty(S, C, N, device="cuda")}
    kept = _space(dw.sscan_kept_bytes(d))
    dw.sscan_fwd(*call, out["y"], _space(dw.sscan_fwd_workspace_bytes(d)), final=out["final"], kept=kept, **more)
    for k in v:
        out["d" + k] = None if on[k] is None else torch.empty_like(on[k])
    dyd = torch.from_numpy(dy).cuda().to(TORCH[dtype])
    dw.sscan_bwd(*call, kept, dyd, out["dx"], out["ddt"], out["dA"], out["dB"], out["dC"], _space(dw.sscan_bwd_workspace_bytes(d)), dD=out["dD"], dz=out["dz"],
                 ddt_bias=out["ddt_bias"], **more)
    with np.errstate(all="ignore"):
        y, final, _ = seq.scan(bounds=bounds, softplus=softplus, **v)
        want = {"y": y, "final": final, **seq.scan_bwd(bounds=bounds, dy=dy, softplus=softplus, **v)}
    return {k: (out[k], want[k]) for k in out if out[k] is not None}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("where", ["x", "B", "one B", "C", "dt", "dy"])
@pytest.mark.parametrize("N", [1, 2, 3, 5, 8, 9, 16, 24, 33, 64])
@pytest.mark.parametrize("C,G", [(70, 1), (24, 2)])
def test_infinities_where_states_or_channels_are_padded(gpu_lib, dtype, where, N, C, G):
    bounds, T, at = [0, 26, 26, 50], 50, 7
    v, dy = _positive(N + C, T, C, N, G, dtype)
    if where == "B" or where == "C":
        v[where][at] = np.inf
    elif where == "one B":
        v["B"][at, G - 1, N // 2] = np.inf
    elif where == "dy":
        dy[at, 3] = np.inf
    else:
        v[where][at, 3] = np.inf
    for k, (got, want) in _both_ways(v, dy, bounds, G, dtype).items():
        tol = TOL["f32"] if got.dtype == torch.float32 else TOL[dtype]
        _same(got, want, tol, "%s of %d states, %d channels, infinite %s" % (k, N, C, where))


@pytest.mark.parametrize("N", [5, 16])
def test_an_infinite_input_without_a_direct_term(gpu_lib, N):
    v, dy = _positive(N, 40, 24, N, 1, "f32")
    v["D"] = None
    v["x"][9, 3] = np.inf
    for k, (got, want) in _both_ways(v, dy, [0, 40], 1, "f32").items():
        _same(got, want, TOL["f32"], k)


@pytest.mark.parametrize("N", [1, 3, 16])
def test_an_infinite_input_of_a_step(gpu_lib, N):
    C = 20
    v, _ = _positive(N, 1, C, N, 1, "f32")
    v["x"][0, 3] = np.inf
    h0 = np.ones((1, C, N), np.float32)
    on = {k: torch.from_numpy(a).cuda() for k, a in v.items()}
    state, y = torch.from_numpy(h0).cuda(), torch.empty(1, C, device="cuda")
    dw.sscan_step(dw.sscan_desc(1, C, N, 1, 1), on["x"], on["dt"], on["A"], on["B"], on["C"], state, y, D=on["D"], z=on["z"], dt_bias=on["dt_bias"])
    want, final, _ = seq.scan(bounds=[0, 1], init=h0, **v)
    _same(y, want, 2e-5, "y")
    _same(state, final, 2e-5, "state")
