"""Paths of the sequence operators that the sizes of test_gpu_sequence.py do not reach: strips of every length in the causal convolution, more rows than teams in the
layer norm's backward pass, rows of y and dy apart, optional parts of the steps, backward passes beyond 32-bit offsets, and sequence starts of any contents.
Tolerances as there."""
import numpy as np
import pytest
import torch

import paper_1803_09926_amd as dw
from oracle import sequence as seq

import gpu_util as gu
from test_gpu_sequence import DTYPE, EVEN, RAGGED, TOL, TOL_SCAN, TOL_SUM, TORCH, Made, _close, _scan_made, _space, _starts

pytestmark = pytest.mark.gpu

# sequences of none, one and a few tokens, some that end with a strip and some inside, and one that is longer than the longest strip
BOUNDS = RAGGED + [301, 308, 308, 384, 385, 700, 700]


def _conv_both_ways(dtype, C, K, bounds, packed, carry, silu=True, bias=True, xs=None, ys=None, shift=0, seed=1):
    T, S = bounds[-1], len(bounds) - 1
    m = Made(seed, dtype, shift)
    x, w, b, dy = m.host((T, C)), m.host((K, C), 0.5), m.host((C,), 0.2) if bias else None, m.host((T, C))
    init = m.host((S, K - 1, C)) if carry else None
    d = dw.cconv_desc(T, C, K, S, DTYPE[dtype], silu, xs, ys)
    starts = _starts(bounds) if packed else None
    on = lambda v: None if v is None else m.dev(v)  # noqa: E731
    xd = m.dev(x, rows=xs)
    y, final = m.out((T, C), rows=ys), m.out((S, K - 1, C))
    dw.cconv_fwd(d, xd, on(w), on(b), y, starts=starts, init=on(init), final=final)
    wy, wf = seq.conv(x, w, b, bounds, init, silu)
    tag = " conv %s C %d K %d" % (dtype, C, K)
    _close(y, wy, TOL[dtype], "y" + tag)
    assert np.array_equal(gu.to_host(final), wf.astype(np.float32)), "final" + tag
    dx, gw, gb = m.out((T, C), rows=xs), m.out((K, C), False), m.out((C,), False)
    dw.cconv_bwd(d, xd, on(w), on(b), m.dev(dy, rows=ys), dx, gw, gb, _space(dw.cconv_bwd_workspace_bytes(d)), starts=starts, init=on(init))
    ref = seq.conv_bwd(x, w, b, bounds, dy, init, silu)
    for got, r, tol, name in ((dx, ref[0], TOL[dtype], "dx"), (gw, ref[1], TOL_SUM, "dw"), (gb, ref[2], TOL_SUM, "db")):
        _close(got, r, tol, name + tag)


# ---- causal convolution ----------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("strip", [1, 3, 4, 8, 12, 20, 32, 64, 128])
@pytest.mark.parametrize("K", range(2, 9))
def test_conv_strips_of_every_length(gpu_lib, dtype, strip, K):
    with dw.tuning_overrides({"DWCONV_TUNE_CCONV_STRIP": strip}):
        # a block has 256 strips of one channel vector, or 4 of 64: each leaves one row of partials
        d = dw.cconv_desc(700, 260, K, 1, DTYPE[dtype])
        assert dw.cconv_bwd_workspace_bytes(d) == -(-700 // (4 * strip)) * (K + 1) * 260 * 4
        _conv_both_ways(dtype, 36, K, BOUNDS, True, True, seed=K)
        _conv_both_ways(dtype, 261, K, BOUNDS, True, strip % 8 == 0, seed=K + 1)
        _conv_both_ways(dtype, 8, K, EVEN(600, 5), False, strip % 8 != 0, seed=K + 2)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", [4, 7])
def test_conv_strips_as_they_are_chosen(gpu_lib, dtype, K):
    """24 tokens a strip forward and 36 backward, by the number of tokens, without being told."""
    T, C = 40001, 264
    d = dw.cconv_desc(T, C, K, 3, DTYPE[dtype])
    assert dw.cconv_bwd_workspace_bytes(d) == -(-T // (4 * 36)) * (K + 1) * C * 4
    _conv_both_ways(dtype, C, K, [0, 20000, 20001, T], True, True, seed=K)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C,xs,ys,shift,silu,bias", [(8, None, 11, 0, True, True), (65, 70, 130, 1, False, False), (200, 400, 400, 0, True, False), (33, None, 40, 1, False, True)])
def test_conv_rows_apart_and_optional_parts(gpu_lib, dtype, C, xs, ys, shift, silu, bias):
    _conv_both_ways(dtype, C, 4, RAGGED, True, True, silu, bias, xs, ys, shift, seed=C)
    _conv_both_ways(dtype, C, 3, EVEN(120, 4), False, False, silu, bias, xs, ys, shift, seed=C + 1)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,C,K,silu,bias,ys", [(5, 33, 4, False, False, None), (9, 260, 3, False, True, 270), (4, 8, 8, True, False, 16)])
def test_conv_steps_without_slots_and_optional_parts(gpu_lib, dtype, T, C, K, silu, bias, ys):
    m = Made(T * C, dtype)
    S = T + 2
    x, w, b, state = m.host((T, C)), m.host((K, C)), m.host((C,)) if bias else None, m.host((S, K - 1, C))
    held, y = m.dev(state), m.out((T, C), rows=ys)
    dw.cconv_step(dw.cconv_desc(T, C, K, S, DTYPE[dtype], silu, None, ys), m.dev(x), m.dev(w), None if b is None else m.dev(b), held, y)
    want_y, final = seq.conv(x, w, b, list(range(T + 1)), state[:T], silu)
    _close(y, want_y, TOL[dtype], "y")
    assert np.array_equal(gu.to_host(held), np.concatenate([final.astype(np.float32), state[T:]]))


def test_conv_gradients_beyond_32_bit_offsets(gpu_lib):
    T, C, n = (1 << 21) + 9, 1024, 12
    x, dy = (torch.zeros(T, C, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    m = Made(31, "bf16")
    xt, dyt, w = m.host((n, C)), m.host((n, C)), m.host((4, C))
    x[-n:], dy[-n:] = m.dev(xt), m.dev(dyt)
    dx, gw, gb = torch.full_like(x, float("nan")), m.out((4, C), False), m.out((C,), False)
    d = dw.cconv_desc(T, C, 4, 1, dw.BF16)
    dw.cconv_bwd(d, x, m.dev(w), None, dy, dx, gw, gb, _space(dw.cconv_bwd_workspace_bytes(d)))
    pad = np.zeros((3, C), np.float32)
    ref = seq.conv_bwd(np.concatenate([pad, xt]), w, None, [0, n + 3], np.concatenate([pad, dyt]))
    _close(dx[-n - 3:], ref[0], 1e-2, "dx")
    _close(gw, ref[1], TOL_SUM, "dw")
    _close(gb, ref[2], TOL_SUM, "db")
    assert not dx[:-n - 3].any()


# ---- layer norm ------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,C,shift", [(2500, 96, 0), (2500, 511, 1), (2500, 520, 0), (2500, 777, 0), (2500, 1024, 0), (2500, 1024, 1),   # a wavefront a row, by 8 and 16 channels
                                       (1024, 1000, 0), (1024, 61, 1),                                                             # few rows: 128 lanes
                                       (1100, 1032, 0), (1100, 2047, 1), (1100, 3000, 0), (1100, 4096, 1),                         # 256 and 512 lanes
                                       (600, 5001, 0), (600, 8192, 0), (600, 9001, 1), (600, 16384, 0)])                           # 1024 lanes
def test_layer_norm_gradients_of_more_rows_than_teams(gpu_lib, dtype, T, C, shift):
    """A team takes a second row and a third, asked for ahead of the one in hand, on the other half of what it shares."""
    m = Made(T + C, dtype, shift)
    x, w, dy, dt = m.host((T, C), 1.5, 0.4), m.host((C,), 0.2, 1.0), m.host((T, C)), m.host((T, C))
    _, mean, rstd, _ = seq.layer_norm(x, w, None, 1e-5)
    mean, rstd = mean.astype(np.float32), rstd.astype(np.float32)
    d = dw.lnorm_desc(T, C, DTYPE[dtype])
    call = (d, m.dev(x), m.dev(w), m.dev(mean, False), m.dev(rstd, False), m.dev(dy))
    space = _space(dw.lnorm_bwd_workspace_bytes(d))
    for given in (dt, None):
        dx, gw, gb = m.out((T, C)), m.out((C,), False), m.out((C,), False)
        dw.lnorm_bwd(*call, dx, gw, gb, space, dtotal=None if given is None else m.dev(given))
        ref = seq.layer_norm_bwd(x, w, mean, rstd, dy, given)
        for got, r, tol, name in ((dx, ref[0], TOL[dtype], "dx"), (gw, ref[1], TOL_SUM, "dw"), (gb, ref[2], TOL_SUM, "db")):
            _close(got, r, tol, name)
    alone = m.out((T, C))
    dw.lnorm_bwd(*call, alone, None, None, None)
    assert torch.equal(alone, dx)


def test_layer_norm_gradients_beyond_32_bit_offsets(gpu_lib):
    T, C, n = (1 << 21) + 5, 1032, 7
    m = Made(32, "bf16")
    xt, dyt = m.host((n, C)), m.host((n, C))
    x, dy = (torch.zeros(T, C, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    x[-n:], dy[-n:] = m.dev(xt), m.dev(dyt)
    _, mt, rt, _ = seq.layer_norm(xt, None, None, 1e-5)
    mean, rstd = torch.zeros(T, device="cuda"), torch.ones(T, device="cuda")
    mean[-n:], rstd[-n:] = torch.from_numpy(mt.astype(np.float32)).cuda(), torch.from_numpy(rt.astype(np.float32)).cuda()
    dx, gw, gb = torch.full_like(x, float("nan")), m.out((C,), False), m.out((C,), False)
    d = dw.lnorm_desc(T, C, dw.BF16)
    dw.lnorm_bwd(d, x, None, mean, rstd, dy, dx, gw, gb, _space(dw.lnorm_bwd_workspace_bytes(d)))
    ref = seq.layer_norm_bwd(xt, None, mt.astype(np.float32), rt.astype(np.float32), dyt)
    for got, r, tol, name in ((dx[-n:], ref[0], 1e-2, "dx"), (gw, ref[1], TOL_SUM, "dw"), (gb, ref[2], TOL_SUM, "db")):
        _close(got, r, tol, name)
    assert not dx[:-n].any()


# ---- selective scan --------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("softplus,gate,skip,bias,slots,wide", [(True, False, True, True, True, True), (True, True, False, True, False, False), (True, True, True, False, True, False),
                                                               (False, True, True, True, False, True), (False, False, False, False, True, True)])
def test_scan_steps_without_their_optional_parts(gpu_lib, dtype, softplus, gate, skip, bias, slots, wide):
    T, C, N, G = 6, 76, 12, 2
    m = Made(41, dtype)
    v = _scan_made(m, T, C, N, G)
    if not softplus:
        v["dt"], v["dt_bias"] = np.abs(v["dt"]) * 0.125, np.abs(v["dt_bias"]) * 0.01
    for name, on in (("z", gate), ("D", skip), ("dt_bias", bias)):
        if not on:
            v[name] = None
    S = 2 * T if slots else T + 3
    state = m.host((S, C, N), stored=False)
    where = m.r.permutation(S)[:T].astype(np.int32) if slots else np.arange(T)
    strides = {"x": C + 5, "dt": 2 * C, "z": C + 1, "B": G * N + 3, "C": 2 * G * N} if wide else {}
    d = dw.sscan_desc(T, C, N, G, S, DTYPE[dtype], softplus, *[strides.get(k) for k in ("x", "dt", "z", "B", "C")], y_stride=C + 7 if wide else None)
    on = {k: None if a is None else m.dev(a, k in ("x", "dt", "z", "B", "C"), strides.get(k)) for k, a in v.items()}
    held, y = m.dev(state, False), m.out((T, C), rows=C + 7 if wide else None)
    dw.sscan_step(d, on["x"], on["dt"], on["A"], on["B"], on["C"], held, y, D=on["D"], z=on["z"], dt_bias=on["dt_bias"],
                  slots=torch.from_numpy(where).cuda() if slots else None)
    want_y, final, _ = seq.scan(bounds=list(range(T + 1)), init=state[where], softplus=softplus, **v)
    want_state = state.astype(np.float64)
    want_state[where] = final
    _close(y, want_y, TOL_SCAN[dtype], "y")
    _close(held, want_state, 2e-5, "state")


# ---- sequence starts of any contents ---------------------------------------------------------------------

STRANGE = [[0, 40, 20, 90, 10, 100], [7, 7, 7, 7, 7, 7], [-5, 200, -300, 1 << 30, -(1 << 31), (1 << 31) - 1], [100, 80, 60, 40, 20, 0],
           [(1 << 31) - 1] * 6, [-(1 << 31)] * 6, [0, 0, 0, 0, 0, 0], [50, 100, 100, 100, 100, 100]]


@pytest.mark.parametrize("starts", STRANGE)
@pytest.mark.parametrize("blocks", [1, 4096])
def test_starts_of_any_contents_stay_inside_the_tensors(gpu_lib, starts, blocks):
    """What comes out is unspecified, but every index is clamped to the tensors: all that lies between and behind them keeps what it held."""
    T, C, N, K, S, edge = 100, 70, 12, 4, 5, 4096
    given = torch.tensor(starts, dtype=torch.int64).to(torch.int32).cuda()
    m = Made(5, "f32")
    v = {k: m.dev(a) for k, a in _scan_made(m, T, C, N, 1).items()}
    w, dy, rows, h = m.dev(m.host((K, C))), m.dev(m.host((T, C))), m.dev(m.host((S, K - 1, C))), m.dev(m.host((S, C, N)))
    guarded = []

    def out(*shape):
        n = int(np.prod(shape))
        t = torch.full((n + 2 * edge,), 12345.0, device="cuda")
        guarded.append((t, n))
        return t[edge:edge + n].view(shape)
    with dw.tuning_overrides({"DWCONV_TUNE_SSCAN_FWD_BLOCKS": blocks, "DWCONV_TUNE_SSCAN_BWD_BLOCKS": blocks, "DWCONV_TUNE_CCONV_STRIP": 4 if blocks > 1 else 64}):
        cd, sd = dw.cconv_desc(T, C, K, S), dw.sscan_desc(T, C, N, 1, S)
        dw.cconv_fwd(cd, v["x"], w, None, out(T, C), starts=given, init=rows, final=out(S, K - 1, C))
        dw.cconv_bwd(cd, v["x"], w, None, dy, out(T, C), out(K, C), out(C), out(dw.cconv_bwd_workspace_bytes(cd) // 4), starts=given, init=rows)
        kept = out(dw.sscan_kept_bytes(sd) // 4)
        call = (sd, v["x"], v["dt"], v["A"], v["B"], v["C"])
        more = {"D": v["D"], "z": v["z"], "dt_bias": v["dt_bias"], "starts": given, "init": h}
        dw.sscan_fwd(*call, out(T, C), out(max(4, dw.sscan_fwd_workspace_bytes(sd) // 4)), final=out(S, C, N), kept=kept, **more)
        dw.sscan_bwd(*call, kept, dy, out(T, C), out(T, C), out(C, N), out(T, N), out(T, N), out(dw.sscan_bwd_workspace_bytes(sd) // 4), dD=out(C), dz=out(T, C),
                     ddt_bias=out(C), **more)
    torch.cuda.synchronize()
    for t, n in guarded:
        assert bool((t[:edge] == 12345.0).all()) and bool((t[edge + n:] == 12345.0).all())
