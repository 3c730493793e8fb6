"""GPU parity of the sequence operators (layer norm, causal convolution, selective scan) with the oracle in 64 bits, element by element: forward, backward and
single tokens, at the sizes where a kernel changes its tile, its vector or its path, packed and carried sequences, strides and odd alignment.

Tolerances (relative, in the max norm and the 2-norm, as for the convolutions): what is stored in bf16 is rounded once, to 2^-9 of itself, 1e-2 leaves room for the largest value's
neighbours.  fp32: a norm or a convolution adds at most 16384 terms in a tree, about log2(16384) * 2^-24 = 1e-6, twice over: 1e-5.  A scan of 300 tokens rounds its state
3 times a token, by 2^-24 each of a sum whose weights are at most one: 300 * 3 * 6e-8 = 5e-5 if all went one way, a fifteenth of it when they do not: 2e-5; sums over tokens likewise."""
import numpy as np
import pytest
import torch

import paper_1803_09926_amd as dw
from oracle import sequence as seq

import gpu_util as gu

pytestmark = pytest.mark.gpu

TOL = {"f32": 1e-5, "bf16": 1e-2}
TOL_SCAN = {"f32": 2e-5, "bf16": 1e-2}
TOL_SUM = 2e-5
DTYPE = {"f32": dw.F32, "bf16": dw.BF16}
TORCH = {"f32": torch.float32, "bf16": torch.bfloat16}


class Made:
    """Random tensors by name: on the device as the call takes them, and in numpy as the oracle does (bf16 values exactly)."""

    def __init__(self, seed, dtype, shift=0):
        self.r, self.dtype, self.shift = np.random.default_rng(seed), dtype, shift

    def host(self, shape, scale=1.0, mean=0.0, stored=True):
        v = torch.from_numpy((self.r.normal(size=shape) * scale + mean).astype(np.float32))
        return v.to(torch.bfloat16).float().numpy() if stored and self.dtype == "bf16" else v.numpy()

    def dev(self, v, stored=True, rows=None):
        """On the device, `shift` elements off a 16-byte boundary; rows: with that stride."""
        t = torch.from_numpy(np.ascontiguousarray(v))
        t = t.to(TORCH[self.dtype]) if stored else t
        if rows and v.shape[0] > 0:
            width = int(np.prod(v.shape[1:]))
            space = torch.full((v.shape[0] * rows + self.shift,), float("nan"), dtype=t.dtype)
            out = space.cuda()[self.shift:].as_strided((v.shape[0], width), (rows, 1))
            out.copy_(t.reshape(v.shape[0], width))
            return out
        space = torch.empty(t.numel() + self.shift, dtype=t.dtype, device="cuda")
        out = space[self.shift:].view(t.shape)
        out.copy_(t)
        return out

    def out(self, shape, stored=True, rows=None):
        """An output, filled with NaN so that an unwritten element cannot pass."""
        return self.dev(np.full(shape, np.nan, np.float32), stored, rows)


def _space(n):
    return torch.full((max(n, 16),), 0xFF, device="cuda", dtype=torch.uint8)


def _close(got, want, tol, what):
    g = gu.to_host(got).reshape(np.shape(want))
    if np.size(want):
        gu.assert_close(g, want, tol, what)


def _starts(bounds):
    return torch.tensor(bounds, dtype=torch.int32, device="cuda")


# ---- layer norm ------------------------------------------------------------------------------------------

CHANNELS = [1, 2, 7, 64, 65, 512, 513, 728, 1024, 1025, 2048, 2050, 4096, 4099, 8192, 8193, 16384]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("C", CHANNELS)
@pytest.mark.parametrize("T,residual,params,shift", [(1, False, True, 0), (5, True, True, 0), (37, True, False, 1), (6, False, False, 1)])
def test_layer_norm(gpu_lib, dtype, C, T, residual, params, shift):
    print("layer norm", dtype, C, T, residual, params, shift, flush=True)
    m = Made(C * 100 + T, dtype, shift)
    x, w, b = m.host((T, C), 1.5, 0.4), m.host((C,), 0.2, 1.0), m.host((C,), 0.2)
    res = m.host((T, C)) if residual else None
    w, b = (w, b) if params else (None, None)
    d = dw.lnorm_desc(T, C, DTYPE[dtype], 1e-5)
    on = lambda v: None if v is None else m.dev(v)  # noqa: E731
    y, mean, rstd = m.out((T, C)), m.out((T,), False), m.out((T,), False)
    total = m.out((T, C)) if residual else None
    dw.lnorm_fwd(d, on(x), on(w), on(b), y, mean, rstd, residual=on(res), total=total)
    want = seq.layer_norm(x, w, b, 1e-5, res)
    for got, ref, name in ((y, want[0], "y"), (mean, want[1], "mean"), (rstd, want[2], "rstd"), (total, want[3], "total")):
        if got is not None:
            _close(got, ref, TOL["f32"] if got.dtype == torch.float32 else TOL[dtype], name)
    s = x if total is None else gu.to_host(total).reshape(T, C)
    dy, dt = m.host((T, C)), (m.host((T, C)) if residual else None)
    dx, gw, gb = m.out((T, C)), (m.out((C,), False) if params else None), (m.out((C,), False) if params else None)
    dw.lnorm_bwd(d, on(s), on(w), mean, rstd, on(dy), dx, gw, gb, _space(dw.lnorm_bwd_workspace_bytes(d)), dtotal=on(dt))
    ref = seq.layer_norm_bwd(s, w, gu.to_host(mean), gu.to_host(rstd), dy, dt)
    if C > 2:      # (with one channel the gradient is zero, with two nearly so: what is left is rounding)
        _close(dx, ref[0], TOL[dtype], "dx")
    if params:
        _close(gw, ref[1], TOL_SUM, "dw")
        _close(gb, ref[2], TOL_SUM, "db")


def test_layer_norm_many_rows_and_none(gpu_lib):
    m = Made(5, "f32")
    T, C = 5003, 96
    x, w, dy = m.host((T, C), 1.5, 3.0), m.host((C,)), m.host((T, C))
    d = dw.lnorm_desc(T, C, dw.F32)
    y, mean, rstd, dx, gw, gb = m.out((T, C)), m.out((T,)), m.out((T,)), m.out((T, C)), m.out((C,)), m.out((C,))
    dw.lnorm_fwd(d, m.dev(x), m.dev(w), None, y, mean, rstd)
    want = seq.layer_norm(x, w, None, 1e-5)
    _close(y, want[0], 1e-5, "y")
    dw.lnorm_bwd(d, m.dev(x), m.dev(w), mean, rstd, m.dev(dy), dx, gw, gb, _space(dw.lnorm_bwd_workspace_bytes(d)))
    ref = seq.layer_norm_bwd(x, w, want[1], want[2], dy)
    for got, r, tol in ((dx, ref[0], 1e-5), (gw, ref[1], TOL_SUM), (gb, ref[2], TOL_SUM)):
        _close(got, r, tol, "gradients of %d rows" % T)
    none = torch.empty(0, C, device="cuda")
    d = dw.lnorm_desc(0, C, dw.F32)
    dw.lnorm_fwd(d, none, m.dev(w), None, none)
    dw.lnorm_bwd(d, none, m.dev(w), none[:, 0], none[:, 0], none, none, gw, gb, None)
    assert not gw.any() and not gb.any()


def test_layer_norm_offsets_beyond_32_bits(gpu_lib):
    T, C = (1 << 21) + 5, 1032                      # 2.16e9 elements
    x = torch.zeros(T, C, device="cuda", dtype=torch.bfloat16)
    tail = torch.randn(7, C, device="cuda").to(torch.bfloat16)
    x[-7:] = tail
    y = torch.empty_like(x)
    dw.lnorm_fwd(dw.lnorm_desc(T, C, dw.BF16), x, None, None, y)
    want = seq.layer_norm(gu.to_host(tail), None, None, 1e-5)[0]
    _close(y[-7:], want, 1e-2, "the last rows")
    assert not y[:3].any() and not y[T // 2:T // 2 + 3].any()


# ---- causal convolution ----------------------------------------------------------------------------------

EVEN = lambda T, S: [T // S * i for i in range(S + 1)]  # noqa: E731
RAGGED = [0, 0, 1, 3, 3, 3, 10, 77, 78, 140, 140, 300, 300]


def _conv_case(dtype, C, K, bounds, packed, carry, silu, xs, shift, seed):
    T, S = bounds[-1], len(bounds) - 1
    m = Made(seed, dtype, shift)
    x, w, b, dy = m.host((T, C)), m.host((K, C), 0.5), m.host((C,), 0.2), m.host((T, C))
    init = m.host((S, K - 1, C)) if carry else None
    stride = C if xs is None else xs
    d = dw.cconv_desc(T, C, K, S, DTYPE[dtype], silu, stride, C)
    starts = _starts(bounds) if packed else None
    on = lambda v: None if v is None else m.dev(v)  # noqa: E731
    xd = m.dev(x, rows=xs)
    y, final = m.out((T, C)), m.out((S, K - 1, C))
    dw.cconv_fwd(d, xd, on(w), on(b), y, starts=starts, init=on(init), final=final)
    wy, wf = seq.conv(x, w, b, bounds, init, silu)
    tag = "conv %s C %d K %d" % (dtype, C, K)
    _close(y, wy, TOL[dtype], "y " + tag)
    assert np.array_equal(gu.to_host(final), wf.astype(np.float32)), "final " + tag
    dx, gw, gb = m.out((T, C), rows=xs), m.out((K, C), False), m.out((C,), False)
    dw.cconv_bwd(d, xd, on(w), on(b), on(dy), dx, gw, gb, _space(dw.cconv_bwd_workspace_bytes(d)), starts=starts, init=on(init))
    ref = seq.conv_bwd(x, w, b, bounds, dy, init, silu)
    _close(dx, ref[0], TOL[dtype], "dx " + tag)
    _close(gw, ref[1], TOL_SUM, "dw " + tag)
    _close(gb, ref[2], TOL_SUM, "db " + tag)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("K", range(2, 9))
@pytest.mark.parametrize("C,xs,shift", [(1, None, 0), (5, 13, 1), (64, None, 0), (200, 400, 0), (263, None, 1), (1040, None, 0)])
def test_conv_packed_and_carried(gpu_lib, dtype, K, C, xs, shift):
    print("conv", dtype, K, C, xs, shift, flush=True)
    _conv_case(dtype, C, K, RAGGED, True, True, K != 3, xs, shift, 1000 * K + C)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,S,carry", [(1, 1, True), (1, 1, False), (2, 2, False), (7, 7, True), (66, 1, False), (256, 4, False), (999, 3, True)])
def test_conv_of_equal_lengths(gpu_lib, dtype, T, S, carry):
    _conv_case(dtype, 72, 4, EVEN(T, S), False, carry, True, None, 0, T)


def test_conv_strips_of_long_launches(gpu_lib):
    # many tokens of few channels: whole blocks of strips, and strips longer than the least
    _conv_case("f32", 8, 4, [0, 1, 900, 70001], True, False, True, None, 0, 3)
    _conv_case("bf16", 512, 4, [0, 3000, 9001], True, True, True, 1024, 0, 4)


def test_conv_carries_nothing_across_sequences(gpu_lib):
    m = Made(9, "f32")
    bounds, K, C = [0, 5, 5, 40], 4, 12
    x, w, dy = m.host((40, C)), m.host((K, C)), m.host((40, C))
    bad, bad_dy = x.copy(), dy.copy()
    bad[:5] = [[np.inf], [np.nan], [-np.inf], [np.nan], [np.inf]]
    bad_dy[:5] = np.nan
    d, outs = dw.cconv_desc(40, C, K, 3, dw.F32), []
    for xv, g in ((x, dy), (bad, bad_dy)):
        y, dx, gw, gb = m.out((40, C)), m.out((40, C)), m.out((K, C)), m.out((C,))
        dw.cconv_fwd(d, m.dev(xv), m.dev(w), None, y, starts=_starts(bounds))
        dw.cconv_bwd(d, m.dev(xv), m.dev(w), None, m.dev(g), dx, gw, gb, _space(dw.cconv_bwd_workspace_bytes(d)), starts=_starts(bounds))
        outs.append((y[5:], dx[5:]))
    assert torch.equal(outs[0][0], outs[1][0]) and torch.equal(outs[0][1], outs[1][1])


def test_conv_of_no_tokens(gpu_lib):
    m = Made(2, "f32")
    init, w = m.host((3, 3, 8)), m.host((4, 8))
    none, final, gw, gb = torch.empty(0, 8, device="cuda"), m.out((3, 3, 8)), m.out((4, 8)), m.out((8,))
    d = dw.cconv_desc(0, 8, 4, 3)
    dw.cconv_fwd(d, none, m.dev(w), None, none, init=m.dev(init), final=final)
    assert np.array_equal(gu.to_host(final), init)
    dw.cconv_fwd(d, none, m.dev(w), None, none, starts=_starts([0, 0, 0, 0]), final=final)
    assert not final.any()
    dw.cconv_bwd(d, none, m.dev(w), None, none, none, gw, gb, None)
    assert not gw.any() and not gb.any()


def test_conv_offsets_beyond_32_bits(gpu_lib):
    T, C = (1 << 21) + 9, 1024
    x = torch.zeros(T, C, device="cuda", dtype=torch.bfloat16)
    tail = torch.randn(9, C, device="cuda").to(torch.bfloat16)
    x[-9:] = tail
    w = torch.randn(4, C, device="cuda").to(torch.bfloat16)
    y = torch.empty_like(x)
    dw.cconv_fwd(dw.cconv_desc(T, C, 4, 1, dw.BF16), x, w, None, y)
    want = seq.conv(np.concatenate([np.zeros((3, C), np.float32), gu.to_host(tail)]), gu.to_host(w), None, [0, 12])[0][3:]
    _close(y[-9:], want, 1e-2, "the last tokens")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,C,K,xs", [(1, 8, 4, None), (3, 1, 2, 5), (5, 77, 8, None), (64, 1040, 4, 2080), (130, 24, 3, None)])
def test_conv_steps(gpu_lib, dtype, T, C, K, xs):
    m = Made(T * C, dtype)
    S = 2 * T + 1
    x, w, b, state = m.host((T, C)), m.host((K, C)), m.host((C,)), m.host((S, K - 1, C))
    slots = m.r.permutation(S)[:T].astype(np.int32)
    pads = [T // 2] if T > 2 else []
    for p, bad in zip(pads, (-1,)):
        slots[p] = bad
    if T > 4:
        slots[T - 1] = S
        pads.append(T - 1)
    d = dw.cconv_desc(T, C, K, S, DTYPE[dtype], True, C if xs is None else xs)
    held, y = m.dev(state), m.out((T, C))
    dw.cconv_step(d, m.dev(x, rows=xs), m.dev(w), m.dev(b), held, y, slots=torch.from_numpy(slots).cuda())
    want_y, want_state = np.zeros((T, C)), state.copy()
    for t in range(T):
        if t not in pads:
            yy, f = seq.conv(x[t:t + 1], w, b, [0, 1], state[slots[t]][None])
            want_y[t], want_state[slots[t]] = yy[0], f[0]
    _close(y, want_y, TOL[dtype], "y")
    assert np.array_equal(gu.to_host(held), want_state)
    assert not gu.to_host(y)[pads].any()


# ---- selective scan --------------------------------------------------------------------------------------

def _scan_made(m, T, C, N, G):
    v = {"x": m.host((T, C)), "dt": m.host((T, C), 0.5), "B": m.host((T, G, N)), "C": m.host((T, G, N)),
         "A": -np.exp(m.host((C, N), 0.7, stored=False)), "D": m.host((C,), 0.3, 1.0, stored=False),
         "z": m.host((T, C)), "dt_bias": m.host((C,), 1.0, -3.0, stored=False)}
    return v


def _scan_case(dtype, C, N, G, bounds, packed, carry, softplus=True, gate=True, skip=True, bias=True, wide=False, shift=0, seed=1):
    T, S = bounds[-1], len(bounds) - 1
    m = Made(seed, dtype, shift)
    v = _scan_made(m, T, C, N, G)
    if not softplus:
        v["dt"] = np.abs(v["dt"]) * 0.125          # (a power of two: bf16 values stay exact)
        v["dt_bias"] = np.abs(v["dt_bias"]) * 0.01
    for name, on in (("z", gate), ("D", skip), ("dt_bias", bias)):
        if not on:
            v[name] = None
    if not bias and softplus:
        v["dt"] = v["dt"] - 2.0
        v["dt"] = torch.from_numpy(v["dt"]).to(TORCH[dtype]).float().numpy()
    init = m.host((S, C, N), stored=False) if carry else None
    dy = m.host((T, C))
    xs, zs, bs = (C + 3, 2 * C, 2 * G * N + 1) if wide else (C, C, G * N)
    d = dw.sscan_desc(T, C, N, G, S, DTYPE[dtype], softplus, x_stride=xs, z_stride=zs, b_stride=bs, c_stride=bs)
    rows = {"x": xs, "z": zs, "B": bs, "C": bs} if wide else {}
    on = {k: None if a is None else m.dev(a, k in ("x", "dt", "z", "B", "C"), rows.get(k)) for k, a in v.items()}
    more = {"D": on["D"], "z": on["z"], "dt_bias": on["dt_bias"], "starts": _starts(bounds) if packed else None,
            "init": None if init is None else m.dev(init, False)}
    call = (d, on["x"], on["dt"], on["A"], on["B"], on["C"])
    y, final = m.out((T, C)), m.out((S, C, N), False)
    kept = torch.full((max(dw.sscan_kept_bytes(d) // 4, 4),), float("nan"), device="cuda")
    dw.sscan_fwd(*call, y, _space(dw.sscan_fwd_workspace_bytes(d)), final=final, kept=kept, **more)
    alone = m.out((T, C))
    dw.sscan_fwd(*call, alone, _space(dw.sscan_fwd_workspace_bytes(d)), **more)
    assert torch.equal(y, alone)
    tag = " %s C %d N %d G %d T %d" % (dtype, C, N, G, T)
    args = dict(bounds=bounds, init=init, softplus=softplus, **v)
    wy, wf, _ = seq.scan(**args)
    _close(y, wy, TOL_SCAN[dtype], "y" + tag)
    _close(final, wf, TOL_SCAN["f32"], "final" + tag)
    grads = {"dx": m.out((T, C), rows=rows.get("x")), "ddt": m.out((T, C)), "dA": m.out((C, N), False),
             "dB": m.out((T, G * N), rows=rows.get("B")), "dC": m.out((T, G * N), rows=rows.get("C")),
             "dD": m.out((C,), False) if skip else None, "dz": m.out((T, C), rows=rows.get("z")) if gate else None, "ddt_bias": m.out((C,), False)}
    dw.sscan_bwd(*call, kept, m.dev(dy), grads["dx"], grads["ddt"], grads["dA"], grads["dB"], grads["dC"], _space(dw.sscan_bwd_workspace_bytes(d)),
                 dD=grads["dD"], dz=grads["dz"], ddt_bias=grads["ddt_bias"], **more)
    ref = seq.scan_bwd(dy=dy, **args)
    for k, got in grads.items():
        if got is not None:
            _close(got, ref[k], TOL_SCAN[dtype] if k in ("dx", "ddt", "dB", "dC", "dz") else TOL_SUM, k + tag)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("N", [1, 3, 4, 8, 9, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("C,G,wide,shift", [(1, 1, False, 0), (24, 2, True, 1), (66, 1, False, 0), (130, 2, True, 0)])
def test_scan_packed_and_carried(gpu_lib, dtype, N, C, G, wide, shift):
    print("scan", dtype, N, C, G, wide, shift, flush=True)
    _scan_case(dtype, C, N, G, RAGGED, True, True, wide=wide, shift=shift, seed=100 * N + C)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,S,carry", [(1, 1, True), (1, 1, False), (2, 2, False), (16, 1, False), (17, 1, True), (32, 1, True), (33, 1, False), (65, 1, True),
                                       (96, 3, False), (256, 8, False), (257, 1, False)])
def test_scan_of_equal_lengths(gpu_lib, dtype, T, S, carry):
    _scan_case(dtype, 80, 16, 1, EVEN(T, S), False, carry, seed=T)


@pytest.mark.parametrize("softplus,gate,skip,bias", [(False, True, True, True), (True, False, True, True), (True, True, False, True), (True, True, True, False),
                                                     (False, False, False, False)])
def test_scan_without_its_optional_parts(gpu_lib, softplus, gate, skip, bias):
    _scan_case("f32", 40, 16, 2, [0, 30, 30, 100], True, False, softplus, gate, skip, bias, seed=7)
    _scan_case("bf16", 40, 8, 1, [0, 50], False, False, softplus, gate, skip, bias, seed=8)


def test_scan_of_whole_sequences_a_part(gpu_lib):
    # enough channel blocks and sequences that no state is carried from part to part; then the same sequences given by their starts
    for packed in (False, True):
        _scan_case("f32", 704, 16, 1, EVEN(32 * 40, 40), packed, True, seed=11)


@pytest.mark.parametrize("blocks,most", [(1, 80), (2, 2), (12, 80), (60, 7), (4096, 80), (4096, 300)])
@pytest.mark.parametrize("N", [8, 16, 33])
def test_scan_however_it_is_split(gpu_lib, blocks, most, N):
    """One part, parts of one tile, more parts than one look back takes, whole sequences a part and several of them: the plans of other sizes, forced on a small one."""
    knobs = {"DWCONV_TUNE_SSCAN_FWD_BLOCKS": blocks, "DWCONV_TUNE_SSCAN_BWD_BLOCKS": blocks, "DWCONV_TUNE_SSCAN_MOST_PARTS": most}
    with dw.tuning_overrides(knobs):
        _scan_case("f32", 70, N, 1, RAGGED, True, True, seed=N)
        _scan_case("f32", 70, N, 1, EVEN(288, 6), False, True, seed=N + 1)
        _scan_case("bf16", 70, N, 2, EVEN(290, 1), False, False, seed=N + 2)


@pytest.mark.parametrize("S,T", [(60, 64), (65, 150), (130, 40), (4200, 150)])
@pytest.mark.parametrize("C,N", [(24, 16), (75, 5)])
def test_scan_of_more_sequences_than_lanes(gpu_lib, S, T, C, N):
    """Sequences of any lengths, most of them empty where they are many; both with one part and with a tile a part."""
    bounds = [0] + sorted(np.random.default_rng(S).integers(0, T + 1, S - 1).tolist()) + [T]
    for blocks in (1, 4096):
        with dw.tuning_overrides({"DWCONV_TUNE_SSCAN_FWD_BLOCKS": blocks, "DWCONV_TUNE_SSCAN_BWD_BLOCKS": blocks}):
            _scan_case("f32", C, N, 1, bounds, True, True, seed=S)


def test_scan_states_and_gradients_that_hardly_decay_and_that_vanish(gpu_lib):
    """Decays next to 1 and far below the smallest number, step sizes from 1e-6 to 20: the parts' products and the kept states hold either way."""
    m = Made(3, "f32")
    T, C, N = 290, 64, 16
    v = _scan_made(m, T, C, N, 1)
    v["A"] = -np.exp(np.linspace(-8, 6, C * N)).reshape(C, N).astype(np.float32)
    v["dt_bias"] = np.linspace(-13, 20, C).astype(np.float32)
    dy = m.host((T, C))
    d = dw.sscan_desc(T, C, N, 1, 1)
    on = {k: m.dev(a) for k, a in v.items()}
    y, kept = m.out((T, C)), torch.empty(dw.sscan_kept_bytes(d) // 4, device="cuda")
    call, more = (d, on["x"], on["dt"], on["A"], on["B"], on["C"]), {k: on[k] for k in ("D", "z", "dt_bias")}
    dw.sscan_fwd(*call, y, _space(dw.sscan_fwd_workspace_bytes(d)), kept=kept, **more)
    _close(y, seq.scan(bounds=[0, T], **v)[0], 2e-5, "y")
    g = {k: m.out(s) for k, s in (("dx", (T, C)), ("ddt", (T, C)), ("dA", (C, N)), ("dB", (T, N)), ("dC", (T, N)), ("dD", (C,)), ("dz", (T, C)), ("ddt_bias", (C,)))}
    dw.sscan_bwd(*call, kept, m.dev(dy), g["dx"], g["ddt"], g["dA"], g["dB"], g["dC"], _space(dw.sscan_bwd_workspace_bytes(d)), dD=g["dD"], dz=g["dz"],
                 ddt_bias=g["ddt_bias"], **more)
    ref = seq.scan_bwd(bounds=[0, T], dy=dy, **v)
    for k in g:
        _close(g[k], ref[k], 2e-5, k)


def test_scan_carries_nothing_across_sequences(gpu_lib):
    m = Made(9, "f32")
    bounds, T, C, N = [0, 70, 70, 290], 290, 70, 16
    v, dy = _scan_made(m, T, C, N, 1), m.host((T, C))
    outs = []
    for bad in (False, True):
        w = {k: a.copy() for k, a in v.items()}
        g = dy.copy()
        if bad:
            w["x"][:70] = np.nan
            w["B"][:70] = np.inf
            w["dt"][:70] = np.nan
            g[:70] = np.inf
        d = dw.sscan_desc(T, C, N, 1, 3)
        on = {k: m.dev(a) for k, a in w.items()}
        call = (d, on["x"], on["dt"], on["A"], on["B"], on["C"])
        more = {"D": on["D"], "z": on["z"], "dt_bias": on["dt_bias"], "starts": _starts(bounds)}
        y, final, kept = m.out((T, C)), m.out((3, C, N)), torch.empty(dw.sscan_kept_bytes(d) // 4, device="cuda")
        dw.sscan_fwd(*call, y, _space(dw.sscan_fwd_workspace_bytes(d)), final=final, kept=kept, **more)
        o = [m.out(s) for s in ((T, C), (T, C), (C, N), (T, N), (T, N))]
        dw.sscan_bwd(*call, kept, m.dev(g), *o, _space(dw.sscan_bwd_workspace_bytes(d)), dD=m.out((C,)), dz=m.out((T, C)), ddt_bias=m.out((C,)), **more)
        outs.append([y[70:], final[1:], o[0][70:], o[1][70:], o[3][70:], o[4][70:]])
    for a, b in zip(*outs):
        assert torch.equal(a, b)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_scan_offsets_beyond_32_bits(gpu_lib, dtype):
    """Rows as far apart as they may be, which the passes read and write as they do dense ones."""
    T, C, N, far = 75, 24, 16, 1 << 25
    m = Made(9, dtype)
    on = {k: m.dev(a, k in ("x", "dt", "z", "B", "C")) for k, a in _scan_made(m, T, C, N, 1).items()}
    on["dy"] = m.dev(m.host((T, C)))
    read, written = (torch.empty((T - 1) * far + 256, dtype=TORCH[dtype], device="cuda") for _ in range(2))
    results = []
    for stride in (None, far):
        d = dw.sscan_desc(T, C, N, 1, 1, DTYPE[dtype], True, *[stride] * 6)
        rows, column = dict(on), 0
        if stride:
            for k in ("x", "dt", "z", "B", "C", "dy"):
                width = on[k].numel() // T
                rows[k] = read.as_strided((T, width), (far, 1), column).copy_(on[k].reshape(T, width))
                column += width
        outs, column = {}, 0
        for k, width in (("y", C), ("dx", C), ("ddt", C), ("dz", C), ("dB", N), ("dC", N)):
            outs[k] = written.as_strided((T, width), (far, 1), column) if stride else torch.empty(T, width, dtype=TORCH[dtype], device="cuda")
            column += width
        sums = {k: torch.empty_like(on[a]) for k, a in (("dA", "A"), ("dD", "D"), ("ddt_bias", "dt_bias"))}
        call = (d, rows["x"], rows["dt"], on["A"], rows["B"], rows["C"])
        more = {"D": on["D"], "z": rows["z"], "dt_bias": on["dt_bias"]}
        kept = torch.empty(dw.sscan_kept_bytes(d) // 4, device="cuda")
        dw.sscan_fwd(*call, outs["y"], _space(dw.sscan_fwd_workspace_bytes(d)), kept=kept, **more)
        dw.sscan_bwd(*call, kept, rows["dy"], outs["dx"], outs["ddt"], sums["dA"], outs["dB"], outs["dC"], _space(dw.sscan_bwd_workspace_bytes(d)),
                     dD=sums["dD"], dz=outs["dz"], ddt_bias=sums["ddt_bias"], **more)
        results.append({k: t.contiguous() for k, t in {**outs, **sums}.items()})
    for k, dense in results[0].items():
        assert torch.isfinite(dense).all() and torch.equal(dense, results[1][k]), k


def test_scan_of_no_tokens(gpu_lib):
    m = Made(2, "f32")
    C, N = 20, 5
    init, A = m.host((3, C, N)), m.host((C, N))
    none, shared, final, dA, dD, db = torch.empty(0, C, device="cuda"), torch.empty(0, N, device="cuda"), m.out((3, C, N)), m.out((C, N)), m.out((C,)), m.out((C,))
    d = dw.sscan_desc(0, C, N, 1, 3)
    for starts in (None, _starts([0, 0, 0, 0])):
        final.fill_(float("nan"))
        dw.sscan_fwd(d, none, none, m.dev(A), shared, shared, none, None, starts=starts, init=m.dev(init), final=final)
        assert np.array_equal(gu.to_host(final), init)
    dw.sscan_bwd(d, none, none, m.dev(A), shared, shared, _space(16), none, none, none, dA, shared, shared, None, D=dD.clone(), dD=dD, ddt_bias=db)
    assert not dA.any() and not dD.any() and not db.any()


def test_scan_in_pieces_and_token_by_token(gpu_lib):
    """A prompt in one call, in two calls that hand their states on, and its last tokens one at a time."""
    m = Made(4, "f32")
    T, C, N, K = 150, 96, 16, 4
    v = _scan_made(m, T, C, N, 1)
    w = m.host((K, C))
    xin = m.dev(v["x"])
    on = {k: m.dev(a) for k, a in v.items()}
    more = {"D": on["D"], "dt_bias": on["dt_bias"]}

    def run(lo, hi, conv_state, state):
        conv_final, final = m.out((1, K - 1, C)), m.out((1, C, N))
        x, y = m.out((hi - lo, C)), m.out((hi - lo, C))
        dw.cconv_fwd(dw.cconv_desc(hi - lo, C, K), xin[lo:hi], m.dev(w), None, x, init=conv_state, final=conv_final)
        d = dw.sscan_desc(hi - lo, C, N)
        dw.sscan_fwd(d, x, on["dt"][lo:hi], on["A"], on["B"][lo:hi], on["C"][lo:hi], y, _space(dw.sscan_fwd_workspace_bytes(d)), z=on["z"][lo:hi],
                     init=state, final=final, **more)
        return y, conv_final, final

    whole, cf, sf = run(0, T, None, None)
    a, c1, s1 = run(0, 101, None, None)
    b, c2, s2 = run(101, T, c1, s1)
    _close(torch.cat([a, b]), gu.to_host(whole), 2e-5, "two pieces")
    _close(s2, gu.to_host(sf), 2e-5, "the state after two pieces")
    assert torch.equal(c2, cf)
    for t in range(101, T):
        x, y = m.out((1, C)), m.out((1, C))
        dw.cconv_step(dw.cconv_desc(1, C, K, 1), xin[t:t + 1], m.dev(w), None, c1, x)
        dw.sscan_step(dw.sscan_desc(1, C, N, 1, 1), x, on["dt"][t:t + 1], on["A"], on["B"][t:t + 1], on["C"][t:t + 1], s1, y, z=on["z"][t:t + 1], **more)
        _close(y, gu.to_host(whole[t:t + 1]), 2e-5, "token %d" % t)
    _close(s1, gu.to_host(sf), 2e-5, "the state token by token")
    assert torch.equal(c1, cf)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,C,N,G,wide", [(1, 8, 16, 1, False), (3, 1, 1, 1, True), (5, 78, 24, 2, True), (33, 520, 16, 1, True), (7, 60, 64, 4, False), (9, 30, 6, 1, False)])
def test_scan_steps(gpu_lib, dtype, T, C, N, G, wide):
    m = Made(T * C + N, dtype)
    S = 2 * T + 1
    v, state = _scan_made(m, T, C, N, G), m.host((S, C, N), stored=False)
    slots = m.r.permutation(S)[:T].astype(np.int32)
    pads = []
    if T > 4:
        slots[2], slots[T - 1] = -7, S
        pads = [2, T - 1]
    zs, bs = (2 * C, 2 * G * N + 1) if wide else (C, G * N)
    d = dw.sscan_desc(T, C, N, G, S, DTYPE[dtype], z_stride=zs, b_stride=bs, c_stride=bs)
    held, y = m.dev(state, False), m.out((T, C))
    rows = {"z": zs, "B": bs, "C": bs} if wide else {}
    on = {k: m.dev(a, k in ("x", "dt", "z", "B", "C"), rows.get(k)) for k, a in v.items()}
    dw.sscan_step(d, on["x"], on["dt"], on["A"], on["B"], on["C"], held, y, D=on["D"], z=on["z"], dt_bias=on["dt_bias"], slots=torch.from_numpy(slots).cuda())
    want_y, want_state = np.zeros((T, C)), state.astype(np.float64)
    for t in range(T):
        if t not in pads:
            one = {k: a[t:t + 1] if k in ("x", "dt", "z", "B", "C") else a for k, a in v.items()}
            yy, f, _ = seq.scan(bounds=[0, 1], init=state[slots[t]][None], **one)
            want_y[t], want_state[slots[t]] = yy[0], f[0]
    _close(y, want_y, TOL_SCAN[dtype], "y")
    _close(held, want_state, 2e-5, "state")
    assert not gu.to_host(y)[pads].any()


# ---- streams, graphs, repetition -------------------------------------------------------------------------

def test_passes_repeat_bit_for_bit_on_any_stream_and_in_a_graph(gpu_lib):
    m = Made(21, "bf16")
    T, C, N, K = 700, 192, 16, 4
    v, dy, w, b = _scan_made(m, T, C, N, 1), m.host((T, C)), m.host((K, C)), m.host((C,))
    on = {k: m.dev(a, k in ("x", "dt", "z", "B", "C")) for k, a in v.items()}
    dyd, wd, bd, starts = m.dev(dy), m.dev(w), m.dev(b), _starts([0, 100, 333, 333, T])
    ld, cd, sd = dw.lnorm_desc(T, C, dw.BF16), dw.cconv_desc(T, C, K, 4, dw.BF16), dw.sscan_desc(T, C, N, 1, 4, dw.BF16)
    space = [_space(n) for n in (dw.lnorm_bwd_workspace_bytes(ld), dw.cconv_bwd_workspace_bytes(cd), dw.sscan_fwd_workspace_bytes(sd),
                                 dw.sscan_bwd_workspace_bytes(sd), dw.sscan_kept_bytes(sd))]

    def fresh():
        stored, f32 = [m.out((T, C)) for _ in range(8)], [m.out(s, False) for s in ((T,), (T,), (C,), (C,), (K, C), (C,), (C, N), (C,), (C,))]
        return stored + f32 + [m.out((T, N)), m.out((T, N))]

    def run(o, stream=None):
        normed, x, y, dxs, ddt, dz, dxc, dxl, mean, rstd, gw, gb, cw, cb, dA, dD, dbias, dB, dC = o
        dw.lnorm_fwd(ld, on["x"], bd, bd, normed, mean, rstd, stream=stream)
        dw.cconv_fwd(cd, normed, wd, bd, x, starts=starts, stream=stream)
        more = {"D": on["D"], "z": on["z"], "dt_bias": on["dt_bias"], "starts": starts, "stream": stream}
        dw.sscan_fwd(sd, x, on["dt"], on["A"], on["B"], on["C"], y, space[2], kept=space[4], **more)
        dw.sscan_bwd(sd, x, on["dt"], on["A"], on["B"], on["C"], space[4], dyd, dxs, ddt, dA, dB, dC, space[3], dD=dD, dz=dz, ddt_bias=dbias, **more)
        dw.cconv_bwd(cd, normed, wd, bd, dxs, dxc, cw, cb, space[1], starts=starts, stream=stream)
        dw.lnorm_bwd(ld, on["x"], bd, mean, rstd, dxc, dxl, gw, gb, space[0], stream=stream)

    want, other = fresh(), fresh()
    run(want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    run(other, side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    assert all(bool(torch.isfinite(a.float()).all()) for a in want)
    o = fresh()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run(o)
    for _ in range(3):
        for a in o:
            a.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, o))
        run(other)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, other))


def test_calls_by_the_general_way_agree(gpu_lib):
    class Sub(torch.Tensor):
        pass
    m = Made(6, "f32")
    x, w, b = m.dev(m.host((6, 8))), m.dev(m.host((4, 8))), m.dev(m.host((8,)))
    d, y, other = dw.cconv_desc(6, 8), m.out((6, 8)), m.out((6, 8))
    dw.cconv_fwd(d, x, w, b, y)
    dw.cconv_fwd(d, x.as_subclass(Sub), w, torch.nn.Parameter(b, requires_grad=False), other)
    assert torch.equal(y, other)
    with pytest.raises(ValueError, match="rows"):
        dw.cconv_fwd(d, x[:, :4], w, b, y)
    with pytest.raises(ValueError, match="w must be contiguous with 32 elements"):
        dw.cconv_fwd(d, x, w[:2], b, y)
    with pytest.raises(ValueError, match="float32"):
        dw.cconv_fwd(d, x.double(), w, b, y)
    s = dw.sscan_desc(6, 8)
    with pytest.raises(ValueError, match="kept must be"):
        dw.sscan_fwd(s, x, x, m.out((8, 16)), m.out((6, 16)), m.out((6, 16)), y, None, kept=torch.empty(4, device="cuda"))
