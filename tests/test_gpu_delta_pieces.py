"""Long sequences of the gated delta rule that go in pieces: the number of chunks that the library chooses by itself, both passes, and pieces over which a state decays to nothing
(whose map is not walked where keys have length one and rates are below one).

Tolerances: those of test_gpu_delta.py.  They have room for four chunks' products; here decays of e^-0.06 a token and less forget a chunk's state to e^-3.8 over the next, so that what
earlier chunks add is a geometric sum of less than 1.03 times the last one's."""
import numpy as np
import pytest
import torch

import paper_1803_09926_amd as dw
from oracle import delta as od

import gpu_util as gu
from test_gpu_delta import TOL, TOL_WIDE, Call, host_inputs
from test_gpu_sequence import Made, _close

pytestmark = pytest.mark.gpu


def _pieces(d):
    """How many pieces the library's own choice makes at most: what `kept` has room for beyond that of sequences that are walked whole, a state and a map for each and head."""
    KP, VP = max(32, 1 << (d.K - 1).bit_length()), -(-d.V // 32) * 32
    with dw.tuning_overrides({"DWCONV_TUNE_GDELTA_PIECE": 0}):
        whole = dw.gdelta_kept_bytes(d)
    return (dw.gdelta_kept_bytes(d) - whole) / (d.H * (KP * VP + KP * KP) * 4)


def _both_passes(m, x, par, bounds, init, even=False, **options):
    call = Call(m, x, par, bounds, even=even, **options)
    y, final = call.forward(init)
    dy = m.host(x["v"].shape)
    g = call.backward(dy)
    rule = od.Rule(**x, **par, bounds=bounds, init=init, **options)
    want = rule.backward(dy)
    _close(y, rule.y, TOL[m.dtype], "y")
    _close(final, rule.final, TOL_WIDE[m.dtype], "final")
    for k in ("dq", "dk", "dv", "da", "db"):
        _close(g[k], want[k], TOL[m.dtype], k)
    for k in ("dA", "da_bias"):                        # (sums of terms of either sign: their rounding is that of the terms)
        terms = np.abs(rule.log_terms if k == "dA" else want["da"]).sum(0)
        assert (np.abs(gu.to_host(g[k]) - want[k]) <= TOL_WIDE[m.dtype] * terms).all(), k
    return call.d


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,bounds,Hk,H,K,V", [(8192, None, 2, 2, 32, 32), (8191, None, 1, 2, 64, 40), (9001, [0, 2100, 2100, 8990, 9001], 1, 1, 100, 64),
                                               (6001, None, 1, 1, 200, 72)])
def test_pieces_that_the_library_chooses(gpu_lib, dtype, T, bounds, Hk, H, K, V):
    print("chosen", dtype, T, Hk, H, K, V, flush=True)
    m = Made(T + K, dtype)
    x, par = host_inputs(m, T, Hk, H, K, V, 0.3)
    par["A"] = np.full(H, -0.3, np.float32)            # (softplus of a - 1 and about is 0.2 at least: e^-0.06)
    x["a"] = np.maximum(x["a"], np.float32(-0.5))
    par["a_bias"] = np.maximum(par["a_bias"], np.float32(-1.0))
    even = bounds is None
    bounds = bounds or [0, T]
    d = _both_passes(m, x, par, bounds, m.host((len(bounds) - 1, H, K, V), 0.3, stored=False), even)
    assert 1 < _pieces(d) < T / 64 / 2               # more than two chunks in each


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("piece", [1, 2])
@pytest.mark.parametrize("options", [{}, {"norm": False}, {"sigmoid": False}])
@pytest.mark.parametrize("Hk,H,K,V", [(1, 2, 24, 40), (1, 1, 64, 64), (2, 2, 100, 33)])
def test_a_piece_in_which_all_decays_to_nothing(gpu_lib, dtype, piece, options, Hk, H, K, V):
    """Of six pieces and more the third's decays multiply to e^-200 and the fifth's to e^-120; the others' keep something."""
    print("nothing left", dtype, piece, options, Hk, H, K, V, flush=True)
    m = Made(K + piece, dtype)
    unit = 64 * piece
    T = 6 * unit + 20
    x, par = host_inputs(m, T, Hk, H, K, V, 0.3)
    par = {"A": np.full(H, -1.0, np.float32), "a_bias": None}
    x["a"][...] = np.maximum(x["a"], np.float32(-0.5)) - np.float32(2.0)       # softplus 0.08 to 0.3
    for p, log in ((2, 200.0), (4, 120.0)):
        x["a"][unit * p:unit * (p + 1)] = log / unit + 0.0                     # (softplus of 1.9 to 3.2 is more than itself)
    if m.dtype == "bf16":
        x["a"] = torch.from_numpy(x["a"]).to(torch.bfloat16).float().numpy()
    if not options.get("norm", True):
        x["k"] = m.host(x["k"].shape, 0.15)
    if not options.get("sigmoid", True):
        x["b"] = m.host(x["b"].shape, 0.2, 0.5)
    with dw.tuning_overrides({"DWCONV_TUNE_GDELTA_PIECE": piece}):
        _both_passes(m, x, par, [0, T], m.host((1, H, K, V), 0.3, stored=False), True, **options)
        _both_passes(m, x, par, [0, 0, T - 7, T], m.host((3, H, K, V), 0.3, stored=False), **options)
