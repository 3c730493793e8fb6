"""The selective scan where the decay over many tokens passes the range of a float: states that grow (A above zero, or step sizes below it), from zeros and from small numbers, and
infinities that decay.  The tokens are split as finely as they may be, so that each part's state comes from those before it."""
import numpy as np
import pytest
import torch

import paper_1803_09926_amd as dw
from oracle import sequence as seq

from test_gpu_sequence_nonfinite import TOL, _both_ways, _positive, _same

pytestmark = pytest.mark.gpu

FINE = {"DWCONV_TUNE_SSCAN_FWD_BLOCKS": 4096, "DWCONV_TUNE_SSCAN_BWD_BLOCKS": 4096}


@pytest.mark.parametrize("N", [5, 16])
@pytest.mark.parametrize("steps", ["zeros", "there and back"])
def test_states_that_grow(gpu_lib, N, steps):
    T, C = 290, 24
    v, dy = _positive(N, T, C, N, 1, "f32")
    v["dt_bias"] = None
    if steps == "zeros":
        # nothing comes in before the last 20 tokens, and no gradient behind the first 20: zeros, however much they would have grown
        v["A"], v["dt"] = np.ones((C, N), np.float32), np.ones((T, C), np.float32)
        v["x"][:-20] = 0
        dy[20:] = 0
    else:
        # up by exp(60) in 120 tokens, and back down
        v["A"], v["dt"] = np.full((C, N), 0.5, np.float32), np.where(np.arange(T)[:, None] % 240 < 120, 1.0, -1.0).astype(np.float32).repeat(C, 1)
    with dw.tuning_overrides(FINE):
        results = _both_ways(v, dy, [0, T], 1, "f32", softplus=False)
    for k, (got, want) in results.items():
        # a decay is off by its exponent's rounding: 90 * 2^-24 over a part's way of 60 / ln 2 in each direction, 5e-6, on top of what 290 tokens have
        _same(got, want, 5e-5, k)


@pytest.mark.parametrize("N", [3, 16])
def test_an_infinity_that_decays_stays_one(gpu_lib, N):
    T, C = 290, 24
    v, dy = _positive(N, T, C, N, 1, "f32")
    v["A"] = (v["A"] - 2).astype(np.float32)               # by exp(-1) a token at the least: far below the smallest float at the end
    v["dt"] = np.abs(v["dt"]) + 0.5
    v["x"][5, 3] = np.inf
    with dw.tuning_overrides(FINE):
        results = _both_ways(v, dy, [0, T], 1, "f32")
    for k in ("y", "final"):
        _same(*results[k], TOL["f32"], k)
