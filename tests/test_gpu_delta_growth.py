"""Decays of the gated delta rule that grow within the 64 tokens that are worked on at once: right up to the bound that the contract names, and behind it NaN from the token on that
passes it, with nothing else touched.

Tolerance: as for the rule's other tests (test_gpu_delta.py), 4e-5; a logarithm of 80 is rounded to 2^-24 of itself, twice, which is 2 * 80 * 2^-24 = 1e-5 of its exponential."""
import numpy as np
import pytest
import torch

import paper_1803_09926_amd as dw
from oracle import delta as od

import gpu_util as gu
from test_gpu_delta import NAMES, Call
from test_gpu_sequence import Made, _close

pytestmark = pytest.mark.gpu

T, BOUNDS = 200, [0, 30, 170, 200]
H, K, V = 2, 24, 40


def _inputs(m, logs):
    """Tokens whose decays' logarithms are logs (of the first head; the other's are small and negative), rates of next to nothing and values of one."""
    x = {"q": m.host((T, 1, K)), "k": m.host((T, 1, K)), "v": m.host((T, H, V)), "a": m.host((T, H), 0.05, -0.1), "b": m.host((T, H), 0.3, -4.0)}
    x["a"][:, 0] = logs
    return x, {"A": np.array([1.0, 1.0], np.float32), "a_bias": None}


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("piece", [0, 1])
@pytest.mark.parametrize("first,rise", [(30, 79.0), (45, 79.0), (93, 79.0), (94, 40.0), (160, 79.0)])
def test_up_to_the_bound(gpu_lib, dtype, piece, first, rise):
    """A rise of nine tokens, at a chunk's start, inside it, at its last token, over its border (as the contract counts them), and at the sequence's end; then a fall."""
    print("growth", dtype, piece, first, rise, flush=True)
    m = Made(first, dtype)
    logs = np.full(T, -0.25, np.float32)
    logs[first:first + 9] = [0.0, 1.0, 30.0, -8.0, 4.0, 0.5, 1.5, rise - 32.0, 3.0]          # (multiples of a half: bf16 holds them, and their sums are exact)
    if first + 9 < 170:
        logs[first + 9:first + 12] = -20.0
    x, par = _inputs(m, logs)
    init = m.host((3, H, K, V), 0.3, stored=False)
    with dw.tuning_overrides({"DWCONV_TUNE_GDELTA_PIECE": piece}):
        call = Call(m, x, par, BOUNDS, softplus=False)
        y, final = call.forward(init)
        rule = od.Rule(**x, **par, bounds=BOUNDS, init=init, softplus=False)
        got, want = gu.to_host(y).reshape(T, H, V), rule.y
        tol = 4e-5 if dtype == "f32" else 1e-2
        for h in range(H):
            for s in range(3):
                _close(final[s, h], rule.final[s, h], 4e-5, "final")
            for t in range(T):                        # (token by token: their sizes differ by e^80)
                _close(torch.from_numpy(got[t, h]), want[t, h], tol, "y of token %d" % t)
        dy = m.host(x["v"].shape)
        grads, wanted = call.backward(dy), rule.backward(dy)
        for k in NAMES:
            _close(grads["d" + k], wanted["d" + k], tol, "d" + k)
        for t in (0, first - 1, 199):                 # of what does not grow with them
            for k in ("dq", "dv"):
                _close(grads[k][t], wanted[k][t], tol, "%s of token %d" % (k, t))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("piece", [0, 1])
@pytest.mark.parametrize("empty", [False, True])
@pytest.mark.parametrize("at", [30, 50, 93, 94, 130])
def test_what_is_behind_the_bound_does_not_reach_what_was_before(gpu_lib, dtype, piece, empty, at):
    """e^96 over three tokens, on a state of something or of nothing, then as much the other way."""
    print("beyond", dtype, piece, empty, at, flush=True)
    m = Made(at, dtype)
    logs = np.full(T, -0.25, np.float32)
    with dw.tuning_overrides({"DWCONV_TUNE_GDELTA_PIECE": piece}):
        def run(logs):
            m.r = np.random.default_rng(at)
            x, par = _inputs(m, logs)
            if empty:
                x["v"][...] = 0
            call = Call(m, x, par, BOUNDS, softplus=False)
            y, final = call.forward(None if empty else m.host((3, H, K, V), 0.3, stored=False))
            g = call.backward(m.host(x["v"].shape))
            return [gu.to_host(y).reshape(T, H, V), gu.to_host(final)] + [gu.to_host(g["d" + k]) for k in NAMES]

        clean = run(logs)
        logs[at:at + 6] = [32.0, 32.0, 32.0, -32.0, -32.0, -32.0]
        y, final, *grads = run(logs)
    was, states = clean[:2]
    third = at + 2                                     # the token at which the run has 96: the chunk's first token counts its own decay, from the state on
    assert np.array_equal(y[:, 1], was[:, 1]) and np.array_equal(final[:, 1], states[:, 1])
    assert np.array_equal(y[:at], was[:at]) and np.array_equal(y[170:], was[170:]) and np.array_equal(final[[0, 2]], states[[0, 2]])
    assert np.isfinite(y[:third]).all()
    if (at - 30) % 64 < 62:                            # (a run over a chunk's border is two there)
        assert np.isnan(y[third:170, 0]).all() and np.isnan(final[1, 0]).all()
    for g, c in zip(grads, clean[2:]):                 # of other sequences (those of the other head where it has rows of its own)
        out = np.r_[0:30, 170:200]
        assert np.array_equal(g[out], c[out])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("value", [0.0, np.nan, np.inf])
def test_a_query_ends_nothing_but_its_own_answer(gpu_lib, dtype, value):
    """Without eps a query of zeros has no length: where decays grow too, its token's answer alone is not finite."""
    m = Made(77, dtype)
    logs = np.full(T, -0.25, np.float32)
    logs[[40, 41, 100, 180]] = 2.0
    x, par = _inputs(m, logs)
    init = m.host((3, H, K, V), 0.3, stored=False)

    def run():
        y, final = Call(m, x, par, BOUNDS, softplus=False, eps=0.0).forward(init)
        return gu.to_host(y).reshape(T, H, V), gu.to_host(final)

    was, states = run()
    assert np.isfinite(was).all() and np.isfinite(states).all()
    x["q"][101] = value
    y, final = run()
    assert np.isnan(y[101]).all() and np.array_equal(final, states)
    assert np.array_equal(np.delete(y, 101, 0), np.delete(was, 101, 0))


def test_single_tokens_have_no_bound(gpu_lib):
    m = Made(5, "f32")
    logs = np.zeros(T, np.float32)
    logs[:6] = [32.0, 32.0, 32.0, -32.0, -32.0, -32.0]
    x, par = _inputs(m, logs)
    state = m.host((1, H, K, V), 1e-12, stored=False)
    rule = od.Rule(**{k: v[:6] for k, v in x.items()}, **par, bounds=[0, 6], init=state, softplus=False)
    st = m.dev(state, stored=False)
    for t in range(6):
        call = Call(m, {k: v[t:t + 1] for k, v in x.items()}, par, [0, 1], softplus=False)
        y = call.rows("y")
        dw.gdelta_step(call.d, *(call.t[k] for k in NAMES), st, y, **call.par)
        _close(y[0, :V], rule.y[t, 0], 4e-5, "y of token %d" % t)
    _close(st, rule.final, 4e-5, "state")
