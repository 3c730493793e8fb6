"""Pins of the sequence operators' oracle: its gradients against central differences in 64 bits, and closed forms."""
import numpy as np
import pytest

from oracle import sequence as seq

BOUNDS = [0, 4, 4, 9]


def _differences(loss, v, eps=1e-6):
    g = np.zeros_like(v)
    it = np.nditer(v, flags=["multi_index"])
    for _ in it:
        i = it.multi_index
        keep = v[i]
        v[i] = keep + eps
        up = loss()
        v[i] = keep - eps
        down = loss()
        v[i] = keep
        g[i] = (up - down) / (2 * eps)
    return g


def _near(got, want):
    # central differences of step 1e-6 on sums of about a hundred terms of order one: 1e-16 * 100 / 1e-6 of rounding, 1e-12 of curvature
    np.testing.assert_allclose(got, want, rtol=1e-6, atol=1e-7)


def test_layer_norm_gradients():
    r = np.random.default_rng(1)
    x, w, b, c = r.normal(size=(3, 7)), r.normal(size=7), r.normal(size=7), r.normal(size=(3, 7))
    loss = lambda: (seq.layer_norm(x, w, b, 1e-5)[0] * c).sum()  # noqa: E731
    _, mean, rstd, s = seq.layer_norm(x, w, b, 1e-5)
    dx, dw, db = seq.layer_norm_bwd(s, w, mean, rstd, c)
    for got, v in ((dx, x), (dw, w), (db, b)):
        _near(got, _differences(loss, v))


@pytest.mark.parametrize("silu", [False, True])
def test_conv_gradients(silu):
    r = np.random.default_rng(2)
    x, w, b, c = r.normal(size=(9, 3)), r.normal(size=(4, 3)), r.normal(size=3), r.normal(size=(9, 3))
    init = r.normal(size=(3, 3, 3))
    loss = lambda: (seq.conv(x, w, b, BOUNDS, init, silu)[0] * c).sum()  # noqa: E731
    for got, v in zip(seq.conv_bwd(x, w, b, BOUNDS, c, init, silu), (x, w, b)):
        _near(got, _differences(loss, v))


@pytest.mark.parametrize("softplus", [False, True])
def test_scan_gradients(softplus):
    r = np.random.default_rng(3)
    T, C, G, N = 9, 4, 2, 3
    v = {"x": r.normal(size=(T, C)), "dt": 0.3 + 0.1 * r.normal(size=(T, C)), "A": -np.exp(r.normal(size=(C, N))), "B": r.normal(size=(T, G, N)),
         "C": r.normal(size=(T, G, N)), "D": r.normal(size=C), "z": r.normal(size=(T, C)), "dt_bias": 0.1 * r.normal(size=C)}
    init, c = r.normal(size=(3, C, N)), r.normal(size=(T, C))
    loss = lambda: (seq.scan(bounds=BOUNDS, init=init, softplus=softplus, **v)[0] * c).sum()  # noqa: E731
    got = seq.scan_bwd(bounds=BOUNDS, dy=c, init=init, softplus=softplus, **v)
    for k in v:
        _near(got["d" + k], _differences(loss, v[k]))


def test_closed_forms():
    # constant inputs: a state that is fed 1 a token and halves is 2 - 2^(1 - t); a filter of ones counts the tokens that it has seen
    T = 6
    one = np.ones((T, 1))
    y, final, _ = seq.scan(one, one, np.full((1, 1), -np.log(2.0)), one[:, :, None], one[:, :, None], [0, T], softplus=False)
    np.testing.assert_allclose(y[:, 0], [2 - 2.0 ** (1 - t) for t in range(1, T + 1)], rtol=1e-15)
    np.testing.assert_allclose(final[0, 0, 0], 2 - 2.0 ** (1 - T), rtol=1e-15)
    y, final = seq.conv(one, np.ones((4, 1)), None, [0, 2, 2, T], silu=False)
    assert y[:, 0].tolist() == [1, 2, 1, 2, 3, 4] and final[0, :, 0].tolist() == [0, 1, 1] and final[1, :, 0].tolist() == [0, 0, 0]
    y, mean, rstd, _ = seq.layer_norm(np.array([[1.0, 3.0]]), None, None, 0.0)
    assert y.tolist() == [[-1.0, 1.0]] and mean.tolist() == [2.0] and rstd.tolist() == [1.0]
