"""The oracle of the delta rule's block against what it must be by other ways: closed forms, gradients against differences, and planted mistakes that it tells apart."""
import numpy as np
import pytest

from oracle import delta as od


def _inputs(seed, T=9, heads=2, H=4, K=5, V=3, bounds=(0, 4, 4, 9)):
    r = np.random.default_rng(seed)
    x = {"q": r.normal(size=(T, heads, K)), "k": r.normal(size=(T, heads, K)), "v": r.normal(size=(T, H, V)), "a": r.normal(size=(T, H)),
         "b": r.normal(size=(T, H)), "A": -np.exp(r.normal(size=H)), "a_bias": r.normal(size=H)}
    return x, list(bounds), r


def test_a_token_alone_writes_its_value():
    """One token on an empty state: y = scale beta (q.k) v, and the state is beta k v^T."""
    x, _, _ = _inputs(0, T=1)
    rule = od.Rule(**x, bounds=[0, 1], scale=0.5)
    kn, qn = rule.kn[0], rule.qn[0]
    assert np.allclose((kn ** 2).sum(1), 1, atol=1e-5)
    assert np.allclose(rule.y[0], 0.5 * (rule.beta[0] * (qn * kn).sum(1))[:, None] * x["v"][0])
    assert np.allclose(rule.final[0], rule.beta[0][:, None, None] * kn[:, :, None] * x["v"][0][:, None, :])


def test_a_key_seen_again_at_rate_one_is_replaced():
    """Without decay and at rate 1 the state answers a key with the last value that was written there."""
    r = np.random.default_rng(1)
    k = np.repeat(r.normal(size=(1, 1, 6)), 5, 0)
    v = r.normal(size=(5, 1, 4))
    rule = od.Rule(k, k, v, np.zeros((5, 1)), np.ones((5, 1)), [0, 5], A=np.zeros(1), scale=1.0, softplus=False, sigmoid=False, eps=0.0)
    assert np.allclose(rule.y, v)


@pytest.mark.parametrize("norm,softplus,sigmoid", [(True, True, True), (False, False, True), (True, False, False)])
def test_gradients_of_the_rule_against_differences(norm, softplus, sigmoid):
    x, bounds, r = _inputs(2)
    if not norm:
        x["k"] = x["k"] / 3
    init = r.normal(size=(3, 4, 5, 3))
    kw = dict(bounds=bounds, init=init, norm=norm, softplus=softplus, sigmoid=sigmoid)
    dy = r.normal(size=(9, 4, 3))
    grads = od.Rule(**x, **kw).backward(dy)
    for name in x:
        at = tuple(r.integers(0, n) for n in x[name].shape)
        h = 1e-6
        sides = []
        for sign in (1, -1):
            moved = {k: v.copy() for k, v in x.items()}
            moved[name][at] += sign * h
            sides.append((od.Rule(**moved, **kw).y * dy).sum())
        # (a central difference of a function of size 10: h^2 and 10 * 2^-53 / h, 1e-9 each; a factor of 100)
        assert abs((sides[0] - sides[1]) / (2 * h) - grads["d" + name][at]) < 1e-6 * max(1, abs(grads["d" + name][at])), name


def test_sequences_are_apart_and_continue():
    x, bounds, r = _inputs(3)
    whole = od.Rule(**x, bounds=[0, 9])
    first = od.Rule(**{k: v if k in ("A", "a_bias") else v[:4] for k, v in x.items()}, bounds=[0, 4])
    rest = od.Rule(**{k: v if k in ("A", "a_bias") else v[4:] for k, v in x.items()}, bounds=[0, 5], init=first.final)
    assert np.allclose(np.concatenate([first.y, rest.y]), whole.y) and np.allclose(rest.final, whole.final)
    apart = od.Rule(**x, bounds=bounds)
    assert np.allclose(apart.y[:4], first.y) and not np.allclose(apart.y[4:], rest.y) and not apart.final[1].any()


@pytest.mark.parametrize("silu", [True, False])
def test_gradients_of_the_norms_against_differences(silu):
    r = np.random.default_rng(4)
    x, z, w, dy = r.normal(size=(3, 2, 6)), r.normal(size=(3, 2, 6)), r.normal(size=6), r.normal(size=(3, 2, 6))
    dx, dw, dz = od.heads_norm_bwd(x, w, z, od.heads_norm(x, w, z, 1e-3, silu)[1], dy, silu)
    loss = lambda x, w, z: (od.heads_norm(x, w, z, 1e-3, silu)[0] * dy).sum()  # noqa: E731

    def slope(f, v):
        at, h = tuple(n // 2 for n in v.shape), 1e-6
        up, down = v.copy(), v.copy()
        up[at] += h
        down[at] -= h
        return at, (f(up) - f(down)) / (2 * h)

    for f, v, g in ((lambda t: loss(t, w, z), x, dx), (lambda t: loss(x, t, z), w, dw), (lambda t: loss(x, w, t), z, dz)):
        at, s = slope(f, v)
        assert abs(s - g[at]) < 1e-7
    p = {"w1": r.normal(size=6), "z": r.normal(size=(4, 6)), "scale": r.normal(size=6), "residual": r.normal(size=(4, 6)), "w2": r.normal(size=6)}
    x, dy, dt = r.normal(size=(4, 6)), r.normal(size=(4, 6)), r.normal(size=(4, 6))

    def total(x, **p):
        o = od.block_norm(x, 1e-3, silu=silu, alpha=0.7, **p)
        return (o["y"] * dy).sum() + (o["total"] * dt).sum()

    o = od.block_norm(x, 1e-3, silu=silu, alpha=0.7, **p)
    g = od.block_norm_bwd(x, o["total"], o["rstd1"], o["rstd2"], dy, dt, **{k: v for k, v in p.items() if k != "residual"}, silu=silu, alpha=0.7)
    for name in list(p) + ["x"]:
        at, s = slope((lambda t: total(t, **p)) if name == "x" else (lambda t: total(x, **dict(p, **{name: t}))), x if name == "x" else p[name])
        assert abs(s - g["d" + name][at]) < 1e-7, name


@pytest.mark.parametrize("mistake", ["decay after the write", "value not corrected", "heads in another order", "rate twice"])
def test_planted_mistakes_show(mistake):
    x, bounds, _ = _inputs(5)
    good = od.Rule(**x, bounds=bounds)
    T, H, V = x["v"].shape
    y = np.zeros_like(good.y)
    order = np.argsort(np.arange(H) % 2, kind="stable") if mistake == "heads in another order" else np.arange(H)
    kn, qn = good.kn[:, order], good.qn[:, order]
    for lo, hi in zip(bounds[:-1], bounds[1:]):
        S = np.zeros((H, 5, V))
        for t in range(lo, hi):
            d = good.decay[t][:, None, None]
            if mistake != "decay after the write":
                S = S * d
            read = 0 if mistake == "value not corrected" else np.einsum("hkv,hk->hv", S, kn[t])
            beta = good.beta[t][:, None] ** (2 if mistake == "rate twice" else 1)
            S = S + kn[t][:, :, None] * (beta * (x["v"][t] - read))[:, None, :]
            if mistake == "decay after the write":
                S = S * d
            y[t] = good.scale * np.einsum("hkv,hk->hv", S, qn[t])
    assert np.abs(y - good.y).max() / np.abs(good.y).max() > 0.02
