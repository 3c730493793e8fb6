"""Oracle of the gated delta rule, of its heads' norm and of the norms around its block, on the CPU in 64 bits: the formulas written out token by token and sequence by
sequence, in numpy.  Test infrastructure only; shares no code with the kernels.  bounds: the first token of each sequence, and the number of tokens."""
import numpy as np


def _sigmoid(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


def _act(z, silu):
    """act(z) and its slope"""
    q = _sigmoid(z)
    return (z * q, q * (1 + z * (1 - q))) if silu else (q, q * (1 - q))


def _wide(*tensors):
    return [None if t is None else np.asarray(t, np.float64) for t in tensors]


class Rule:
    """q, k: [T, key heads, K]; v: [T, H, V]; a, b: [T, H]; A, a_bias: [H] or None; init: [sequences, H, K, V] or None"""

    def __init__(self, q, k, v, a, b, bounds, A=None, a_bias=None, init=None, scale=None, softplus=True, sigmoid=True, norm=True, eps=1e-6):
        self.q, self.k, self.v, a, b, self.A, bias, self.init = _wide(q, k, v, a, b, A, a_bias, init)
        self.bounds, self.norm, self.softplus, self.sigmoid = bounds, norm, softplus, sigmoid
        T, self.heads, K = self.q.shape
        H, V = self.v.shape[1:]
        self.scale = K ** -0.5 if scale is None else scale
        self.A = -np.ones(H) if A is None else self.A
        self.raw = a + (0.0 if bias is None else bias)
        self.soft = np.logaddexp(self.raw, 0.0) if softplus else self.raw
        self.decay = np.exp(self.A * self.soft)
        self.beta = _sigmoid(b) if sigmoid else b
        length = lambda x: 1.0 / np.sqrt((x * x).sum(2, keepdims=True) + eps) if norm else np.ones_like(x[:, :, :1])  # noqa: E731
        self.rq, self.rk = length(self.q), length(self.k)
        share = np.arange(H) // (H // self.heads)
        self.qn, self.kn = (self.q * self.rq)[:, share], (self.k * self.rk)[:, share]
        self.y, self.met, self.u = np.zeros((T, H, V)), np.zeros((T, H, K, V)), np.zeros((T, H, V))
        self.final = np.zeros((len(bounds) - 1, H, K, V))
        for s, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):
            S = np.zeros((H, K, V)) if init is None else self.init[s].copy()
            for t in range(lo, hi):
                S = S * self.decay[t][:, None, None]
                self.met[t] = S
                self.u[t] = self.beta[t][:, None] * (self.v[t] - np.einsum("hkv,hk->hv", S, self.kn[t]))
                S = S + self.kn[t][:, :, None] * self.u[t][:, None, :]
                self.y[t] = self.scale * np.einsum("hkv,hk->hv", S, self.qn[t])
            self.final[s] = S

    def backward(self, dy):
        """The gradients by name"""
        dy = np.asarray(dy, np.float64) * self.scale
        T, H, V = self.v.shape
        K = self.q.shape[2]
        dq, dk, dv = np.zeros((T, H, K)), np.zeros((T, H, K)), np.zeros((T, H, V))
        dbeta, dlog = np.zeros((T, H)), np.zeros((T, H))
        for lo, hi in zip(self.bounds[:-1], self.bounds[1:]):
            g = np.zeros((H, K, V))
            for t in range(hi - 1, lo - 1, -1):
                S = self.met[t] + self.kn[t][:, :, None] * self.u[t][:, None, :]
                dq[t] = np.einsum("hkv,hv->hk", S, dy[t])
                g = g + self.qn[t][:, :, None] * dy[t][:, None, :]
                du = np.einsum("hkv,hk->hv", g, self.kn[t])
                dbeta[t] = (du * (self.v[t] - np.einsum("hkv,hk->hv", self.met[t], self.kn[t]))).sum(1)
                dv[t] = self.beta[t][:, None] * du
                dk[t] = np.einsum("hkv,hv->hk", g, self.u[t]) - np.einsum("hkv,hv->hk", self.met[t], dv[t])
                g = g - self.kn[t][:, :, None] * dv[t][:, None, :]
                dlog[t] = (g * self.met[t]).sum((1, 2))
                g = g * self.decay[t][:, None, None]
        shared = lambda x: x.reshape(T, self.heads, H // self.heads, K).sum(2)  # noqa: E731
        dq, dk = shared(dq), shared(dk)
        if self.norm:
            dq, dk = ((d - n * (d * n).sum(2, keepdims=True)) * r for d, n, r in ((dq, self.q * self.rq, self.rq), (dk, self.k * self.rk, self.rk)))
        da = dlog * self.A * (_sigmoid(self.raw) if self.softplus else 1.0)
        db = dbeta * self.beta * (1 - self.beta) if self.sigmoid else dbeta
        self.log_terms = dlog * self.soft        # of each token
        return {"dq": dq, "dk": dk, "dv": dv, "da": da, "db": db, "dA": self.log_terms.sum(0), "da_bias": da.sum(0)}


def _rms(x, eps):
    return 1.0 / np.sqrt((x * x).mean(-1) + eps)


def _rms_bwd(x, rstd, dn):
    n = x * rstd[..., None]
    return rstd[..., None] * (dn - n * (dn * n).mean(-1, keepdims=True))


def heads_norm(x, w, z, eps, silu=True):
    """(y, rstd) of x [T, H, D]"""
    x, w, z = _wide(x, w, z)
    rstd = _rms(x, eps)
    return x * rstd[..., None] * (1.0 if w is None else w) * (1.0 if z is None else _act(z, silu)[0]), rstd


def heads_norm_bwd(x, w, z, rstd, dy, silu=True):
    """(dx, dw, dz)"""
    x, w, z, rstd, dy = _wide(x, w, z, rstd, dy)
    act, slope = (1.0, 0.0) if z is None else _act(z, silu)
    w = 1.0 if w is None else w
    n = x * rstd[..., None]
    return _rms_bwd(x, rstd, dy * act * w), (dy * act * n).sum((0, 1)), dy * n * w * slope


def block_norm(x, eps, w1=None, z=None, scale=None, residual=None, w2=None, post=True, silu=False, alpha=1.0):
    """total, y, rstd1 and rstd2 by name"""
    x, w1, z, scale, residual, w2 = _wide(x, w1, z, scale, residual, w2)
    rstd1 = _rms(x, eps)
    p = x * rstd1[:, None] * (1.0 if w1 is None else w1) if post else x
    s = alpha * p * (1.0 if scale is None else scale) * (1.0 if z is None else _act(z, silu)[0]) + (0.0 if residual is None else residual)
    rstd2 = _rms(s, eps)
    return {"total": s, "y": s * rstd2[:, None] * (1.0 if w2 is None else w2), "rstd1": rstd1, "rstd2": rstd2}


def block_norm_bwd(x, total, rstd1, rstd2, dy=None, dtotal=None, w1=None, z=None, scale=None, w2=None, post=True, silu=False, alpha=1.0):
    """The gradients by name"""
    x, total, rstd1, rstd2, dy, dtotal, w1, z, scale, w2 = _wide(x, total, rstd1, rstd2, dy, dtotal, w1, z, scale, w2)
    w1, w2, scale = (1.0 if t is None else t for t in (w1, w2, scale))
    out, ds = {}, 0.0 if dtotal is None else dtotal
    if dy is not None:
        ds = ds + _rms_bwd(total, rstd2, dy * w2)
        out["dw2"] = (dy * total * rstd2[:, None]).sum(0)
    act, slope = (1.0, 0.0) if z is None else _act(z, silu)
    n = x * rstd1[:, None] if post else x
    p = n * w1 if post else n
    out |= {"dresidual": ds, "dscale": (alpha * ds * p * act).sum(0), "dz": alpha * scale * ds * p * slope}
    d = alpha * scale * ds * act
    out["dw1"] = (d * n).sum(0)
    out["dx"] = _rms_bwd(x, rstd1, d * w1) if post else d
    return out
