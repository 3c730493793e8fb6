"""Oracle of the sequence operators, on the CPU in 64 bits: the formulas written out token by token and sequence by sequence, in numpy.
Test infrastructure only; shares no code with the kernels.  bounds: the first token of each sequence, and the number of tokens."""
import numpy as np


def layer_norm(x, w, b, eps, residual=None):
    """(y, mean, rstd, s)"""
    s = x.astype(np.float64) + (0.0 if residual is None else residual.astype(np.float64))
    mean = s.mean(1)
    rstd = 1.0 / np.sqrt(((s - mean[:, None]) ** 2).mean(1) + eps)
    xhat = (s - mean[:, None]) * rstd[:, None]
    return xhat * (1.0 if w is None else w.astype(np.float64)) + (0.0 if b is None else b.astype(np.float64)), mean, rstd, s


def layer_norm_bwd(s, w, mean, rstd, dy, dtotal=None):
    """(dx, dw, db)"""
    s, dy, mean, rstd = (v.astype(np.float64) for v in (s, dy, mean, rstd))
    xhat = (s - mean[:, None]) * rstd[:, None]
    g = dy * (1.0 if w is None else w.astype(np.float64))
    dx = rstd[:, None] * (g - g.mean(1, keepdims=True) - xhat * (g * xhat).mean(1, keepdims=True))
    return dx + (0.0 if dtotal is None else dtotal.astype(np.float64)), (dy * xhat).sum(0), dy.sum(0)


def _sigmoid(v):
    with np.errstate(over="ignore"):
        return 1.0 / (1.0 + np.exp(-v))


def conv(x, w, b, bounds, init=None, silu=True):
    """(y, final)"""
    x, w = x.astype(np.float64), w.astype(np.float64)
    K, C = w.shape
    y = np.zeros_like(x)
    final = np.zeros((len(bounds) - 1, K - 1, C))
    for s, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):
        head = np.zeros((K - 1, C)) if init is None else init[s].astype(np.float64)
        line = np.concatenate([head, x[lo:hi]])
        for t in range(hi - lo):
            p = (w * line[t:t + K]).sum(0) + (0.0 if b is None else b.astype(np.float64))
            y[lo + t] = p * _sigmoid(p) if silu else p
        final[s] = line[hi - lo:]
    return y, final


def conv_bwd(x, w, b, bounds, dy, init=None, silu=True):
    """(dx, dw, db)"""
    x, w, dy = x.astype(np.float64), w.astype(np.float64), dy.astype(np.float64)
    K, C = w.shape
    dx, dw, db = np.zeros_like(x), np.zeros_like(w), np.zeros(C)
    for s, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):
        head = np.zeros((K - 1, C)) if init is None else init[s].astype(np.float64)
        line = np.concatenate([head, x[lo:hi]])
        dline = np.zeros_like(line)
        for t in range(hi - lo):
            p = (w * line[t:t + K]).sum(0) + (0.0 if b is None else b.astype(np.float64))
            q = _sigmoid(p)
            dp = dy[lo + t] * (q * (1.0 + p * (1.0 - q)) if silu else 1.0)
            dline[t:t + K] += w * dp
            dw += line[t:t + K] * dp
            db += dp
        dx[lo:hi] = dline[K - 1:]
    return dx, dw, db


def _steps(dt, dt_bias, softplus):
    raw = dt.astype(np.float64) + (0.0 if dt_bias is None else dt_bias.astype(np.float64))
    return raw, (np.logaddexp(raw, 0.0) if softplus else raw)


def scan(x, dt, A, B, C, bounds, D=None, z=None, dt_bias=None, init=None, softplus=True):
    """(y, final, h of every token); B and C are [T, groups, N]"""
    x, A, B, C = (v.astype(np.float64) for v in (x, A, B, C))
    T, ch = x.shape
    N, group = A.shape[1], np.arange(ch) // (ch // B.shape[1])
    _, delta = _steps(dt, dt_bias, softplus)
    y, hs, final = np.zeros_like(x), np.zeros((T, ch, N)), np.zeros((len(bounds) - 1, ch, N))
    for s, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):
        h = np.zeros((ch, N)) if init is None else init[s].astype(np.float64)
        for t in range(lo, hi):
            h = np.exp(delta[t][:, None] * A) * h + (delta[t] * x[t])[:, None] * B[t][group]
            hs[t] = h
            y[t] = (h * C[t][group]).sum(1)
        final[s] = h
    y = y + (0.0 if D is None else D.astype(np.float64) * x)
    if z is not None:
        zz = z.astype(np.float64)
        y = y * zz * _sigmoid(zz)
    return y, final, hs


def scan_bwd(x, dt, A, B, C, bounds, dy, D=None, z=None, dt_bias=None, init=None, softplus=True):
    """The gradients by name"""
    x, A, B, C, dy = (v.astype(np.float64) for v in (x, A, B, C, dy))
    T, ch = x.shape
    G, N = B.shape[1], A.shape[1]
    group = np.arange(ch) // (ch // G)
    raw, delta = _steps(dt, dt_bias, softplus)
    Dv = np.zeros(ch) if D is None else D.astype(np.float64)
    v, _, hs = scan(x, dt, A, B, C, bounds, D, None, dt_bias, init, softplus)
    out = {"dA": np.zeros_like(A), "dB": np.zeros_like(B), "dC": np.zeros_like(C), "dx": np.zeros_like(x)}
    dv = dy
    if z is not None:
        zz = z.astype(np.float64)
        q = _sigmoid(zz)
        dv = dy * zz * q
        out["dz"] = dy * v * q * (1.0 + zz * (1.0 - q))
    ddelta = np.zeros_like(x)
    for s, (lo, hi) in enumerate(zip(bounds[:-1], bounds[1:])):
        g = np.zeros((ch, N))
        for t in range(hi - 1, lo - 1, -1):
            before = hs[t - 1] if t > lo else np.zeros((ch, N)) if init is None else init[s].astype(np.float64)
            a = np.exp(delta[t][:, None] * A)
            g = g + dv[t][:, None] * C[t][group]
            gB = (g * B[t][group]).sum(1)
            for k in range(G):
                out["dC"][t, k] = (dv[t][:, None] * hs[t])[group == k].sum(0)
                out["dB"][t, k] = (g * (delta[t] * x[t])[:, None])[group == k].sum(0)
            out["dx"][t] = Dv * dv[t] + delta[t] * gB
            r = g * a * before
            ddelta[t] = x[t] * gB + (r * A).sum(1)
            out["dA"] += r * delta[t][:, None]
            g = g * a
    out["ddt"] = ddelta * (_sigmoid(raw) if softplus else 1.0)
    out["ddt_bias"] = out["ddt"].sum(0)
    out["dD"] = (dv * x).sum(0)
    return out
