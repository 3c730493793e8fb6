"""The operators of a block that learns by the gated delta rule: the rule over packed token sequences, the gated norm of its heads, and the norms around the
block (C ABI in include/deltaops.h, which states the formulas).

Calls are as in sequence.py: a descriptor, input and output tensors, a workspace where one is needed, and a stream (torch's current one by default); nothing is
allocated and nothing synchronises.  Tensors of tokens are T rows whose stride the descriptor names, so parts of a projection's or a convolution's output need no
copy; all other tensors are contiguous.
"""
from __future__ import annotations

import ctypes

from . import F32
from . import sequence as _seq

MAX_KEY = MAX_VALUE = 256
MAX_RUN = 1024
MAX_CHANNELS_BLOCK = 8192

DELTA_EXPORTS = ("gdelta_kept_bytes", "gdelta_fwd_workspace_bytes", "gdelta_bwd_workspace_bytes", "gdelta_fwd", "gdelta_bwd", "gdelta_step",
                 "hnorm_fwd", "hnorm_bwd_workspace_bytes", "hnorm_bwd", "rnorm_fwd", "rnorm_bwd_workspace_bytes", "rnorm_bwd")


class GdeltaDesc(ctypes.Structure):
    """Mirror of struct gdelta_desc."""
    _fields_ = ([(k, ctypes.c_int32) for k in ("T", "H", "K", "V", "key_heads", "sequences", "dtype", "softplus", "sigmoid", "norm")]
                + [("scale", ctypes.c_float), ("eps", ctypes.c_float)]
                + [(k, ctypes.c_int64) for k in ("q_stride", "k_stride", "v_stride", "a_stride", "b_stride", "y_stride")])


class HnormDesc(ctypes.Structure):
    """Mirror of struct hnorm_desc."""
    _fields_ = ([(k, ctypes.c_int32) for k in ("T", "H", "D", "dtype", "silu")] + [("eps", ctypes.c_float)]
                + [(k, ctypes.c_int64) for k in ("x_stride", "z_stride", "y_stride")])


class RnormDesc(ctypes.Structure):
    """Mirror of struct rnorm_desc."""
    _fields_ = ([(k, ctypes.c_int32) for k in ("T", "C", "dtype", "post", "silu")] + [("eps", ctypes.c_float), ("alpha", ctypes.c_float),
                                                                                     ("reserved", ctypes.c_int32)]
                + [(k, ctypes.c_int64) for k in ("x_stride", "z_stride")])


gdelta_tensors = _seq._struct("gdelta_tensors", ("q", "k", "v", "a", "b", "A", "a_bias", "starts", "init", "y", "final", "kept", "slots", "state", "dy", "dq",
                                                 "dk", "dv", "da", "db", "dA", "da_bias"))
hnorm_tensors = _seq._struct("hnorm_tensors", ("x", "z", "w", "y", "rstd", "dy", "dx", "dz", "dw"))
rnorm_tensors = _seq._struct("rnorm_tensors", ("x", "z", "residual", "w1", "scale", "w2", "total", "y", "rstd1", "rstd2", "dy", "dtotal", "dx", "dz",
                                               "dresidual", "dw1", "dscale", "dw2"))


def gdelta_desc(T, H, K, V, key_heads=None, sequences=1, dtype=F32, scale=None, softplus=True, sigmoid=True, norm=True, eps=1e-6, q_stride=None, k_stride=None,
                v_stride=None, a_stride=None, b_stride=None, y_stride=None) -> GdeltaDesc:
    """T tokens in `sequences` sequences, H value heads with states of K x V, which share key_heads key heads (H of them by default); scale: of the output,
    K ** -0.5 by default; strides of the rows in elements (dense by default).  For gdelta_step: T rows, and `sequences` slots of carried states."""
    H, K, V = int(H), int(K), int(V)
    heads = H if key_heads is None else int(key_heads)
    dense = (heads * K, heads * K, H * V, H, H, H * V)
    strides = [int(d if s is None else s) for s, d in zip((q_stride, k_stride, v_stride, a_stride, b_stride, y_stride), dense)]
    scale = (K ** -0.5 if K > 0 else 1.0) if scale is None else float(scale)
    return GdeltaDesc(int(T), H, K, V, heads, int(sequences), int(dtype), int(softplus), int(sigmoid), int(norm), scale, float(eps), *strides)


def hnorm_desc(T, H, D, dtype=F32, eps=1e-6, silu=True, x_stride=None, z_stride=None, y_stride=None) -> HnormDesc:
    """T tokens of H runs of D channels; the gate is z * sigmoid(z), or sigmoid(z) without silu; strides of the rows in elements (dense by default)."""
    H, D = int(H), int(D)
    return HnormDesc(int(T), H, D, int(dtype), int(silu), float(eps), *[int(H * D if s is None else s) for s in (x_stride, z_stride, y_stride)])


def rnorm_desc(T, C, dtype=F32, eps=1e-6, post=True, silu=False, alpha=1.0, x_stride=None, z_stride=None) -> RnormDesc:
    """T tokens of C channels; post: the block's output is normalised; the gate is sigmoid(z), or z * sigmoid(z) with silu; alpha: what the block's output is
    multiplied by before it is added to the residual; strides of the rows of x and z in elements (dense by default)."""
    C = int(C)
    return RnormDesc(int(T), C, int(dtype), int(post), int(silu), float(eps), float(alpha), 0, *[int(C if s is None else s) for s in (x_stride, z_stride)])


# ---- what a call checks (see sequence.py) ----------------------------------------------------------------

_seq._STRUCT.update({"gdelta": (gdelta_tensors, GdeltaDesc), "hnorm": (hnorm_tensors, HnormDesc), "rnorm": (rnorm_tensors, RnormDesc)})
_seq._WORKSPACE += ("gdelta_fwd", "gdelta_bwd", "hnorm_bwd", "rnorm_bwd")
_seq._EXPORTS += DELTA_EXPORTS
_seq._ROW.update({
    "gdelta": {"q": lambda d: (d.key_heads * d.K, d.q_stride), "k": lambda d: (d.key_heads * d.K, d.k_stride), "v": lambda d: (d.H * d.V, d.v_stride),
               "a": lambda d: (d.H, d.a_stride), "b": lambda d: (d.H, d.b_stride), "y": lambda d: (d.H * d.V, d.y_stride)},
    "hnorm": {"x": lambda d: (d.H * d.D, d.x_stride), "z": lambda d: (d.H * d.D, d.z_stride), "y": lambda d: (d.H * d.D, d.y_stride)},
    "rnorm": {"x": lambda d: (d.C, d.x_stride), "z": lambda d: (d.C, d.z_stride)} | {k: (lambda d: (d.C, d.C)) for k in ("residual", "total", "y")}})
for _of in ("gdelta", "hnorm", "rnorm"):
    _seq._ROW[_of].update({"d" + k: f for k, f in _seq._ROW[_of].items()})
_states = ("f32", lambda d: d.sequences * d.H * d.K * d.V)
_seq._FLAT.update({
    "gdelta": {k: ("f32", lambda d: d.H) for k in ("A", "a_bias", "dA", "da_bias")} | {"init": _states, "final": _states, "state": _states}
    | {"starts": ("i32", lambda d: d.sequences + 1), "slots": ("i32", lambda d: d.T)},
    "hnorm": {"w": ("stored", lambda d: d.D), "dw": ("f32", lambda d: d.D), "rstd": ("f32", lambda d: d.T * d.H)},
    "rnorm": {k: ("stored", lambda d: d.C) for k in ("w1", "scale", "w2")} | {k: ("f32", lambda d: d.C) for k in ("dw1", "dscale", "dw2")}
    | {k: ("f32", lambda d: d.T) for k in ("rstd1", "rstd2")}})


def _call(symbol, d, names, tensors, workspace=None, stream=None):
    native = getattr(_seq._native or _seq._bind(), symbol)
    rc = native(d, *tensors, workspace, stream) if symbol in _seq._WORKSPACE else native(d, *tensors, stream)
    if rc != 0:
        _seq._done(rc, symbol, d, names, tensors, workspace, stream)


# ---- gated delta rule ------------------------------------------------------------------------------------

def gdelta_kept_bytes(d: GdeltaDesc) -> int:
    return _seq._bytes("gdelta_kept_bytes", d)


def gdelta_fwd_workspace_bytes(d: GdeltaDesc) -> int:
    return _seq._bytes("gdelta_fwd_workspace_bytes", d)


def gdelta_bwd_workspace_bytes(d: GdeltaDesc) -> int:
    return _seq._bytes("gdelta_bwd_workspace_bytes", d)


_FWD = ("q", "k", "v", "a", "b", "A", "a_bias", "starts", "init", "y", "final", "kept")
_BWD = ("q", "k", "v", "a", "b", "A", "a_bias", "starts", "kept", "dy", "dq", "dk", "dv", "da", "db", "dA", "da_bias")
_STEP = ("q", "k", "v", "a", "b", "A", "a_bias", "slots", "state", "y")


def gdelta_fwd(d: GdeltaDesc, q, k, v, a, b, y, workspace, A=None, a_bias=None, starts=None, init=None, final=None, kept=None, stream=None):
    """Enqueue y = what the states answer to q while they learn v at k, with decays from a (A and a_bias: fp32 [H]) and rates from b.  `starts` (int32) packs
    sequences of any lengths; init and final (fp32 [sequences,H,K,V]) carry the states from call to call; kept (a device tensor of gdelta_kept_bytes(d) bytes) gets
    what gdelta_bwd needs.  `workspace`: a device tensor of at least gdelta_fwd_workspace_bytes(d) bytes (None where there is kept)."""
    _call("gdelta_fwd", d, _FWD, (q, k, v, a, b, A, a_bias, starts, init, y, final, kept), workspace, stream)
    return y


def gdelta_bwd(d: GdeltaDesc, q, k, v, a, b, kept, dy, dq, dk, dv, da, db, workspace, A=None, a_bias=None, starts=None, dA=None, da_bias=None, stream=None):
    """Enqueue the gradients of everything that gdelta_fwd read with `kept` (init aside, which is a constant): dq, dk, dv, da and db in the rows of their tensors,
    dA and da_bias in fp32.  `workspace`: a device tensor of at least gdelta_bwd_workspace_bytes(d) bytes."""
    _call("gdelta_bwd", d, _BWD, (q, k, v, a, b, A, a_bias, starts, kept, dy, dq, dk, dv, da, db, dA, da_bias), workspace, stream)
    return dv


def gdelta_step(d: GdeltaDesc, q, k, v, a, b, state, y, A=None, a_bias=None, slots=None, stream=None):
    """Enqueue one new token for each of d.T rows; `state` (fp32 [slots,H,K,V]) is moved on in place.  slots (int32 [T]) says which slot a row has (row t slot t
    without it); a row whose slot is outside the table is padding and gets zeros."""
    _call("gdelta_step", d, _STEP, (q, k, v, a, b, A, a_bias, slots, state, y), None, stream)
    return y


# ---- norm of heads with a gate ---------------------------------------------------------------------------

def hnorm_bwd_workspace_bytes(d: HnormDesc) -> int:
    return _seq._bytes("hnorm_bwd_workspace_bytes", d)


def hnorm_fwd(d: HnormDesc, x, w, y, z=None, rstd=None, stream=None):
    """Enqueue y = each run of x divided by its root mean square, times w (may be None) and the gate of z, and the runs' rstd (fp32 [T,H]) where a backward pass
    is to follow."""
    _call("hnorm_fwd", d, ("x", "z", "w", "y", "rstd"), (x, z, w, y, rstd), None, stream)
    return y


def hnorm_bwd(d: HnormDesc, x, w, rstd, dy, dx, dw, workspace, z=None, dz=None, stream=None):
    """Enqueue dx, dw (fp32, or None) and, where there is a gate, dz.  `workspace`: a device tensor of at least hnorm_bwd_workspace_bytes(d) bytes."""
    _call("hnorm_bwd", d, ("x", "z", "w", "rstd", "dy", "dx", "dz", "dw"), (x, z, w, rstd, dy, dx, dz, dw), workspace, stream)
    return dx


# ---- norms around a block --------------------------------------------------------------------------------

def rnorm_bwd_workspace_bytes(d: RnormDesc) -> int:
    return _seq._bytes("rnorm_bwd_workspace_bytes", d)


def rnorm_fwd(d: RnormDesc, x, total, y=None, w1=None, z=None, scale=None, residual=None, w2=None, rstd1=None, rstd2=None, stream=None):
    """Enqueue total = residual + alpha * scale * (the block's output x, normalised where the descriptor says so and times w1) * the gate of z, and y = total
    normalised times w2 for the next block (None: no block follows); rstd1 and rstd2 (fp32 [T]) where a backward pass is to follow."""
    _call("rnorm_fwd", d, ("x", "z", "residual", "w1", "scale", "w2", "total", "y", "rstd1", "rstd2"), (x, z, residual, w1, scale, w2, total, y, rstd1, rstd2),
          None, stream)
    return total


def rnorm_bwd(d: RnormDesc, x, total, dx, workspace, dy=None, dtotal=None, w1=None, z=None, scale=None, w2=None, rstd1=None, rstd2=None, dz=None, dresidual=None,
              dw1=None, dscale=None, dw2=None, stream=None):
    """Enqueue dx and what else is asked for: dz (where there is z), dresidual, and dw1, dscale, dw2 (fp32).  dy and dtotal are the gradients that arrive at y and at
    total.  `workspace`: a device tensor of at least rnorm_bwd_workspace_bytes(d) bytes, where a weight's gradient is asked for."""
    _call("rnorm_bwd", d, ("x", "z", "w1", "scale", "w2", "total", "rstd1", "rstd2", "dy", "dtotal", "dx", "dz", "dresidual", "dw1", "dscale", "dw2"),
          (x, z, w1, scale, w2, total, rstd1, rstd2, dy, dtotal, dx, dz, dresidual, dw1, dscale, dw2), workspace, stream)
    return dx
