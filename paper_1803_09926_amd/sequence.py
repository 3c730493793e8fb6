"""The operators around a depthwise convolution over a token sequence: layer norm, the short causal depthwise convolution, and the
selective state space scan that reads it (C ABI in include/seqops.h, which states the formulas).

As for the convolutions of the package, a call takes a descriptor, its input and output tensors, a workspace where it needs one, and a stream
(torch's current one by default); it allocates nothing and does not synchronise.  Tensors of tokens are T rows whose stride the descriptor
names, so the halves of a projection's output need no copy; all other tensors are contiguous.
"""
from __future__ import annotations

import ctypes

from . import BF16, F32, DwconvError, _stream, _workspace, load

MAX_CHANNELS_NORM = 16384
MAX_TAPS = 8
MAX_STATES = 64

SEQ_EXPORTS = ("lnorm_fwd", "lnorm_bwd_workspace_bytes", "lnorm_bwd", "cconv_fwd", "cconv_bwd_workspace_bytes", "cconv_bwd", "cconv_step",
               "sscan_kept_bytes", "sscan_fwd_workspace_bytes", "sscan_bwd_workspace_bytes", "sscan_fwd", "sscan_bwd", "sscan_step")

_EXPORTS = SEQ_EXPORTS                       # and those of delta.py, whose calls are checked here too


class LnormDesc(ctypes.Structure):
    """Mirror of struct lnorm_desc."""
    _fields_ = [("T", ctypes.c_int32), ("C", ctypes.c_int32), ("dtype", ctypes.c_int32), ("eps", ctypes.c_float)]


class CconvDesc(ctypes.Structure):
    """Mirror of struct cconv_desc."""
    _fields_ = [(k, ctypes.c_int32) for k in ("T", "C", "K", "sequences", "dtype", "silu")] + [(k, ctypes.c_int64) for k in ("x_stride", "y_stride")]


class SscanDesc(ctypes.Structure):
    """Mirror of struct sscan_desc."""
    _fields_ = ([(k, ctypes.c_int32) for k in ("T", "C", "N", "groups", "sequences", "dtype", "softplus", "reserved")]
                + [(k, ctypes.c_int64) for k in ("x_stride", "dt_stride", "z_stride", "b_stride", "c_stride", "y_stride")])


def _struct(name, fields):
    return type(name, (ctypes.Structure,), {"__doc__": "Mirror of struct %s." % name, "_fields_": [(f, ctypes.c_void_p) for f in fields]})


lnorm_tensors = _struct("lnorm_tensors", ("x", "residual", "w", "b", "y", "total", "mean", "rstd", "dy", "dtotal", "dx", "dw", "db"))
cconv_tensors = _struct("cconv_tensors", ("x", "w", "b", "starts", "init", "y", "final", "slots", "state", "dy", "dx", "dw", "db"))
sscan_tensors = _struct("sscan_tensors", ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "starts", "init", "y", "final", "kept", "slots", "state",
                                          "dy", "dx", "ddt", "dA", "dB", "dC", "dD", "dz", "ddt_bias"))


def lnorm_desc(T, C, dtype=F32, eps=1e-5) -> LnormDesc:
    """T tokens of C channels."""
    return LnormDesc(int(T), int(C), int(dtype), float(eps))


def cconv_desc(T, C, K=4, sequences=1, dtype=F32, silu=True, x_stride=None, y_stride=None) -> CconvDesc:
    """T tokens of C channels in `sequences` sequences, K taps; strides of the rows in elements (dense by default).  For cconv_step: T rows, and
    `sequences` slots of carried rows."""
    return CconvDesc(int(T), int(C), int(K), int(sequences), int(dtype), int(silu), int(C if x_stride is None else x_stride),
                     int(C if y_stride is None else y_stride))


def sscan_desc(T, C, N=16, groups=1, sequences=1, dtype=F32, softplus=True, x_stride=None, dt_stride=None, z_stride=None, b_stride=None,
               c_stride=None, y_stride=None) -> SscanDesc:
    """T tokens of C channels in `sequences` sequences, N states a channel, `groups` rows of B and C a token; strides of the rows in elements (dense
    by default).  For sscan_step: T rows, and `sequences` slots of carried states."""
    C, N, groups = int(C), int(N), int(groups)
    dense = (C, C, C, groups * N, groups * N, C)
    strides = [int(d if s is None else s) for s, d in zip((x_stride, dt_stride, z_stride, b_stride, c_stride, y_stride), dense)]
    return SscanDesc(int(T), C, N, groups, int(sequences), int(dtype), int(softplus), 0, *strides)


# ---- what a call checks and passes on --------------------------------------------------------------------
# As for the convolutions, native code (csrc/seq_binding.cpp) checks plain device tensors and calls the library, and answers None to anything else; that
# is then checked here, argument by argument.

_native = _library = None


def _lib():
    global _library
    if _library is None:
        lib = load()
        VP, SZ = ctypes.c_void_p, ctypes.c_size_t
        for name in _EXPORTS:
            f = getattr(lib, name)
            if name.endswith("_bytes"):
                f.argtypes, f.restype = [VP], SZ
            else:
                f.argtypes, f.restype = [VP, VP, VP, SZ, VP] if name in _WORKSPACE else [VP, VP, VP], ctypes.c_int
        _library = lib
    return _library


def _bind():
    global _native
    lib = _lib()
    import torch
    try:
        from . import _seq_binding as native
    except ImportError as e:
        raise RuntimeError("the binding's native part is not built: run `python -m paper_1803_09926_amd.build` (or "
                           "__graft_entry__.build()) first") from e
    native.bind(lambda symbol: ctypes.cast(getattr(lib, symbol), ctypes.c_void_p).value, *(_STRUCT[op][1] for op in _STRUCT), torch.Tensor, torch.nn.Parameter)
    _native = native
    return native


_WORKSPACE = ("lnorm_bwd", "cconv_bwd", "sscan_fwd", "sscan_bwd")

# Of each tensor: its type, and its rows (width, stride) or its number of elements, from the descriptor
_ROW = {"lnorm": {k: (lambda d: (d.C, d.C)) for k in ("x", "residual", "y", "total", "dy", "dtotal", "dx")},
        "cconv": {"x": lambda d: (d.C, d.x_stride), "y": lambda d: (d.C, d.y_stride)},
        "sscan": {"x": lambda d: (d.C, d.x_stride), "dt": lambda d: (d.C, d.dt_stride), "z": lambda d: (d.C, d.z_stride),
                  "B": lambda d: (d.groups * d.N, d.b_stride), "C": lambda d: (d.groups * d.N, d.c_stride), "y": lambda d: (d.C, d.y_stride)}}
for _of, _grads in (("cconv", ("x", "y")), ("sscan", ("x", "dt", "z", "B", "C", "y"))):
    for _k in _grads:
        _ROW[_of]["d" + _k] = _ROW[_of][_k]
_FLAT = {"lnorm": {"w": ("stored", lambda d: d.C), "b": ("stored", lambda d: d.C), "mean": ("f32", lambda d: d.T), "rstd": ("f32", lambda d: d.T),
                   "dw": ("f32", lambda d: d.C), "db": ("f32", lambda d: d.C)},
         "cconv": {"w": ("stored", lambda d: d.K * d.C), "b": ("stored", lambda d: d.C), "starts": ("i32", lambda d: d.sequences + 1),
                   "init": ("stored", lambda d: d.sequences * (d.K - 1) * d.C), "final": ("stored", lambda d: d.sequences * (d.K - 1) * d.C),
                   "state": ("stored", lambda d: d.sequences * (d.K - 1) * d.C), "slots": ("i32", lambda d: d.T),
                   "dw": ("f32", lambda d: d.K * d.C), "db": ("f32", lambda d: d.C)},
         "sscan": {"A": ("f32", lambda d: d.C * d.N), "D": ("f32", lambda d: d.C), "dt_bias": ("f32", lambda d: d.C),
                   "starts": ("i32", lambda d: d.sequences + 1), "init": ("f32", lambda d: d.sequences * d.C * d.N),
                   "final": ("f32", lambda d: d.sequences * d.C * d.N), "state": ("f32", lambda d: d.sequences * d.C * d.N),
                   "slots": ("i32", lambda d: d.T), "dA": ("f32", lambda d: d.C * d.N), "dD": ("f32", lambda d: d.C),
                   "ddt_bias": ("f32", lambda d: d.C)}}
_STRUCT = {"lnorm": (lnorm_tensors, LnormDesc), "cconv": (cconv_tensors, CconvDesc), "sscan": (sscan_tensors, SscanDesc)}


def _is_rows(t, T, width, stride) -> bool:
    """Whether t is T rows of `width`, `stride` apart, whatever its dimensions are."""
    if t.numel() != T * width:
        return False
    if t.numel() == 0:
        return True
    inner, expected, outer = 1, 1, width == 1
    if outer:
        expected = stride
    for n, s in zip(reversed(t.shape), reversed(t.stride())):
        if n == 1:
            continue
        if s != expected:
            return False
        if outer:
            expected *= n
            continue
        inner *= n
        if inner > width:
            return stride == width and t.is_contiguous()
        expected *= n
        if inner == width:
            outer, expected = True, stride
    return True


def _pointer(op, name, t, d):
    if t is None:
        return None
    import torch
    if not getattr(t, "is_cuda", False):
        raise ValueError("%s must be a device tensor" % name)
    if name == "kept":
        need = _bytes(op + "_kept_bytes", d)
        if not t.is_contiguous() or t.numel() * t.element_size() < need:
            raise ValueError("kept must be contiguous with at least %d bytes" % need)
        return t.data_ptr()
    stored = torch.float32 if d.dtype == F32 else torch.bfloat16
    row = _ROW[op].get(name)
    kind, count = ("stored", None) if row else _FLAT[op][name]
    want = {"stored": stored, "f32": torch.float32, "i32": torch.int32}[kind]
    if t.dtype != want:
        raise ValueError("%s must be %s" % (name, want))
    if row:
        width, stride = row(d)
        if not _is_rows(t, d.T, width, stride):
            raise ValueError("%s must be %d rows of %d elements, %d apart (is %s with strides %s)" % (name, d.T, width, stride, tuple(t.shape), t.stride()))
    elif t.numel() != count(d) or not t.is_contiguous():
        raise ValueError("%s must be contiguous with %d elements (has %d)" % (name, count(d), t.numel()))
    return t.data_ptr()


def _general(symbol, d, names, tensors, workspace, stream):
    """A call whose arguments native code left alone."""
    op = symbol.split("_")[0]
    struct, desc = _STRUCT[op]
    if not isinstance(d, desc):
        raise TypeError("%s takes a %s" % (symbol, desc.__name__))
    lib = _lib()
    if d.dtype not in (F32, BF16):
        raise DwconvError(-3, symbol)
    io = struct(**{k: _pointer(op, k, t, d) for k, t in zip(names, tensors)})
    if symbol not in _WORKSPACE:
        return getattr(lib, symbol)(ctypes.byref(d), ctypes.byref(io), _stream(stream))
    ws, nbytes = (None, 0) if workspace is None else _workspace(workspace)
    return getattr(lib, symbol)(ctypes.byref(d), ctypes.byref(io), ws, nbytes, _stream(stream))


def _done(rc, symbol, d, names, tensors, workspace=None, stream=None):
    if rc is None:
        from . import _bind_torch
        _bind_torch()
        rc = _general(symbol, d, names, tensors, workspace, stream)
    if rc != 0:
        raise DwconvError(rc, symbol)


def _bytes(symbol, d) -> int:
    return int(getattr(_lib(), symbol)(ctypes.byref(d)))


# ---- layer norm ------------------------------------------------------------------------------------------

def lnorm_bwd_workspace_bytes(d: LnormDesc) -> int:
    return _bytes("lnorm_bwd_workspace_bytes", d)


def lnorm_fwd(d: LnormDesc, x, w, b, y, mean=None, rstd=None, residual=None, total=None, stream=None):
    """Enqueue y = the normalised rows of x (of total = x + residual, which is written too) times w plus b, and the rows' mean and rstd (fp32) where
    a backward pass is to follow.  w and b may be None."""
    rc = (_native or _bind()).lnorm_fwd(d, x, residual, w, b, y, total, mean, rstd, stream)
    if rc != 0:
        _done(rc, "lnorm_fwd", d, ("x", "residual", "w", "b", "y", "total", "mean", "rstd"), (x, residual, w, b, y, total, mean, rstd), None, stream)
    return y


def lnorm_bwd(d: LnormDesc, x, w, mean, rstd, dy, dx, dw, db, workspace, dtotal=None, stream=None):
    """Enqueue dx, dw and db (both fp32, or both None).  x is what was normalised: total where there was a residual, whose gradient dtotal is
    added to dx.  `workspace`: a device tensor of at least lnorm_bwd_workspace_bytes(d) bytes."""
    rc = (_native or _bind()).lnorm_bwd(d, x, w, mean, rstd, dy, dtotal, dx, dw, db, workspace, stream)
    if rc != 0:
        _done(rc, "lnorm_bwd", d, ("x", "w", "mean", "rstd", "dy", "dtotal", "dx", "dw", "db"), (x, w, mean, rstd, dy, dtotal, dx, dw, db), workspace, stream)
    return dx


# ---- causal depthwise convolution ------------------------------------------------------------------------

def cconv_bwd_workspace_bytes(d: CconvDesc) -> int:
    return _bytes("cconv_bwd_workspace_bytes", d)


def cconv_fwd(d: CconvDesc, x, w, b, y, starts=None, init=None, final=None, stream=None):
    """Enqueue y = the causal depthwise convolution of x with w ([K,C]) plus b, through SiLU where the descriptor says so.  `starts` (int32) packs sequences
    of any lengths; init and final ([sequences,K-1,C]) carry a sequence's last rows from call to call."""
    rc = (_native or _bind()).cconv_fwd(d, x, w, b, starts, init, y, final, stream)
    if rc != 0:
        _done(rc, "cconv_fwd", d, ("x", "w", "b", "starts", "init", "y", "final"), (x, w, b, starts, init, y, final), None, stream)
    return y


def cconv_bwd(d: CconvDesc, x, w, b, dy, dx, dw, db, workspace, starts=None, init=None, stream=None):
    """Enqueue dx, dw (fp32 [K,C]) and db (fp32 [C], may be None).  `workspace`: a device tensor of at least cconv_bwd_workspace_bytes(d) bytes."""
    rc = (_native or _bind()).cconv_bwd(d, x, w, b, starts, init, dy, dx, dw, db, workspace, stream)
    if rc != 0:
        _done(rc, "cconv_bwd", d, ("x", "w", "b", "starts", "init", "dy", "dx", "dw", "db"), (x, w, b, starts, init, dy, dx, dw, db), workspace, stream)
    return dx


def cconv_step(d: CconvDesc, x, w, b, state, y, slots=None, stream=None):
    """Enqueue one new token for each of d.T rows; `state` ([slots,K-1,C]) is moved on in place.  slots (int32 [T]) says which slot a row has (row t
    slot t without it); a row whose slot is outside the table is padding and gets zeros."""
    rc = (_native or _bind()).cconv_step(d, x, w, b, slots, state, y, stream)
    if rc != 0:
        _done(rc, "cconv_step", d, ("x", "w", "b", "slots", "state", "y"), (x, w, b, slots, state, y), None, stream)
    return y


# ---- selective state space scan --------------------------------------------------------------------------

def sscan_kept_bytes(d: SscanDesc) -> int:
    return _bytes("sscan_kept_bytes", d)


def sscan_fwd_workspace_bytes(d: SscanDesc) -> int:
    return _bytes("sscan_fwd_workspace_bytes", d)


def sscan_bwd_workspace_bytes(d: SscanDesc) -> int:
    return _bytes("sscan_bwd_workspace_bytes", d)


def sscan_fwd(d: SscanDesc, x, dt, A, B, C, y, workspace, D=None, z=None, dt_bias=None, starts=None, init=None, final=None, kept=None, stream=None):
    """Enqueue y = the scan of x with the step sizes dt.  init and final (fp32 [sequences,C,N]) carry the states from call to call; kept (a device tensor of
    sscan_kept_bytes(d) bytes) gets what sscan_bwd needs.  `workspace`: a device tensor of at least sscan_fwd_workspace_bytes(d) bytes."""
    rc = (_native or _bind()).sscan_fwd(d, x, dt, A, B, C, D, z, dt_bias, starts, init, y, final, kept, workspace, stream)
    if rc != 0:
        _done(rc, "sscan_fwd", d, ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "starts", "init", "y", "final", "kept"),
              (x, dt, A, B, C, D, z, dt_bias, starts, init, y, final, kept), workspace, stream)
    return y


def sscan_bwd(d: SscanDesc, x, dt, A, B, C, kept, dy, dx, ddt, dA, dB, dC, workspace, D=None, z=None, dt_bias=None, starts=None, init=None, dD=None,
              dz=None, ddt_bias=None, stream=None):
    """Enqueue the gradients of everything that sscan_fwd read with `kept` (init aside, which is a constant): dx, ddt, dB, dC and dz in the rows of their
    tensors, dA, dD and ddt_bias in fp32.  `workspace`: a device tensor of at least sscan_bwd_workspace_bytes(d) bytes."""
    rc = (_native or _bind()).sscan_bwd(d, x, dt, A, B, C, D, z, dt_bias, starts, init, kept, dy, dx, ddt, dA, dB, dC, dD, dz, ddt_bias, workspace, stream)
    if rc != 0:
        _done(rc, "sscan_bwd", d, ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "starts", "init", "kept", "dy", "dx", "ddt", "dA", "dB", "dC", "dD", "dz",
                                   "ddt_bias"),
              (x, dt, A, B, C, D, z, dt_bias, starts, init, kept, dy, dx, ddt, dA, dB, dC, dD, dz, ddt_bias), workspace, stream)
    return dx


def sscan_step(d: SscanDesc, x, dt, A, B, C, state, y, D=None, z=None, dt_bias=None, slots=None, stream=None):
    """Enqueue one new token for each of d.T rows; `state` (fp32 [slots,C,N]) is moved on in place, on the slots as in cconv_step."""
    rc = (_native or _bind()).sscan_step(d, x, dt, A, B, C, D, z, dt_bias, slots, state, y, stream)
    if rc != 0:
        _done(rc, "sscan_step", d, ("x", "dt", "A", "B", "C", "D", "z", "dt_bias", "slots", "state", "y"),
              (x, dt, A, B, C, D, z, dt_bias, slots, state, y), None, stream)
    return y
