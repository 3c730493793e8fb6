"""Host-side checks of the C ABI and binding of the delta rule's block: exports, structs, and every refusal before the first HIP call (no GPU needed)."""
import ctypes
import inspect
import os
import re

import pytest
import torch

import paper_1803_09926_amd as dw
from paper_1803_09926_amd import delta as dl
from paper_1803_09926_amd import sequence as sq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TEXT = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "deltaops.h")).read(), flags=re.S)
OK, E_NULL, E_DIM, E_ENUM, E_WS, E_ALIGN, E_UNSUP, E_LARGE = 0, -1, -2, -3, -4, -5, -6, -8

DESCS = {"gdelta": lambda **k: dw.gdelta_desc(**{"T": 6, "H": 4, "K": 8, "V": 8, "key_heads": 2, "sequences": 2, **k}),
         "hnorm": lambda **k: dw.hnorm_desc(**{"T": 6, "H": 2, "D": 8, **k}),
         "rnorm": lambda **k: dw.rnorm_desc(**{"T": 6, "C": 8, **k})}
CALLS = ["gdelta_fwd", "gdelta_bwd", "gdelta_step", "hnorm_fwd", "hnorm_bwd", "rnorm_fwd", "rnorm_bwd"]
NEEDED = {"gdelta_fwd": "q k v a b y", "gdelta_bwd": "q k v a b kept dy dq dk dv da db", "gdelta_step": "q k v a b state y", "hnorm_fwd": "x y",
          "hnorm_bwd": "x rstd dy dx", "rnorm_fwd": "x total", "rnorm_bwd": "x total rstd1 rstd2 dy dx"}
HUGE = 1 << 40


def _call(name, d, space=0x9000, nbytes=HUGE, **pointers):
    """A call with addresses that are never followed: all that are needed, but for those given."""
    struct = sq._STRUCT[name.split("_")[0]][0]
    at = {k: 0x1000 * (i + 16) for i, k in enumerate(NEEDED[name].split())}
    io = struct(**{**at, **pointers})
    args = (ctypes.byref(d), ctypes.byref(io)) + ((space, nbytes) if name in sq._WORKSPACE else ()) + (None,)
    return getattr(sq._lib(), name)(*args)


def test_library_exports_every_declared_symbol():
    declared = set(re.findall(r"\b((?:gdelta|hnorm|rnorm)_[a-z_]+)\s*\(", TEXT))
    assert declared == set(dl.DELTA_EXPORTS)
    for name in declared:
        assert hasattr(dw.load(), name) and hasattr(dw, name), name


@pytest.mark.parametrize("name", ["gdelta", "hnorm", "rnorm"])
def test_structs_match_the_header(name):
    body = re.search(r"typedef struct %s_desc \{(.*?)\} %s_desc;" % (name, name), TEXT, re.S).group(1)
    fields = [(f.strip(), kind) for kind, names in re.findall(r"(int32_t|int64_t|float)\s+([^;]+);", body) for f in names.split(",")]
    tensors, desc = sq._STRUCT[name]
    assert fields == [(f, "float" if t is ctypes.c_float else {4: "int32_t", 8: "int64_t"}[ctypes.sizeof(t)]) for f, t in desc._fields_]
    body = re.search(r"typedef struct %s_tensors \{(.*?)\} %s_tensors;" % (name, name), TEXT, re.S).group(1)
    assert re.findall(r"\*(\w+)", body) == [f for f, _ in tensors._fields_]


@pytest.mark.parametrize("op,change,code", [
    ("gdelta", {"T": -1}, E_DIM), ("gdelta", {"H": 0}, E_DIM), ("gdelta", {"K": 0}, E_DIM), ("gdelta", {"V": 0}, E_DIM), ("gdelta", {"key_heads": 3}, E_DIM),
    ("gdelta", {"key_heads": 0}, E_DIM), ("gdelta", {"sequences": 0}, E_DIM), ("gdelta", {"dtype": 2}, E_ENUM), ("gdelta", {"softplus": 2}, E_ENUM),
    ("gdelta", {"sigmoid": -1}, E_ENUM), ("gdelta", {"norm": 3}, E_ENUM), ("gdelta", {"eps": -1.0}, E_DIM), ("gdelta", {"eps": float("nan")}, E_DIM),
    ("gdelta", {"scale": float("inf")}, E_DIM), ("gdelta", {"K": 257}, E_UNSUP), ("gdelta", {"V": 257}, E_UNSUP), ("gdelta", {"q_stride": 15}, E_DIM),
    ("gdelta", {"k_stride": 15}, E_DIM), ("gdelta", {"v_stride": 31}, E_DIM), ("gdelta", {"a_stride": 3}, E_DIM), ("gdelta", {"b_stride": 3}, E_DIM),
    ("gdelta", {"y_stride": 31}, E_DIM), ("gdelta", {"y_stride": 1 << 31}, E_LARGE), ("gdelta", {"T": 0x7fff0002, "sequences": 1}, E_LARGE),
    ("gdelta", {"H": 65536, "key_heads": 1}, E_LARGE), ("gdelta", {"sequences": 0x7fff0000, "T": 0x7fff0000}, E_LARGE),
    ("gdelta", {"sequences": 0x7fff0000, "H": 65535, "key_heads": 1}, E_LARGE),
    ("hnorm", {"T": -1}, E_DIM), ("hnorm", {"H": 0}, E_DIM), ("hnorm", {"D": 0}, E_DIM), ("hnorm", {"D": 1025}, E_UNSUP), ("hnorm", {"dtype": -1}, E_ENUM),
    ("hnorm", {"silu": 2}, E_ENUM), ("hnorm", {"eps": -1e-6}, E_DIM), ("hnorm", {"x_stride": 15}, E_DIM), ("hnorm", {"z_stride": 15}, E_DIM),
    ("hnorm", {"y_stride": 15}, E_DIM), ("hnorm", {"z_stride": 1 << 31}, E_LARGE), ("hnorm", {"H": 1 << 22}, E_LARGE), ("hnorm", {"T": 0x7fff0001}, E_LARGE),
    ("rnorm", {"T": -1}, E_DIM), ("rnorm", {"C": 0}, E_DIM), ("rnorm", {"C": 8193}, E_UNSUP), ("rnorm", {"dtype": 5}, E_ENUM), ("rnorm", {"post": 2}, E_ENUM),
    ("rnorm", {"silu": 2}, E_ENUM), ("rnorm", {"eps": float("nan")}, E_DIM), ("rnorm", {"alpha": float("nan")}, E_DIM), ("rnorm", {"x_stride": 7}, E_DIM),
    ("rnorm", {"z_stride": 7}, E_DIM), ("rnorm", {"x_stride": 1 << 31}, E_LARGE), ("rnorm", {"T": 0x7fffffff}, E_LARGE),
])
def test_bad_descriptors(op, change, code):
    for name in CALLS:
        if name.startswith(op):
            assert _call(name, DESCS[op](**change)) == code, name
    for name in dl.DELTA_EXPORTS:
        if name.startswith(op) and name.endswith("_bytes"):
            assert getattr(dw, name)(DESCS[op](**change)) == 0


def test_reserved_field_has_to_be_zero():
    d = DESCS["rnorm"]()
    d.reserved = 1
    assert _call("rnorm_fwd", d) == E_ENUM


@pytest.mark.parametrize("name", CALLS)
def test_missing_and_misaligned_tensors(name):
    d = DESCS[name.split("_")[0]](**({"sequences": 6} if name.endswith("step") else {}))
    for k in NEEDED[name].split():
        assert _call(name, d, **{k: 0x1001}) == E_ALIGN, k
        assert _call(name, d, **{k: None}) == E_NULL, k
    lib = sq._lib()
    rest = (0x9000, HUGE, None) if name in sq._WORKSPACE else (None,)
    assert getattr(lib, name)(None, None, *rest) == E_NULL
    assert getattr(lib, name)(ctypes.byref(d), None, *rest) == E_NULL


def test_tensors_that_go_together():
    assert _call("gdelta_fwd", DESCS["gdelta"](), kept=0x1008) == E_ALIGN
    assert _call("gdelta_bwd", DESCS["gdelta"](), kept=0x1008) == E_ALIGN
    assert _call("gdelta_fwd", DESCS["gdelta"](), init=0x1002) == E_ALIGN
    assert _call("hnorm_bwd", DESCS["hnorm"](), z=0x1000) == E_NULL                   # needs dz
    assert _call("hnorm_bwd", DESCS["hnorm"](), dz=0x1000) == E_NULL
    d = DESCS["rnorm"]()
    assert _call("rnorm_bwd", d, z=0x1000) == E_NULL                                  # needs dz
    assert _call("rnorm_bwd", d, dy=None) == E_NULL                                   # nothing arrives
    assert _call("rnorm_bwd", d, dy=None, dtotal=0x1000, dw2=0x2000) == E_NULL        # dw2 needs dy
    assert _call("rnorm_bwd", d, dscale=0x1000) == E_NULL                             # needs scale
    d = DESCS["rnorm"](post=False)
    assert _call("rnorm_fwd", d, w1=0x1000) == E_NULL                                 # needs post
    assert _call("rnorm_bwd", d, dw1=0x1000) == E_NULL
    assert _call("rnorm_bwd", d, x=None, scale=0x1000) == E_NULL                      # x is read


def test_sequences_have_to_divide_the_tokens():
    d = DESCS["gdelta"](T=7)
    assert _call("gdelta_fwd", d) == E_DIM and _call("gdelta_bwd", d) == E_DIM
    assert _call("gdelta_step", d) == E_DIM                                           # seven rows, two slots, and nothing that says which


@pytest.mark.parametrize("name", ["gdelta_fwd", "gdelta_bwd", "hnorm_bwd", "rnorm_bwd"])
def test_workspaces(name):
    d = DESCS[name.split("_")[0]](T=4096)
    more = {"hnorm_bwd": {"dw": 0x1000}, "rnorm_bwd": {"dw2": 0x1000}}.get(name, {})
    need = getattr(dw, name + "_workspace_bytes")(d)
    assert 0 < need < 1 << 30
    assert _call(name, d, None, HUGE, **more) == E_WS
    assert _call(name, d, 0x9000, need - 1, **more) == E_WS
    assert _call(name, d, 0x9008, need, **more) == E_ALIGN


def test_kept_has_room_for_ragged_sequences():
    """Sequences of any lengths have at most T / 64 + sequences chunks, and the sizes do not depend on how the tokens are dealt out."""
    chunk = lambda T, S: dw.gdelta_kept_bytes(DESCS["gdelta"](T=T, sequences=S))  # noqa: E731
    one = chunk(1, 1)
    assert one > 0 and chunk(64, 1) == 2 * one and chunk(640, 7) == 17 * one and chunk(63, 3) == 3 * one


def test_no_tokens_need_no_tensors_of_tokens():
    for op in DESCS:
        for name in dl.DELTA_EXPORTS:
            if name.startswith(op) and name.endswith("_bytes"):
                assert getattr(dw, name)(DESCS[op](T=0)) == 0
    for name in CALLS:
        d = DESCS[name.split("_")[0]](T=0)
        assert _call(name, d, None, 0, **{k: None for k in NEEDED[name].split()}) == OK, name


@pytest.mark.parametrize("name", CALLS)
def test_host_tensors_and_other_descriptors_are_refused(name):
    d = DESCS[name.split("_")[0]]()
    f = getattr(dw, name)
    args = [p for p in list(inspect.signature(f).parameters.values())[1:] if p.default is inspect.Parameter.empty]
    t = [torch.zeros(4) for _ in args]
    with pytest.raises(ValueError, match="device tensor"):
        f(d, *t)
    with pytest.raises(TypeError):
        f(object(), *t)
    d.dtype = 5
    with pytest.raises(dw.DwconvError):
        f(d, *t)
    with pytest.raises(TypeError):
        getattr(sq._native or sq._bind(), name)(d)


@pytest.mark.parametrize("call,word", [
    (lambda: _call("gdelta_fwd", DESCS["gdelta"](K=257)), "GDELTA_MAX_K"), (lambda: _call("hnorm_fwd", DESCS["hnorm"](D=1025)), "HNORM_MAX_D"),
    (lambda: _call("rnorm_fwd", DESCS["rnorm"](C=8193)), "RNORM_MAX_C"), (lambda: _call("gdelta_fwd", DESCS["gdelta"](), None), "workspace")])
def test_a_refusal_says_what_was_refused(call, word):
    rc = call()
    assert rc != OK and word in dw.status_string(rc)
