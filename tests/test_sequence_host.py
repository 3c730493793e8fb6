"""Host-side checks of the sequence operators' C ABI and binding: exports, structs, and every refusal before the first HIP call (no GPU needed)."""
import ctypes
import os
import re

import pytest
import torch

import paper_1803_09926_amd as dw
from paper_1803_09926_amd import sequence as sq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
TEXT = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "seqops.h")).read(), flags=re.S)
OK, E_NULL, E_DIM, E_ENUM, E_WS, E_ALIGN, E_UNSUP, E_LARGE = 0, -1, -2, -3, -4, -5, -6, -8

DESCS = {"lnorm": lambda **k: dw.lnorm_desc(**{"T": 6, "C": 8, **k}),
         "cconv": lambda **k: dw.cconv_desc(**{"T": 6, "C": 8, "sequences": 2, **k}),
         "sscan": lambda **k: dw.sscan_desc(**{"T": 6, "C": 8, "sequences": 2, **k})}
CALLS = ["lnorm_fwd", "lnorm_bwd", "cconv_fwd", "cconv_bwd", "cconv_step", "sscan_fwd", "sscan_bwd", "sscan_step"]
NEEDED = {"lnorm_fwd": "x y", "lnorm_bwd": "x mean rstd dy dx", "cconv_fwd": "x w y", "cconv_bwd": "x w dy dx dw", "cconv_step": "x w state y",
          "sscan_fwd": "x dt A B C y", "sscan_bwd": "x dt A B C kept dy dx ddt dA dB dC", "sscan_step": "x dt A B C state y"}
HUGE = 1 << 40


def _call(name, d, space=0x9000, nbytes=HUGE, **pointers):
    """A call with addresses that are never followed: all that are needed, but for those given."""
    struct = sq._STRUCT[name.split("_")[0]][0]
    at = {k: 0x1000 * (i + 16) for i, k in enumerate(NEEDED[name].split())}
    io = struct(**{**at, **pointers})
    args = (ctypes.byref(d), ctypes.byref(io)) + ((space, nbytes) if name in sq._WORKSPACE else ()) + (None,)
    return getattr(sq._lib(), name)(*args)


def test_library_exports_every_declared_symbol():
    declared = set(re.findall(r"\b((?:lnorm|cconv|sscan)_[a-z_]+)\s*\(", TEXT))
    assert declared == set(sq.SEQ_EXPORTS)
    for name in declared:
        assert hasattr(dw.load(), name), name


@pytest.mark.parametrize("name,desc", [("lnorm_desc", sq.LnormDesc), ("cconv_desc", sq.CconvDesc), ("sscan_desc", sq.SscanDesc)])
def test_descriptors_match_the_header(name, desc):
    body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (name, name), TEXT, re.S).group(1)
    fields = [(f.strip(), kind) for kind, names in re.findall(r"(int32_t|int64_t|float)\s+([^;]+);", body) for f in names.split(",")]
    assert fields == [(f, {4: "float" if t is ctypes.c_float else "int32_t", 8: "int64_t"}[ctypes.sizeof(t)]) for f, t in desc._fields_]


@pytest.mark.parametrize("name", ["lnorm", "cconv", "sscan"])
def test_structs_of_tensors_match_the_header(name):
    body = re.search(r"typedef struct %s_tensors \{(.*?)\} %s_tensors;" % (name, name), TEXT, re.S).group(1)
    assert re.findall(r"\*(\w+)", body) == [f for f, _ in sq._STRUCT[name][0]._fields_]


@pytest.mark.parametrize("op,change,code", [
    ("lnorm", {"T": -1}, E_DIM), ("lnorm", {"C": 0}, E_DIM), ("lnorm", {"C": 16385}, E_UNSUP), ("lnorm", {"dtype": 2}, E_ENUM),
    ("lnorm", {"eps": -1.0}, E_DIM), ("lnorm", {"eps": float("nan")}, E_DIM),
    ("cconv", {"T": -1}, E_DIM), ("cconv", {"C": 0}, E_DIM), ("cconv", {"K": 1}, E_DIM), ("cconv", {"K": 9}, E_UNSUP), ("cconv", {"sequences": 0}, E_DIM),
    ("cconv", {"dtype": -1}, E_ENUM), ("cconv", {"silu": 2}, E_ENUM), ("cconv", {"x_stride": 7}, E_DIM), ("cconv", {"y_stride": 0}, E_DIM),
    ("cconv", {"T": 0x7fff0002, "sequences": 1}, E_LARGE), ("cconv", {"C": (1 << 24) + 1}, E_LARGE), ("cconv", {"x_stride": 1 << 31}, E_LARGE),
    ("sscan", {"T": -1}, E_DIM), ("sscan", {"C": 0}, E_DIM), ("sscan", {"N": 0}, E_DIM), ("sscan", {"N": 65}, E_UNSUP), ("sscan", {"groups": 0}, E_DIM),
    ("sscan", {"groups": 3}, E_DIM), ("sscan", {"sequences": 0}, E_DIM), ("sscan", {"dtype": 7}, E_ENUM), ("sscan", {"softplus": 2}, E_ENUM),
    ("sscan", {"z_stride": 7}, E_DIM), ("sscan", {"dt_stride": 7}, E_DIM), ("sscan", {"b_stride": 15}, E_DIM), ("sscan", {"c_stride": 15}, E_DIM),
    ("sscan", {"y_stride": 1 << 31}, E_LARGE), ("sscan", {"T": 0x7fff0002, "sequences": 1}, E_LARGE),
])
def test_bad_descriptors(op, change, code):
    for name in CALLS:
        if name.startswith(op):
            assert _call(name, DESCS[op](**change)) == code, name
    for name in sq.SEQ_EXPORTS:
        if name.startswith(op) and name.endswith("_bytes"):
            assert getattr(dw, name)(DESCS[op](**change)) == 0


def test_reserved_field_has_to_be_zero():
    d = DESCS["sscan"]()
    d.reserved = 1
    assert _call("sscan_fwd", d) == E_ENUM


@pytest.mark.parametrize("name", CALLS)
def test_missing_and_misaligned_tensors(name):
    d = DESCS[name.split("_")[0]](**({"sequences": 6} if name.endswith("step") else {}))
    for k in NEEDED[name].split():
        if k not in ("kept",):
            assert _call(name, d, **{k: 0x1001}) == E_ALIGN, k
        assert _call(name, d, **{k: None}) == E_NULL, k
    lib = sq._lib()
    rest = (0x9000, HUGE, None) if name in sq._WORKSPACE else (None,)
    assert getattr(lib, name)(None, None, *rest) == E_NULL
    assert getattr(lib, name)(ctypes.byref(d), None, *rest) == E_NULL


def test_tensors_that_go_together():
    d = DESCS["lnorm"]()
    assert _call("lnorm_fwd", d, residual=0x1000) == E_NULL           # needs total
    assert _call("lnorm_fwd", d, mean=0x1000) == E_NULL               # with rstd
    assert _call("lnorm_bwd", d, dw=0x1000) == E_NULL                 # with db
    d = DESCS["sscan"]()
    assert _call("sscan_bwd", d, z=0x1000) == E_NULL                  # needs dz
    assert _call("sscan_bwd", d, D=0x1000) == E_NULL                  # needs dD
    assert _call("sscan_fwd", d, kept=0x1008) == E_ALIGN


def test_sequences_have_to_divide_the_tokens():
    for op in ("cconv", "sscan"):
        d = DESCS[op](T=7)
        for name in (op + "_fwd", op + "_bwd"):
            assert _call(name, d) == E_DIM
        assert _call(op + "_step", d) == E_DIM                        # seven rows, two slots, and nothing that says which


@pytest.mark.parametrize("name", ["lnorm_bwd", "cconv_bwd", "sscan_fwd", "sscan_bwd"])
def test_workspaces(name):
    op = name.split("_")[0]
    d = DESCS[op](T=4096, C=256)
    more = {"dw": 0x1000, "db": 0x2000} if name == "lnorm_bwd" else {}
    need = getattr(dw, name + "_workspace_bytes")(d)
    assert 0 < need < 1 << 30
    assert _call(name, d, None, HUGE, **more) == E_WS
    assert _call(name, d, 0x9000, need - 1, **more) == E_WS
    assert _call(name, d, 0x9008, need, **more) == E_ALIGN


def test_no_tokens_need_no_tensors_of_tokens():
    for op in ("lnorm", "cconv", "sscan"):
        for name in sq.SEQ_EXPORTS:
            if name.startswith(op) and name.endswith("_bytes"):
                assert getattr(dw, name)(DESCS[op](T=0)) == 0
    none = {k: None for k in "x y mean rstd dy dx dt B C kept ddt dB dC state".split()}
    for name in ("lnorm_fwd", "cconv_fwd", "cconv_step", "sscan_fwd", "sscan_step", "lnorm_bwd"):
        d = DESCS[name.split("_")[0]](T=0)
        assert _call(name, d, None, 0, **{k: None for k in NEEDED[name].split() if k in none}) == OK, name


@pytest.mark.parametrize("name", CALLS)
def test_host_tensors_and_other_descriptors_are_refused(name):
    op = name.split("_")[0]
    d = DESCS[op]()
    f = getattr(dw, name)
    import inspect
    args = [p for p in list(inspect.signature(f).parameters.values())[1:] if p.default is inspect.Parameter.empty]
    t = [torch.zeros(4) for _ in args]
    with pytest.raises(ValueError, match="device tensor"):
        f(d, *t)
    with pytest.raises(TypeError):
        f(object(), *t)
    d.dtype = 5
    with pytest.raises(dw.DwconvError):
        f(d, *t)
    native = sq._native or sq._bind()
    with pytest.raises(TypeError):
        getattr(native, name)(d)


def test_rows_are_recognised_whatever_the_dimensions():
    both = torch.zeros(2, 3, 16)
    half = both[..., 8:]
    assert sq._is_rows(half, 6, 8, 16) and not sq._is_rows(half, 6, 8, 8)
    assert sq._is_rows(torch.zeros(6, 8), 6, 8, 8) and sq._is_rows(torch.zeros(48), 6, 8, 8)
    assert sq._is_rows(torch.zeros(6, 2, 4), 6, 8, 8) and sq._is_rows(torch.zeros(6, 16)[:, :8].unflatten(1, (2, 4)), 6, 8, 16)
    assert sq._is_rows(torch.zeros(1, 16)[:, :8], 1, 8, 16) and sq._is_rows(torch.zeros(6, 4)[:, :1], 6, 1, 4)
    assert not sq._is_rows(torch.zeros(8, 6).t(), 6, 8, 8) and not sq._is_rows(torch.zeros(6, 7), 6, 8, 8)
    assert not sq._is_rows(torch.zeros(2, 5, 8)[:, :3], 6, 8, 8)


def test_more_rows_than_a_norm_takes():
    assert _call("lnorm_fwd", DESCS["lnorm"](T=0x7fff0001)) == E_LARGE
    assert _call("lnorm_bwd", DESCS["lnorm"](T=0x7fffffff)) == E_LARGE and dw.lnorm_bwd_workspace_bytes(DESCS["lnorm"](T=0x7fffffff)) == 0
    assert dw.lnorm_bwd_workspace_bytes(DESCS["lnorm"](T=0x7fff0000)) > 0


def test_tuning_numbers_of_zero():
    """Plans are divided by them: zero counts as one, and no size or query ends in an arithmetic fault."""
    d = DESCS["sscan"](T=4096, C=256, sequences=64)
    queries = [dw.sscan_fwd_workspace_bytes, dw.sscan_bwd_workspace_bytes, dw.sscan_kept_bytes]
    knobs = ["DWCONV_TUNE_SSCAN_FWD_BLOCKS", "DWCONV_TUNE_SSCAN_BWD_BLOCKS", "DWCONV_TUNE_SSCAN_MOST_PARTS"]
    with dw.tuning_overrides({k: 1 for k in knobs}):
        want = [q(d) for q in queries]
    with dw.tuning_overrides({k: 0 for k in knobs}):
        assert [q(d) for q in queries] == want


@pytest.mark.parametrize("call,word", [
    (lambda: _call("lnorm_fwd", DESCS["lnorm"](C=16385)), "LNORM_MAX_C"), (lambda: _call("sscan_fwd", DESCS["sscan"](N=65)), "SSCAN_MAX_N"),
    (lambda: _call("cconv_fwd", DESCS["cconv"](K=9)), "MAX_K"), (lambda: _call("cconv_fwd", DESCS["cconv"](), x=0x1001), "elements"),
    (lambda: _call("cconv_fwd", DESCS["cconv"](x_stride=1 << 31)), "stride"), (lambda: _call("cconv_fwd", DESCS["cconv"](silu=2)), "switch"),
    (lambda: _call("sscan_bwd", DESCS["sscan"](T=7)), "divide"), (lambda: _call("sscan_bwd", DESCS["sscan"](T=8), None), "workspace")])
def test_a_refusal_says_what_was_refused(call, word):
    rc = call()
    assert rc != OK and word in dw.status_string(rc)
