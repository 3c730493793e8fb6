"""Bits of the gated delta rule: answers do not depend on what else a call is asked for, and bf16 tensors lose nothing but their own rounding.

The kernels hold 24 bits of whatever they compute, so a call with bf16 tensors does what one with fp32 tensors of the same numbers does, in the same order (the further parts of its
factors are zeros), and rounds at the end.  What may differ is whether the compiler fuses a product with the sum that it goes into, which moves the sum by at most half a step of the
product, 2^-24 of it.  On the way of an element behind the matrix instructions there are three such places at most (a gradient of q or k: the part that the state has in it, the sum over
its row, what the length takes off), and their terms are of the size of the tensor's largest element or less: less than 2^-22 of that.  So an element has to be the rounding of something
that is no further than that from fp32's."""
import pytest
import torch

import paper_1803_09926_amd as dw

from test_gpu_delta import RAGGED, Call, host_inputs
from test_gpu_sequence import Made

pytestmark = pytest.mark.gpu

SIZES = [(1, 1, 1, 1), (2, 4, 24, 40), (1, 2, 40, 33), (2, 2, 64, 64), (1, 2, 64, 130), (1, 2, 128, 128), (1, 1, 200, 48)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("piece", [0, 1, 2])
@pytest.mark.parametrize("Hk,H,K,V", SIZES)
def test_answers_do_not_depend_on_what_else_is_asked(gpu_lib, dtype, piece, Hk, H, K, V):
    print("asked", dtype, piece, Hk, H, K, V, flush=True)
    m = Made(K * 7 + V, dtype)
    x, par = host_inputs(m, 420, Hk, H, K, V, 0.3)
    bounds = [0, 0, 250, 251, 251, 420]
    init = m.host((5, H, K, V), 0.3, stored=False)
    with dw.tuning_overrides({"DWCONV_TUNE_GDELTA_PIECE": piece}):
        call = Call(m, x, par, bounds)
        y, final = call.forward(init, keep=True, last=True)
        for keep, last in ((True, False), (False, True), (False, False)):
            other, states = call.forward(init, keep=keep, last=last)
            assert torch.equal(other, y), (keep, last)
            assert states is None or torch.equal(states, final), (keep, last)


@pytest.mark.parametrize("piece", [0, 2])
@pytest.mark.parametrize("Hk,H,K,V", SIZES)
def test_bf16_tensors_round_what_fp32_tensors_hold(gpu_lib, piece, Hk, H, K, V):
    print("rounded", piece, Hk, H, K, V, flush=True)
    m = Made(K * 5 + V, "bf16")
    x, par = host_inputs(m, 200, Hk, H, K, V, 0.3)
    dy = m.host(x["v"].shape)
    init = m.host((len(RAGGED) - 1, H, K, V), 0.3, stored=False)
    got = {}
    with dw.tuning_overrides({"DWCONV_TUNE_GDELTA_PIECE": piece}):
        for dtype in ("f32", "bf16"):
            call = Call(Made(0, dtype), x, par, RAGGED)
            y, final = call.forward(init)
            alone, _ = call.forward(init, keep=False, last=False)
            call.forward(init)
            got[dtype] = {"y": y, "y alone": alone, "final": final} | call.backward(dy)
    for k, wide in got["f32"].items():
        if K == 1 and k in ("dq", "dk"):             # (what is left of a difference of numbers that are alike but for their last bits, as in test_gpu_delta.check)
            continue
        stored = got["bf16"][k]
        off = wide.abs().max() * 2.0 ** -22
        assert bool(((wide - off).to(stored.dtype) <= stored).all()) and bool((stored <= (wide + off).to(stored.dtype)).all()), k
