"""What calls of the gated delta rule with device tensors refuse: a `kept` with too little room, in calls that go by the binding's native part and by Python."""
import pytest
import torch

import paper_1803_09926_amd as dw

from test_gpu_delta import NAMES, Call, host_inputs
from test_gpu_sequence import Made, _space

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("T,piece", [(70, 0), (200, 0), (200, 1)])
def test_kept_has_to_have_room(gpu_lib, dtype, T, piece):
    m = Made(T, dtype)
    x, par = host_inputs(m, T, 1, 2, 24, 40)
    with dw.tuning_overrides({"DWCONV_TUNE_GDELTA_PIECE": piece}):
        call = Call(m, x, par, [0, T])
        ins = [call.t[k] for k in NAMES]
        need = dw.gdelta_kept_bytes(call.d)
        with pytest.raises(ValueError, match="kept must be contiguous with at least %d bytes" % need):
            dw.gdelta_fwd(call.d, *ins, call.rows("y"), None, **call.par, starts=call.starts, kept=_space(need - 1))
        y, kept = call.rows("y"), _space(need)
        dw.gdelta_fwd(call.d, *ins, y, None, **call.par, starts=call.starts, kept=kept)
        dy, out, back = torch.ones_like(y), [call.rows(k) for k in NAMES], _space(dw.gdelta_bwd_workspace_bytes(call.d))
        with pytest.raises(ValueError, match="kept must be"):
            dw.gdelta_bwd(call.d, *ins, kept[:-1], dy, *out, back, **call.par, starts=call.starts)
        with pytest.raises(dw.DwconvError):
            dw.gdelta_bwd(call.d, *ins, kept, dy, *out, back[:-1], **call.par, starts=call.starts)
        dw.gdelta_bwd(call.d, *ins, kept, dy, *out, back, **call.par, starts=call.starts)
        assert all(torch.isfinite(o).all() for o in out)
