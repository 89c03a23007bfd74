"""dx = dres in the norm's backward pass, which the header allows: the same bits as with an
output of its own."""
import pytest
import torch

import _ffn as F
from _ffn import BF16, FP32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("rows,cols,xdt,ydt,layout", [
    (5, 200, FP32, BF16, "padded"), (5, 201, FP32, BF16, "odd"), (3000, 1153, FP32, BF16, "dense"),
    (2000, 2048, BF16, BF16, "dense"), (700, 8000, BF16, FP32, "offset"), (4, 40000, FP32, FP32, "dense"),
])
def test_norm_backward_onto_the_residual_gradient(rows, cols, xdt, ydt, layout):
    from paper_1807_11091_gb300 import sadmm
    g = F.gen(rows + cols)
    x, dy = F.matrix(g, rows, cols, xdt, layout, 1.5, 0.5), F.matrix(g, rows, cols, ydt, layout, 0.1)
    dres = F.matrix(g, rows, cols, xdt, layout, 0.1)
    ga = torch.randn(cols, generator=g, device="cuda")
    _, mean, rstd = sadmm.layer_norm(x, stats=True)
    want = sadmm.layer_norm_backward(dy, x, mean, rstd, ga, dres=dres)
    dg, db = torch.empty(cols, device="cuda"), torch.empty(cols, device="cuda")
    code = {BF16: sadmm.SADMM_BF16, FP32: sadmm.SADMM_FP32}
    a = sadmm.LayerNormBwdArgs(rows=rows, cols=cols, x=x.data_ptr(), ldx=x.stride(0), xdt=code[xdt], dy=dy.data_ptr(),
                               lddy=dy.stride(0), dydt=code[ydt], gamma=ga.data_ptr(), mean=mean.data_ptr(),
                               rstd=rstd.data_ptr(), dres=dres.data_ptr(), lddres=dres.stride(0), dx=dres.data_ptr(),
                               lddx=dres.stride(0), dgamma=dg.data_ptr(), dbeta=db.data_ptr())
    before = F.guard(dres)
    need = sadmm.sadmm_layernorm_bwd_workspace_size(a)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    st = sadmm.sadmm_layernorm_bwd(a, ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream)
    assert st == sadmm.SADMM_OK and sadmm.device_status() == 0
    assert torch.equal(dres, want[0]) and torch.equal(dg, want[1]) and torch.equal(db, want[2])
    assert F.untouched(dres, before)
