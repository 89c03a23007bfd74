"""Large gradients of products whose weights have scales of single rows: the same bits, whichever others are wanted."""
import pytest
import torch

from _ffn import BF16, FP32, gen, matrix, rounded
from _q8 import operand, product, quantized
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tiles", [False, True])
def test_linear(tiles):
    """dx: 77 tiles of 512 x 128 (with tiles 78 of 256 x 256), a few more than pairs of CTAs, whose last ones are
    computed apart."""
    tokens, n_in, n_out = 512, 9856, 2048
    g = gen(1)
    xt, Wt = operand(g, n_in, tokens, False), operand(g, n_in, n_out, tiles)
    dy = matrix(g, tokens, n_out, BF16, "padded", 0.01)
    dx, dW, db = sadmm.linear8_backward(dy, *xt, *Wt, dx_dtype=FP32, dw_dtype=FP32)
    assert torch.equal(sadmm.linear8_backward(dy, None, None, *Wt, want_dw=False, dx_dtype=FP32)[0], dx)
    assert torch.equal(sadmm.linear8_backward(dy, *xt, None, None, want_dx=False, dw_dtype=FP32)[1], dW)
    for got, d, other in ((dx, dy.double(), Wt), (dW, dy.double().t(), xt)):
        v, e = product(quantized(d.float()), other)
        assert ((got.double() - v).abs() <= rounded(v, e, FP32)).all()
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("tiles", [False, True])
def test_gated(tiles):
    tokens, n_in, hidden = 512, 9856, 1024
    g = gen(2)
    xt, Wgt, Wut = operand(g, n_in, tokens, False), operand(g, n_in, hidden, tiles), operand(g, n_in, hidden, tiles)
    dh, z, u = (matrix(g, tokens, hidden, BF16, "padded") for _ in range(3))
    dx, dWg, dWu, dbg, dbu = sadmm.gated8_backward(dh, *xt, *Wgt, *Wut, z, u, want_db=True, dx_dtype=FP32, dw_dtype=FP32)
    alone = sadmm.gated8_backward(dh, None, None, *Wgt, *Wut, z, u, want_dw=False, dx_dtype=FP32)
    assert torch.equal(alone[0], dx)
    alone = sadmm.gated8_backward(dh, *xt, *(None,) * 4, z, u, want_dx=False, dw_dtype=FP32)
    assert torch.equal(alone[1], dWg) and torch.equal(alone[2], dWu)
    assert sadmm.device_status() == 0
