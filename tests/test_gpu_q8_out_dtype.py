"""out beside out_dtype in the calls on 8-bit tensors."""
import pytest
import torch

from _ffn import BF16, FP32, gen, matrix
from _q8 import E4M3, operand
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu


def test_an_out_for_8_bit_results_is_refused():
    g = gen(1)
    x, (q, s), W = matrix(g, 6, 200), operand(g, 6, 200), operand(g, 150, 200, True)
    for out in (matrix(g, 6, 200), matrix(g, 6, 200, FP32)):
        before = out.clone()
        with pytest.raises(TypeError, match="float8_e4m3fn"):
            sadmm.rms_norm(x, out=out, out_dtype=E4M3)
        assert torch.equal(out, before)
    out = matrix(g, 6, 150)
    before = out.clone()
    with pytest.raises(TypeError, match="float8_e4m3fn"):
        sadmm.linear8(q, s, *W, out=out, out_dtype=E4M3)
    assert torch.equal(out, before)


def test_otherwise_out_is_written_in_its_own_type():
    g = gen(2)
    x, (q, s), W = matrix(g, 6, 200), operand(g, 6, 200), operand(g, 150, 200, True)
    for asked in (None, BF16, FP32):
        out = matrix(g, 6, 200, FP32)
        assert sadmm.rms_norm(x, out=out, out_dtype=asked).data_ptr() == out.data_ptr()
        assert torch.equal(out, sadmm.rms_norm(x, out_dtype=FP32))
        out = matrix(g, 6, 150, BF16)
        assert sadmm.linear8(q, s, *W, out=out, out_dtype=asked).data_ptr() == out.data_ptr()
        assert torch.equal(out, sadmm.linear8(q, s, *W, out_dtype=BF16))
