"""RMS norm: 1/rms to the last digit."""
import pytest
import torch

from _ffn import FP32
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [1, 256, 4096, 16384, 65536])
def test_rstd_is_rounded_once(cols):
    """One number in a row of 4^k: its square, the average and the average's root are exact in fp32, so
    2^k / |x| rounded once is what a rounded root and quotient give."""
    x = torch.zeros(1000, cols, device="cuda")
    x[:, cols // 3] = torch.arange(3096, 4096, 1, device="cuda")[:1000] / 64.0
    _, rstd = sadmm.rms_norm(x, eps=0.0, out_dtype=FP32, stats=True)
    assert torch.equal(rstd, (cols ** 0.5 / x[:, cols // 3].double()).float())
    assert sadmm.device_status() == 0
