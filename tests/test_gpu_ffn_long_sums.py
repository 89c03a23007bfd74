"""fp32 results of long contractions.  A sum inside the tensor cores loses about 1e-9
of itself per term, so the kernels take no more than 1024 terms before they add it
up in fp32: 1.0e-6 in norm, and the additions of the at most 100 pieces each lose
2^-24 of a sum that grows from nothing (rms sqrt(100 / 3) 2^-24 = 0.35e-6).  Held to
1.5e-6; sums of 4096 terms and more are off by 4e-6."""
import pytest
import torch

import _ffn as F
from _ffn import BF16, FP32

pytestmark = pytest.mark.gpu


def off(got, want):
    return float((got.double() - want).norm() / want.norm())


@pytest.mark.parametrize("T,K,N", [(16, 8192, 20000), (8, 16384, 20000), (2, 16384, 20480), (32, 65536, 256),
                                   (1, 65536, 2048), (1, 65537, 515), (5, 30001, 20000), (7, 65535, 300)])
def test_linear_of_long_rows(T, K, N):
    from paper_1807_11091_gb300 import sadmm
    g = F.gen(T + N)
    x, W = F.matrix(g, T, K, layout="padded"), F.matrix(g, N, K, layout="padded", scale=K ** -0.5)
    y = sadmm.linear(x, W, out_dtype=FP32)
    assert sadmm.device_status() == 0
    assert off(y, x.double() @ W.double().t()) < 1.5e-6
