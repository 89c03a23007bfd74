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


@pytest.mark.parametrize("T,K,N", [
    (65536, 1024, 64),   # weights' operand on the tile's 128-row side
    (65536, 64, 40),     # and the other way round
    (20000, 130, 33),
    (65536, 300, 700),
    (30001, 640, 96),
])
def test_weight_gradient_of_many_tokens(T, K, N):
    from paper_1807_11091_gb300 import sadmm
    g = F.gen(T + N)
    dy, x = F.matrix(g, T, N, layout="padded", scale=0.1), F.matrix(g, T, K, layout="padded")
    W = F.matrix(g, N, K, layout="padded")
    _, dw, _ = sadmm.linear_backward(dy, x, W, dw_dtype=FP32)
    assert sadmm.device_status() == 0
    assert off(dw, dy.double().t() @ x.double()) < 1.5e-6


@pytest.mark.parametrize("T,K,N", [(16, 8192, 20000), (8, 16384, 20000), (2, 16384, 20480), (32, 65536, 256),
                                   (1, 65536, 2048), (1, 65537, 515), (5, 30001, 20000), (7, 65535, 300),
                                   (40, 32768, 515), (40, 16384, 5000)])
def test_linear_of_long_rows(T, K, N):
    from paper_1807_11091_gb300 import sadmm
    g = F.gen(T + N)
    x, W = F.matrix(g, T, K, layout="padded"), F.matrix(g, N, K, layout="padded", scale=K ** -0.5)
    y = sadmm.linear(x, W, out_dtype=FP32)
    assert sadmm.device_status() == 0
    assert off(y, x.double() @ W.double().t()) < 1.5e-6


@pytest.mark.parametrize("T,K,H", [(40, 130, 32768), (64, 1024, 20000), (3000, 96, 40000)])
def test_input_gradient_of_many_units(T, K, H):
    """dx of the pair is one contraction over both matrices' units; dg and du are exact here (no
    activation, u a power of two and g one)."""
    from paper_1807_11091_gb300 import sadmm
    gn = F.gen(T + H)
    dh, x = F.matrix(gn, T, H, layout="padded", scale=0.1), F.matrix(gn, T, K, layout="padded")
    Wg, Wu = (F.matrix(gn, H, K, layout="padded", scale=0.1) for _ in range(2))
    g, u = torch.ones(T, H, dtype=BF16, device="cuda"), torch.full((T, H), 0.5, dtype=BF16, device="cuda")
    dx = sadmm.gated_backward(dh, x, Wg, Wu, g, u, act=sadmm.SADMM_ACT_NONE, want_dw=False, dx_dtype=FP32)[0]
    assert sadmm.device_status() == 0
    assert off(dx, 0.5 * dh.double() @ Wg.double() + dh.double() @ Wu.double()) < 1.5e-6


@pytest.mark.parametrize("T,K,H,xdt,wdt", [(100, 64, 20000, FP32, BF16), (130, 40, 9000, FP32, FP32),
                                           (4000, 70, 66, BF16, FP32), (20000, 66, 70, FP32, FP32)])
def test_products_of_long_and_short_contractions_together(T, K, H, xdt, wdt):
    """All gradients of one call, some cut and some not, within the bounds of the other sizes' test."""
    import test_gpu_linear as L
    L.test_gated_backward(T, K, H, "silu", xdt, wdt, "padded")
    L.test_linear_backward(T, K, H, "silu", BF16, xdt, wdt, "padded")
