"""FeedForward8's inference pass against its own roundings in 64 bits: n and h are made 8-bit from fp32, once.

What is left are values that stand on a border between two of e4m3's.  A product's fp32 sum is known to within 2^-18 of
its terms, so one value in 2^13 falls the other way, by 2^-3 of itself: 2^-9 in norm for each of n and h, and one of the
smallest block's 77 units alone 2^-3 / sqrt 77 = 0.014.  4 U16 (0.016) hold both, and no block of a product can be
left out so."""
import pytest
import torch

import _ffn as F
from _ffn import BF16, FP32, U16
from _q8 import quantized, values
from paper_1807_11091_gb300 import run_ffn, sadmm

pytestmark = pytest.mark.gpu


def made8(v, tiles=False):
    return values(*quantized(v.float(), tiles))


def branch(b, x):
    x = x.double()
    n = made8(x * (x.square().mean(1, keepdim=True) + b.eps).rsqrt() * b.gamma.double())
    g, u = n @ made8(b.Wg, True).t(), n @ made8(b.Wu, True).t()
    return made8(g * torch.sigmoid(g) * u) @ made8(b.Wd, True).t() + b.bias.double()


@pytest.mark.parametrize("tokens,d,hidden,keep", [(1, 96, 200, 77), (40, 256, 512, 131), (700, 320, 1000, 501),
                                                  (2100, 513, 3000, 1501)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_inference(tokens, d, hidden, keep, dtype):
    b = run_ffn.make_block(d, hidden, seed=tokens, bits=8).pruned(keep)
    x = torch.randn(tokens, d, generator=F.gen(tokens), device="cuda").to(dtype)
    want = branch(b, x)
    y = b.forward(x)
    step = U16 * x.double().norm() * (dtype == BF16)
    assert y.dtype == dtype and (y.double() - x.double() - want).norm() <= 4 * U16 * want.norm() + step
    assert sadmm.device_status() == 0
