"""The gated pair's backward pass on blocks whose tokens and units are both few: all
three products then have their operands the other way round and share a launch.
Against 64 bits, within the bounds of the larger sizes' test."""
import pytest

import test_gpu_linear as L
from _ffn import BF16, FP32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,K,H,act,xdt,wdt,layout", [
    (16, 256, 64, "silu", BF16, BF16, "dense"),
    (1, 128, 40, "gelu", FP32, BF16, "padded"),
    (64, 130, 64, "relu", BF16, FP32, "odd"),
    (33, 65, 17, "none", FP32, FP32, "offset"),
    (64, 2048, 1, "silu", BF16, BF16, "padded"),
    (2, 1030, 63, "gelu", BF16, BF16, "dense"),
])
def test_gated_backward_of_few_units(T, K, H, act, xdt, wdt, layout):
    L.test_gated_backward(T, K, H, act, xdt, wdt, layout)
