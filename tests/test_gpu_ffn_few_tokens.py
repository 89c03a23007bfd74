"""Products of nine to 32 tokens whose rows start on 16-byte boundaries, and of up to
eight whose rows do not: ragged contractions, tokens short of a whole eight, and
outputs short of a whole sixteen.  Against 64 bits, within the bounds of the other
sizes' tests."""
import pytest

import test_gpu_linear as L
from _ffn import BF16, FP32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("T,K,N,act,bias,res,dt,save", [
    (9, 1001, 777, "silu", True, True, BF16, True),
    (9, 64, 5, "none", False, False, FP32, False),
    (13, 2050, 130, "gelu", True, True, FP32, True),
    (15, 333, 15, "relu", True, False, BF16, True),
    (16, 4099, 2001, "none", True, True, FP32, False),
    (17, 1001, 300, "silu", True, True, BF16, True),
    (25, 515, 1021, "gelu", True, False, FP32, True),
    (31, 7, 33, "none", False, True, BF16, False),
    (32, 2047, 1000, "none", True, True, FP32, True),
    (32, 4096, 4096, "silu", False, False, BF16, False),
])
def test_linear_of_few_tokens(T, K, N, act, bias, res, dt, save):
    L.test_linear(T, K, N, act, bias, res, dt, save, "padded")


@pytest.mark.parametrize("T,K,H,act,bias,save", [
    (9, 1001, 777, "silu", True, True),
    (11, 63, 9, "gelu", True, True),
    (13, 2050, 130, "relu", True, True),
    (16, 515, 2731, "silu", True, True),
    (16, 2048, 5461, "none", False, False),
    (1, 1023, 2731, "silu", True, True),
    (1, 1023, 2400, "gelu", True, True),
    (1, 2047, 2731, "relu", False, True),
])
def test_gated_of_few_tokens(T, K, H, act, bias, save):
    L.test_gated(T, K, H, act, bias, save, "padded")


@pytest.mark.parametrize("layout", ["odd", "offset", "dense"])
@pytest.mark.parametrize("T,K,N,act,bias,save", [
    (1, 2047, 5461, "silu", True, True),
    (1, 33, 9, "gelu", True, True),
    (1, 515, 130, "none", False, False),
    (2, 1001, 777, "silu", True, True),
    (5, 333, 15, "relu", True, True),
    (8, 4099, 301, "gelu", False, True),
])
def test_unaligned_rows_of_few_tokens(T, K, N, act, bias, save, layout):
    L.test_linear(T, K, N, act, bias, True, FP32 if bias else BF16, save, layout)
    L.test_gated(T, K, N, act, bias, save, layout)
