"""The quantiser's quotients where a correction of x / s could go astray: scales near the smallest, and zeros
with a sign.  Compared by bytes, the signs of zeros with them."""
import pytest
import torch

from _ffn import BF16, FP32, gen
from _q8 import E4M3, FLOOR, operand, quantized
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu


def same_bytes(x, tiles=False):
    q, s, qt, st = sadmm.quantize(x, tiles=tiles, transposed=True)
    alone = sadmm.quantize(x, tiles=tiles)
    for (a, b), m in (((q, s), x), ((qt, st), x.t()), (alone, x)):
        want, scale = quantized(m, tiles)
        assert torch.equal(a.contiguous().view(torch.uint8), want.contiguous().view(torch.uint8))
        assert torch.equal(b, scale)


@pytest.mark.parametrize("tiles", [False, True])
@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_signs_of_zeros(tiles, dtype):
    g = gen(1)
    x = torch.randn(200, 300, generator=g, device="cuda").to(dtype)
    x[torch.rand(200, 300, generator=g, device="cuda") < 0.3] = 0.0
    x[torch.rand(200, 300, generator=g, device="cuda") < 0.3] *= -1
    x[5], x[6] = 0.0, -0.0
    x[7, ::2] = -1e-30  # the quotient falls to zero
    same_bytes(x, tiles)


@pytest.mark.parametrize("power", [-96, -95, -94, -90, -84, -78, -60, 100, 127])
def test_borders_at_the_ends_of_the_scales(power):
    """Rows whose scale is any fp32 number, and values a unit or two from half-way between two of e4m3's."""
    g = gen(power + 200)
    rows = 20000
    top = (torch.rand(rows, 1, generator=g, device="cuda", dtype=torch.float64) + 1) * 0.999 * 2.0 ** power
    top = top.float().clamp_min(FLOOR)
    s = top / torch.full_like(top, 448.0)
    # below 2^-6 steps of 2^-9, above it eight of them between two powers of two
    half = torch.cat([torch.arange(1, 16, 2) * 2.0 ** -10] + [(torch.arange(8, 16) + 0.5) * 2.0 ** p for p in range(-9, 5)])
    half = half.double().cuda()
    x = (s.double() * half[torch.randint(len(half), (rows, 127), generator=g, device="cuda")]).float()
    x = (x.view(torch.int32) + torch.randint(-2, 3, x.shape, generator=g, device="cuda", dtype=torch.int32)).view(FP32)
    sign = torch.randint(0, 2, x.shape, generator=g, device="cuda") * 2 - 1
    same_bytes(torch.cat([top, x * sign], 1))


def test_a_rest_below_the_normal_numbers():
    """0x1.67fdc8p-112 by 0x1.3ffe06p-105 is a unit more than 9 * 2^-10, half-way between two of e4m3's: it goes up."""
    s, x = float.fromhex("0x1.3ffe06p-105"), float.fromhex("0x1.67fdc8p-112")
    top = torch.tensor(s, dtype=torch.float64, device="cuda").mul(448).float()
    assert float(top / torch.full_like(top, 448.0)) == s
    row = torch.zeros(1, 128, device="cuda")
    row[0, 0], row[0, 1], row[0, 2] = top, x, -x
    q, scale = sadmm.quantize(row)
    assert float(scale) == s and q[0, 1:3].float().tolist() == [10 * 2.0 ** -10, -10 * 2.0 ** -10]
    same_bytes(row)


def test_signs_of_zeros_of_norms_and_gated_units():
    g = gen(2)
    y = torch.randn(40, 256, generator=g, device="cuda")
    y[:, ::3] = -0.0
    q, s = sadmm.rms_norm(y, out_dtype=E4M3)
    want = sadmm.rms_norm(y, out_dtype=FP32)
    assert torch.equal(q.contiguous().view(torch.uint8), quantized(want)[0].contiguous().view(torch.uint8))
    for tokens in (5, 300):  # ReLU's zeros times a negative u
        x, Wg, Wu = operand(g, tokens, 200), operand(g, 256, 200, True), operand(g, 256, 200, True)
        q, s, a, u = sadmm.gated8(*x, *Wg, *Wu, act=sadmm.SADMM_ACT_RELU, save=True)
        b = q.contiguous().view(torch.uint8)
        off = (a <= 0) & (a.abs() > 0) & (u.abs() > 0)
        assert off.any() and torch.equal(b[off], torch.where(u[off] < 0, 0x80, 0).to(torch.uint8))
