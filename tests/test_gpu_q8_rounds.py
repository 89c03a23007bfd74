"""Products by CTA pairs in several rounds of tiles (76 pairs): the order of tiles across the products of one
launch, sums of two products with their last tiles apart, and the pairs' general forms.

With ReLU (or no activation) and bf16 operands dg = dh u [g > 0] and du = dh g [g > 0] are exact in fp32, and so are their
8-bit forms: the gradients are held to their product's bound, value by value."""
import pytest
import torch

from _ffn import ACT_U, ACTS, BF16, FP32, LIPSCHITZ, U32, act, check, gen, matrix, rounded
from _q8 import E4M3, check8, operand, product, quantized
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu


def gated_backward(g, tokens, n_in, hidden, tiles=(True, True), want_dx=True, want_dw=True, dtype=FP32, layout="padded"):
    xt = operand(g, n_in, tokens, False, layout) if want_dw else (None, None)
    W = [operand(g, n_in, hidden, t, layout) if want_dx else (None, None) for t in tiles]
    dh, z, u = (matrix(g, tokens, hidden, BF16, layout) for _ in range(3))
    dx, dWg, dWu, _, _ = sadmm.gated8_backward(dh, *xt, *W[0], *W[1], z, u, act=ACTS["relu"], want_dx=want_dx,
                                               want_dw=want_dw, dx_dtype=dtype, dw_dtype=dtype)
    assert sadmm.device_status() == 0
    on = (z > 0).float()
    dg, du = dh.float() * u.float() * on, dh.float() * z.float() * on
    if want_dx:
        (v1, e1), (v2, e2) = product(quantized(dg), W[0]), product(quantized(du), W[1])
        e = e1 + e2 + U32 * (v1.abs() + v2.abs())
        check(dx, v1 + v2, rounded(v1 + v2, e, dtype), "dx")
    if want_dw:
        for got, d, what in ((dWg, dg, "dWg"), (dWu, du, "dWu")):
            v, e = product(quantized(d.t()), xt)
            check(got, v, rounded(v, e, dtype), what)


@pytest.mark.parametrize("tokens,n_in,hidden", [(1500, 2100, 2600), (2048, 1664, 3000), (1000, 5000, 1030)])
def test_weight_gradients_that_share_a_launch(tokens, n_in, hidden):
    """dWg and dWu, some hundred tiles of 512 x 128 each."""
    gated_backward(gen(tokens), tokens, n_in, hidden, want_dx=False)
    gated_backward(gen(hidden), tokens, n_in, hidden, dtype=BF16, layout="odd")


@pytest.mark.parametrize("tokens,n_in", [(19622, 250), (19712, 256), (250, 19622), (256, 39040), (5000, 2304)])
def test_sum_of_two_products_in_rounds(tokens, n_in):
    """dx = dg Wg + du Wu of a few tiles of 256 x 256 more than one or two rounds."""
    gated_backward(gen(n_in), tokens, n_in, 1100, want_dw=False)
    gated_backward(gen(tokens), tokens, n_in, 2048, want_dw=False, dtype=BF16)


@pytest.mark.parametrize("tiles", [(False, False), (True, False), (False, True)])
@pytest.mark.parametrize("tokens,n_in,hidden", [(5, 300, 200), (300, 300, 200), (1100, 640, 1500), (512, 9856, 1024),
                                                (39000, 120, 600)])
def test_weights_with_scales_of_rows(tokens, n_in, hidden, tiles):
    """Of both weights, or of one: dx in tiles of 512 x 128."""
    gated_backward(gen(tokens), tokens, n_in, hidden, tiles, want_dw=tokens < 2000)


@pytest.mark.parametrize("off", ["bias", "u's bias", "both"])
def test_biases_off_16_byte_boundaries(off):
    g = gen(5)
    tokens, n_in, n = 1000, 2048, 2048
    x, W, U = operand(g, tokens, n_in), operand(g, n, n_in, True, scale=n_in ** -0.5), operand(g, n, n_in, True, scale=n_in ** -0.5)

    def vector(away):
        b = torch.randn(n + 1, generator=g, device="cuda")[1 if away else 0:][:n]
        assert b.data_ptr() % 16 == (4 if away else 0)
        return b

    bg, bu = vector(off != "u's bias"), vector(off != "bias")
    (zg, eg), (zu, eu) = product(x, W), product(x, U)
    zg, zu = zg + bg.double(), zu + bu.double()
    eg, eu = eg + U32 * zg.abs(), eu + U32 * zu.abs()
    y = sadmm.linear8(*x, *W, bg, out_dtype=FP32)
    check(y, zg, rounded(zg, eg, FP32), "y")
    a = act("silu", zg)[0]
    ea = eg * LIPSCHITZ + ACT_U * (zg.abs() + 1)
    h = a * zu
    eh = ea * zu.abs() + (a.abs() + ea) * eu + U32 * h.abs()
    check8(*sadmm.gated8(*x, *W, *U, bg, bu), h, eh, "h")
    check(sadmm.gated8(*x, *W, *U, bg, bu, out_dtype=BF16), h, rounded(h, eh, BF16), "h")
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("tokens,n_in,n_out", [(131, 257, 96), (300, 1000, 333), (1000, 130, 2000), (2500, 2048, 1100)])
@pytest.mark.parametrize("name", ["gelu", "silu"])
@pytest.mark.parametrize("dy_dtype", [BF16, FP32])
def test_linear_gradients_in_norm(tokens, n_in, n_out, name, dy_dtype):
    """Of activations whose dz is not exact.  Against its 8-bit form in 64 bits: that of the kernel differs where a value
    stands on a border between two of e4m3's, one in 2^12 at ACT_U of an error, by 2^-3 of itself, which leaves 2^-9 in
    norm: 2^-8 for fp32 gradients, with bf16's rounding 2^-7.  No block of the contraction can be left out so."""
    g = gen(tokens)
    xt, Wt = operand(g, n_in, tokens, False), operand(g, n_in, n_out, True)
    dy, z = matrix(g, tokens, n_out, dy_dtype, "padded", 0.01), matrix(g, tokens, n_out, BF16, "padded", 1.5)
    dz = (dy.double() * act(name, z.double())[1])
    wdx, wdW = product(quantized(dz.float()), Wt)[0], product(quantized(dz.t().float()), xt)[0]
    for dtype, bound in ((FP32, 2.0 ** -8), (BF16, 2.0 ** -7)):
        dx, dW, db = sadmm.linear8_backward(dy, *xt, *Wt, z=z, act=ACTS[name], dx_dtype=dtype, dw_dtype=dtype)
        assert (dx.double() - wdx).norm() <= bound * wdx.norm()
        assert (dW.double() - wdW).norm() <= bound * wdW.norm()
        assert (db.double() - dz.sum(0)).norm() <= 2.0 ** -18 * dz.abs().sum(0).norm()
    assert sadmm.device_status() == 0
