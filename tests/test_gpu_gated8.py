"""The 8-bit gated pair, forward and backward, against 64 bits."""
import pytest
import torch

from _ffn import ACT_U, ACTS, BF16, FP32, LIPSCHITZ, U32, act, check, column_sum, gen, matrix, rounded
from _q8 import E4M3, check8, operand, product, quantized, rounded8, values
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu


def forward(g, tokens, n_in, hidden, name="silu", bias=False, out=E4M3, layout="padded", tiles=True, save=False):
    x = operand(g, tokens, n_in, False, layout)
    Wg, Wu = (operand(g, hidden, n_in, tiles, layout, "rows", n_in ** -0.5) for _ in range(2))
    bg, bu = ((torch.randn(hidden, generator=g, device="cuda") for _ in range(2)) if bias else (None, None))
    got = sadmm.gated8(*x, *Wg, *Wu, bg, bu, act=ACTS[name], out_dtype=out, save=save)
    got = list(got) if isinstance(got, tuple) else [got]
    (zg, eg), (zu, eu) = product(x, Wg), product(x, Wu)
    if bias:
        zg, zu = zg + bg.double(), zu + bu.double()
        eg, eu = eg + U32 * zg.abs(), eu + U32 * zu.abs()
    if save:
        check(got.pop(), zu, rounded(zu, eu, BF16), "u")
        check(got.pop(), zg, rounded(zg, eg, BF16), "g")
    a = act(name, zg)[0]
    ea = eg * LIPSCHITZ + (0 if name == "none" else ACT_U * (zg.abs() + 1))
    h = a * zu
    eh = ea * zu.abs() + (a.abs() + ea) * eu + U32 * h.abs()
    if out == E4M3:
        check8(*got, h, eh, "h")
    else:
        check(got[0], h, rounded(h, eh, BF16), "h")
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("tokens", [1, 3, 16, 17, 40, 65, 130, 260])
@pytest.mark.parametrize("n_in,hidden", [(1, 1), (40, 17), (128, 128), (300, 129), (1153, 700)])
def test_sizes(tokens, n_in, hidden):
    g = gen(tokens + hidden)
    forward(g, tokens, n_in, hidden)
    forward(g, tokens, n_in, hidden, "gelu", True, BF16, "dense", False, True)


@pytest.mark.parametrize("layout", ["dense", "padded", "odd", "offset"])
@pytest.mark.parametrize("name", list(ACTS))
def test_layouts_and_activations(layout, name):
    for tokens in (4, 50, 200):
        forward(gen(tokens), tokens, 257, 300, name, True, E4M3, layout, tokens != 50, True)


@pytest.mark.parametrize("tokens,n_in,hidden", [(600, 1024, 1500), (2048, 512, 2048), (1025, 2000, 129)])
def test_large(tokens, n_in, hidden):
    forward(gen(tokens), tokens, n_in, hidden, "silu", False, E4M3, save=True)
    forward(gen(tokens), tokens, n_in, hidden, "relu", True, BF16, tiles=False)


def test_no_tokens_and_leading_dimensions():
    g = gen(1)
    Wg, Wu = operand(g, 70, 256, True), operand(g, 70, 256, True)
    x = torch.empty(0, 256, dtype=E4M3, device="cuda"), torch.empty(0, 2, device="cuda")
    q, s = sadmm.gated8(*x, *Wg, *Wu)
    assert q.shape == (0, 70) and s.shape == (0, 1)
    x = operand(g, 6, 256)
    q, s = sadmm.gated8(*x, *Wg, *Wu)
    q3, s3 = sadmm.gated8(x[0].view(3, 2, 256), x[1].reshape(3, 2, 2), *Wg, *Wu)
    assert torch.equal(q3.float(), q.float().view(3, 2, 70)) and torch.equal(s3, s.reshape(3, 2, 1))


def test_values_that_are_not_finite():
    """A NaN in x spoils its token, one in a weight its unit; other units keep the block's scale of finite values."""
    g = gen(2)
    for tokens in (5, 140):
        x, Wg, Wu = operand(g, tokens, 200), operand(g, 150, 200, True), operand(g, 150, 200, True)
        Wu[0][9, 3] = float("nan")
        x[0][2, 100] = float("nan")
        q, s = sadmm.gated8(*x, *Wg, *Wu)
        bad = torch.zeros(tokens, 150, dtype=torch.bool, device="cuda")
        bad[2], bad[:, 9] = True, True
        assert torch.equal(torch.isnan(q.float()), bad) and torch.isfinite(s).all()


def backward(g, tokens, n_in, hidden, name="silu", dx_dtype=None, dw_dtype=None, layout="padded"):
    xt = operand(g, n_in, tokens, False, layout)
    Wgt, Wut = operand(g, n_in, hidden, True, layout), operand(g, n_in, hidden, True, layout)
    dh = matrix(g, tokens, hidden, BF16, layout, 0.01)
    z, u = matrix(g, tokens, hidden, BF16, layout, 1.5), matrix(g, tokens, hidden, BF16, layout)
    dx, dWg, dWu, dbg, dbu = sadmm.gated8_backward(dh, *xt, *Wgt, *Wut, z, u, act=ACTS[name], want_db=True,
                                                  dx_dtype=dx_dtype, dw_dtype=dw_dtype)
    zd, ud, hd = z.double(), u.double(), dh.double()
    a, slope = act(name, zd)
    dg, du = hd * ud * slope, hd * a
    rough = 0 if name in ("none", "relu") else ACT_U * (zd.abs() + 1)
    eg = (hd * ud).abs() * rough + 2 * U32 * dg.abs()
    eu = hd.abs() * rough + U32 * du.abs()
    for got, d, e, what in ((dbg, dg, eg, "dbg"), (dbu, du, eu, "dbu")):
        v, b = column_sum(d, e)
        check(got, v, b, what)

    def made8(d, e, other):
        o = values(*other)
        return d @ o.t(), (d.shape[1] / 16 + 32) * U32 * (d.abs() @ o.abs().t()) * 1.1 + rounded8(d, e) @ o.abs().t()

    (v1, e1), (v2, e2) = made8(dg, eg, Wgt), made8(du, eu, Wut)
    check(dx, v1 + v2, rounded(v1 + v2, e1 + e2, dx.dtype), "dx")
    for got, d, e, what in ((dWg, dg, eg, "dWg"), (dWu, du, eu, "dWu")):
        v, b = made8(d.t(), e.t(), xt)
        check(got, v, rounded(v, b, got.dtype), what)
    # against the 8-bit forms by their definition: they differ where a value stands on a border between two of e4m3's, one in
    # 2^12 at ACT_U of an error, by 2^-3 of itself, which leaves 2^-9 in norm; with bf16's rounding (2^-9) less than 2^-7
    q = quantized(dg.float()), quantized(du.float())
    want = product(q[0], Wgt)[0] + product(q[1], Wut)[0]
    assert (dx.double() - want).norm() <= 2.0 ** -7 * want.norm()
    for got, d in ((dWg, dg), (dWu, du)):
        want = product(quantized(d.t().float()), xt)[0]
        assert (got.double() - want).norm() <= 2.0 ** -7 * want.norm()
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("tokens,n_in,hidden", [(1, 1, 1), (2, 40, 129), (128, 128, 128), (131, 257, 96), (300, 500, 333),
                                                (1030, 130, 700)])
@pytest.mark.parametrize("name", ["relu", "silu"])
def test_backward(tokens, n_in, hidden, name):
    backward(gen(tokens + n_in), tokens, n_in, hidden, name)
    backward(gen(tokens), tokens, n_in, hidden, name, FP32, FP32, "dense")
    backward(gen(tokens), tokens, n_in, hidden, name, BF16, FP32, "odd")


def test_backward_of_a_batch():
    backward(gen(1), 1536, 1024, 1100, "silu")


def test_backward_parts_alone():
    g = gen(3)
    xt, Wgt, Wut = operand(g, 200, 77), operand(g, 200, 130, True), operand(g, 200, 130, True)
    dh, z, u = (matrix(g, 77, 130) for _ in range(3))
    dx, dWg, dWu, dbg, dbu = sadmm.gated8_backward(dh, *xt, *Wgt, *Wut, z, u, want_db=True)
    none = (None,) * 4
    assert torch.equal(sadmm.gated8_backward(dh, None, None, *Wgt, *Wut, z, u, want_dw=False)[0], dx)
    got = sadmm.gated8_backward(dh, *xt, *none, z, u, want_dx=False)
    assert torch.equal(got[1], dWg) and torch.equal(got[2], dWu) and got[3] is None
    got = sadmm.gated8_backward(dh, None, None, *none, z, u, want_dx=False, want_dw=False, want_db=True)
    assert torch.equal(got[3], dbg) and torch.equal(got[4], dbu)


def test_no_tokens_backward():
    g = gen(4)
    Wgt, Wut = operand(g, 64, 70, True), operand(g, 64, 70, True)
    e = torch.empty(0, 70, dtype=BF16, device="cuda")
    xt = torch.empty(64, 0, dtype=E4M3, device="cuda"), torch.empty(64, 0, device="cuda")
    dx, dWg, dWu, dbg, dbu = sadmm.gated8_backward(e, *xt, *Wgt, *Wut, e, e, want_db=True)
    assert dx.shape == (0, 64) and not dWg.any() and not dWu.any() and not dbg.any() and not dbu.any()
