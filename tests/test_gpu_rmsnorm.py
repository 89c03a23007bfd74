"""RMS norm with the residual's addition, forward and backward, against 64 bits.

Bounds: the sum of a row's squares is of non-negative terms, added up at most 80 deep
(a thread's 32, 8 x 4, the warp's 5, the block's warps), so 80 U32 of itself; rstd half of that and 4 for the
division, eps and rsqrtf.  The gradients' sums of n terms: n / 32 + 80 deep."""
import pytest
import torch

from _ffn import BF16, FP32, U32, check, gen, guard, matrix, rounded, untouched
from _q8 import E4M3, check8
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu
EPS = 1e-5


def forward(x, gamma, residual, out_dtype, stats=True, **kw):
    """Runs the call; (y or (q, s), h, rstd) checked against 64 bits."""
    got = sadmm.rms_norm(x, gamma, residual, EPS, out_dtype, stats, **kw)
    got = list(got) if isinstance(got, tuple) else [got]
    rstd = got.pop() if stats else None
    h = x
    if residual is not None:
        h = got.pop()
        assert torch.equal(h, (x.float() + residual.float()).to(residual.dtype))
    cols = x.shape[-1]
    h64 = h.double().reshape(-1, cols)
    want = (h64.square().mean(1) + EPS) ** -0.5
    er = want * 44 * U32
    if stats:
        check(rstd, want, er, "rstd")
    y = h64 * want[:, None] * (1.0 if gamma is None else gamma.double())
    e = y.abs() * 48 * U32 + 2.0 ** -126
    if out_dtype == E4M3:
        check8(got[0].reshape(-1, cols), got[1].reshape(-1, got[1].shape[-1]), y, e, "y")
    else:
        check(got[0].reshape(-1, cols), y, rounded(y, e, got[0].dtype), "y")
    return got, h, rstd


@pytest.mark.parametrize("layout", ["dense", "padded", "odd", "offset"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 7), (9, 128), (5, 129), (4, 256), (17, 511), (6, 513), (2, 1153),
                                       (3, 4096), (2, 8192), (2, 8200), (2, 20001)])
def test_forward(rows, cols, layout):
    g = gen(rows * 100 + cols)
    types = [(BF16, None, E4M3), (BF16, FP32, E4M3), (FP32, FP32, BF16), (FP32, BF16, FP32), (BF16, BF16, BF16)]
    for xt, rt, out in types:
        x = matrix(g, rows, cols, xt, layout, 1.5, 0.25)
        r = None if rt is None else matrix(g, rows, cols, rt, layout, 2.0)
        gamma = torch.randn(cols, generator=g, device="cuda")
        forward(x, gamma, r, out)
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("cols", [32769, 40000])
def test_long_rows(cols):
    g = gen(cols)
    for out in (E4M3, FP32):
        for layout in ("dense", "odd"):
            x = matrix(g, 2, cols, BF16, layout)
            forward(x, torch.randn(cols, generator=g, device="cuda"), matrix(g, 2, cols, FP32, layout), out)
            forward(x, None, None, out)
    dy, x = matrix(g, 3, cols, BF16, "odd", 0.01), matrix(g, 3, cols, FP32, "odd")
    backward(g, dy, x, True, matrix(g, 3, cols, FP32, "dense"))


def test_arguments_left_out_and_leading_dimensions():
    g = gen(1)
    x = torch.randn(2, 3, 5, 200, generator=g, device="cuda").to(BF16)
    y = sadmm.rms_norm(x)
    assert y.shape == x.shape and y.dtype == BF16
    got, _, _ = forward(x, None, None, E4M3, stats=False)
    assert got[0].shape == x.shape and got[1].shape == (2, 3, 5, 2)
    q, s = got
    # what the call leaves is what the products and the quantiser take
    y32 = sadmm.rms_norm(x, out_dtype=FP32)
    q2, s2 = sadmm.quantize(y32)
    assert torch.equal(q.float(), q2.float()) and torch.equal(s, s2)


def test_in_place():
    g = gen(2)
    for cols in (130, 1024, 33000):
        for layout in ("dense", "odd"):
            x, r = matrix(g, 5, cols, BF16, layout), matrix(g, 5, cols, FP32, layout)
            want = sadmm.rms_norm(x, residual=r, out_dtype=E4M3)
            keep, before = guard(r), r.clone()
            got = sadmm.rms_norm(x, residual=r, out_dtype=E4M3, sum_out=r)
            assert got[2].data_ptr() == r.data_ptr() and torch.equal(r, want[2]) and not torch.equal(r, before)
            assert torch.equal(got[0].float(), want[0].float()) and torch.equal(got[1], want[1])
            assert untouched(r, keep)
            y = sadmm.rms_norm(x)
            keep = guard(x)
            assert sadmm.rms_norm(x, out=x).data_ptr() == x.data_ptr()
            assert torch.equal(x, y) and untouched(x, keep)


def test_values_that_are_not_finite():
    """A NaN or infinity spoils its own row (through rstd) and no other; a zero row gives zeros."""
    x = torch.ones(6, 300, device="cuda")
    x[1, 5], x[3, 250], x[4] = float("nan"), float("inf"), 0
    q, s = sadmm.rms_norm(x, out_dtype=E4M3)
    v = q.float()
    assert torch.isfinite(v[[0, 2, 4, 5]]).all() and torch.isnan(v[1]).all() and not v[4].any()
    # row 3: rstd = 0, so 0 where x is finite and NaN where it is not
    assert torch.isnan(v[3, 250]) and not v[3, :250].any() and not v[3, 251:].any()
    assert torch.isfinite(s).all()


def backward(g, dy, h, want_gamma, dres=None):
    rows, cols = h.shape
    gamma = torch.randn(cols, generator=g, device="cuda") if want_gamma else None
    rstd = (h.float().square().mean(1) + EPS).rsqrt()
    dx, dgamma = sadmm.rms_norm_backward(dy, h, rstd, gamma, dres)
    hhat, d = h.double() * rstd.double()[:, None], dy.double()
    dg = d * hhat
    check(dgamma, dg.sum(0), dg.abs().sum(0) * (rows + 8) * U32, "dgamma")
    d = d * (1.0 if gamma is None else gamma.double())
    m = (d * hhat).mean(1, keepdim=True)
    em = (d * hhat).abs().mean(1, keepdim=True) * (cols / 32 + 80) * U32
    r = rstd.double()[:, None]
    want = r * (d - hhat * m)
    e = r * (hhat.abs() * em + 6 * U32 * (d.abs() + (hhat * m).abs()))
    if dres is not None:
        want = want + dres.double()
        e = e + U32 * want.abs()
    check(dx, want, rounded(want, e, h.dtype), "dx")
    # one alone, with the same bits
    assert torch.equal(sadmm.rms_norm_backward(dy, h, rstd, gamma, dres, want_dgamma=False)[0], dx)
    assert torch.equal(sadmm.rms_norm_backward(dy, h, rstd, gamma, want_dx=False)[1], dgamma)


@pytest.mark.parametrize("layout", ["dense", "padded", "odd", "offset"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (700, 7), (9, 128), (400, 255), (33, 513), (3, 2048), (350, 2049),
                                       (2, 8192), (3, 8193)])
def test_backward(rows, cols, layout):
    g = gen(rows + cols)
    for ht, yt, res in [(BF16, BF16, True), (FP32, BF16, True), (FP32, FP32, False), (BF16, FP32, False)]:
        h = matrix(g, rows, cols, ht, layout, 1.5, 0.25)
        dy = matrix(g, rows, cols, yt, layout, 0.01)
        dres = matrix(g, rows, cols, ht, layout, 0.01) if res else None
        backward(g, dy, h, res, dres)
    assert sadmm.device_status() == 0


def test_gradient_is_the_differences():
    """dx and dgamma against central differences of the plain formula in 64 bits: an error of step^2 and
    of 64 bits over the step, far below the fp32 gradient's 1e-6."""
    g = gen(5)
    h, gamma = torch.randn(3, 40, generator=g, device="cuda"), torch.randn(40, generator=g, device="cuda")
    dy = torch.randn(3, 40, generator=g, device="cuda")
    rstd = (h.square().mean(1) + EPS).rsqrt()
    dx, dgamma = sadmm.rms_norm_backward(dy, h, rstd, gamma)

    def loss(h, gamma):
        return (h * (h.square().mean(-1, keepdim=True) + EPS).rsqrt() * gamma * dy.double()).sum((-1, -2))

    step = 1e-5
    eye = torch.eye(120, dtype=torch.float64, device="cuda").view(120, 3, 40) * step
    num = (loss(h.double() + eye, gamma.double()) - loss(h.double() - eye, gamma.double())) / (2 * step)
    assert (num.view(3, 40) - dx.double()).abs().max() < 1e-5
    eye = torch.eye(40, dtype=torch.float64, device="cuda")[:, None] * step
    num = (loss(h.double(), gamma.double() + eye) - loss(h.double(), gamma.double() - eye)) / (2 * step)
    assert (num - dgamma.double()).abs().max() < 1e-5


def test_no_rows():
    x = torch.empty(0, 300, dtype=BF16, device="cuda")
    q, s, h, rstd = sadmm.rms_norm(x, residual=x, out_dtype=E4M3, stats=True)
    assert q.shape == (0, 300) and s.shape == (0, 3) and h.shape == (0, 300) and rstd.shape == (0,)
    dx, dgamma = sadmm.rms_norm_backward(x, x, rstd)
    assert dx.shape == (0, 300) and dgamma.shape == (300,) and not dgamma.any()
