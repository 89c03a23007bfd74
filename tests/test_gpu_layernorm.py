"""sadmm_layernorm_fwd / _bwd against 64-bit forms."""
import pytest
import torch

import _ffn as F
from _ffn import BF16, FP32, U16, U32

pytestmark = pytest.mark.gpu

EPS = 1e-5


def lib():
    from paper_1807_11091_gb300 import sadmm
    return sadmm


# rows, cols, x dtype, y dtype, layout
CASES = [
    (1, 1, FP32, FP32, "dense"),
    (1, 2048, BF16, BF16, "dense"),
    (5, 7, BF16, FP32, "odd"),
    (9, 32, FP32, BF16, "dense"),
    (33, 255, BF16, BF16, "dense"),
    (70, 256, FP32, FP32, "padded"),
    (16, 300, FP32, BF16, "offset"),
    (40, 512, BF16, BF16, "padded"),
    (1000, 1024, BF16, BF16, "dense"),
    (13, 1000, BF16, BF16, "odd"),
    (700, 1025, FP32, BF16, "dense"),
    (300, 1153, FP32, BF16, "dense"),
    (21, 4096, FP32, FP32, "dense"),
    (17, 5000, BF16, FP32, "padded"),
    (6, 8192, BF16, BF16, "dense"),
    (5, 8193, BF16, BF16, "padded"),
    (4, 12288, FP32, BF16, "dense"),
    (3, 20001, BF16, BF16, "dense"),
    (2, 40000, FP32, FP32, "dense"),
    (3000, 40, BF16, BF16, "dense"),
    (2000, 2048, FP32, BF16, "padded"),
]


def stats(x):
    x = x.double()
    mean = x.mean(1, keepdim=True)
    return mean, ((x - mean).square().mean(1, keepdim=True) + EPS).rsqrt()


def levels(cols):
    """fp32 additions that one element passes through in a sum over a row: 32 in a thread's registers
    (or one per 1024 columns of a long row), then two trees of 5."""
    return 32 + 10 + cols / 1024


@pytest.mark.parametrize("rows,cols,xdt,ydt,layout", CASES)
@pytest.mark.parametrize("affine", [True, False])
def test_forward(rows, cols, xdt, ydt, layout, affine):
    s, g = lib(), F.gen(rows + cols)
    x = F.matrix(g, rows, cols, xdt, layout, 1.5, 0.5)
    out = F.matrix(g, rows, cols, ydt, layout)
    before = F.guard(out)
    ga = torch.randn(cols, generator=g, device="cuda") if affine else None
    be = torch.randn(cols, generator=g, device="cuda") if affine else None
    y, mean, rstd = s.layer_norm(x, ga, be, eps=EPS, stats=True, out=out)
    assert s.device_status() == 0
    wm, wr = stats(x)
    xd = x.double()
    em = levels(cols) * U32 * xd.abs().mean(1, keepdim=True)
    F.check(mean, wm[:, 0], em[:, 0] + U32 * wm[:, 0].abs(), "mean")
    # var: each (x - mean) is off by em + U32 |x - mean|; the sum of squares then by the levels.  The error of a
    # shifted mean enters squared (the deviations sum to 0); rstd moves by half the relative error of var + eps.
    dev = (xd - wm).abs()
    var = dev.square().mean(1, keepdim=True)
    ev = em.square() + (levels(cols) + 4) * U32 * var + 2 * U32 * (dev * (xd.abs() + em)).mean(1, keepdim=True)
    er = wr * (0.5 * ev * wr.square() + 4 * U32) * (1 + 1e-2)
    F.check(rstd, wr[:, 0], er[:, 0], "rstd")
    xh = (xd - wm) * wr
    eh = (em + U32 * (xd.abs() + dev)) * wr + dev * er + 2 * U32 * xh.abs()
    want = xh if not affine else xh * ga.double() + be.double()
    err = eh if not affine else eh * ga.double().abs() + 2 * U32 * (xh * ga.double()).abs() + U32 * want.abs()
    F.check(y, want, F.rounded(want, err * (1 + 1e-3), ydt), "y")
    assert F.untouched(out, before)
    assert torch.equal(s.layer_norm(x, ga, be, eps=EPS, out_dtype=ydt), y)


def backward_reference(x, dy, mean, rstd, gamma, dres, cols):
    xd, d = x.double(), dy.double()
    m, r = mean.double()[:, None], rstd.double()[:, None]
    xh = (xd - m) * r
    eh = U32 * ((xd.abs() + (xd - m).abs()) * r + 2 * xh.abs())
    e = d * gamma.double() if gamma is not None else d
    n = cols
    c1, c2 = e.mean(1, keepdim=True), (e * xh).mean(1, keepdim=True)
    lv = levels(n) + 4
    e1 = lv * U32 * e.abs().mean(1, keepdim=True)
    e2 = lv * U32 * (e * xh).abs().mean(1, keepdim=True) + (e.abs() * eh).mean(1, keepdim=True)
    dx = r * (e - c1 - xh * c2)
    err = r * (e1 + xh.abs() * e2 + eh * c2.abs() + 6 * U32 * (e.abs() + c1.abs() + (xh * c2).abs()))
    if dres is not None:
        dx = dx + dres.double()
        err = err + U32 * dx.abs()
    # column sums: any order
    k = x.shape[0] + 8
    dg, eg = (d * xh).sum(0), (d.abs() * eh).sum(0) + k * U32 * (d * xh).abs().sum(0)
    db, eb = d.sum(0), k * U32 * d.abs().sum(0)
    return dx, err * (1 + 1e-3), dg, eg, db, eb


@pytest.mark.parametrize("rows,cols,xdt,ydt,layout", CASES)
@pytest.mark.parametrize("full", [True, False])
def test_backward(rows, cols, xdt, ydt, layout, full):
    s, g = lib(), F.gen(rows * 3 + cols)
    x, dy = F.matrix(g, rows, cols, xdt, layout, 1.5, 0.5), F.matrix(g, rows, cols, ydt, layout, 0.1)
    ga = torch.randn(cols, generator=g, device="cuda") if full else None
    dres = F.matrix(g, rows, cols, xdt, layout, 0.1) if full else None
    mean, rstd = (t[:, 0].float().contiguous() for t in stats(x))
    dx, dg, db = s.layer_norm_backward(dy, x, mean, rstd, ga, dres=dres)
    assert s.device_status() == 0
    wx, ex, wg, eg, wb, eb = backward_reference(x, dy, mean, rstd, ga, dres, cols)
    F.check(dx, wx, F.rounded(wx, ex, xdt), "dx")
    F.check(dg, wg, eg + U32 * wg.abs() + 1e-30, "dgamma")
    F.check(db, wb, eb + U32 * wb.abs() + 1e-30, "dbeta")
    # each output alone gives the same bits
    for k, want in (("dx", dx), ("dgamma", dg), ("dbeta", db)):
        only = s.layer_norm_backward(dy, x, mean, rstd, ga, dres=dres if k == "dx" else None,
                                     **{f"want_{o}": o == k for o in ("dx", "dgamma", "dbeta")})
        assert torch.equal([t for t in only if t is not None][0], want)


def test_gradients_against_differences():
    """<gradient, direction> against central differences of the 64-bit loss, whose step (1e-5) leaves
    h^2 = 1e-10 of third derivatives of order 10 here; the gradient in fp32 is within the bounds of
    backward_reference, so 1e-5 of the magnitudes covers both."""
    s, g = lib(), F.gen(4)
    rows, cols = 12, 96
    x, dy = F.matrix(g, rows, cols, FP32, scale=1.5, offset=0.3), F.matrix(g, rows, cols, FP32)
    ga, be = torch.randn(cols, generator=g, device="cuda"), torch.randn(cols, generator=g, device="cuda")
    _, mean, rstd = s.layer_norm(x, ga, be, stats=True)
    grads = s.layer_norm_backward(dy, x, mean, rstd, ga)

    def loss(x, ga, be):
        m = x.mean(1, keepdim=True)
        r = ((x - m).square().mean(1, keepdim=True) + EPS).rsqrt()
        return (dy.double() * ((x - m) * r * ga + be)).sum()

    at = [t.double() for t in (x, ga, be)]
    for k, grad in enumerate(grads):
        v = torch.randn(at[k].shape, generator=g, device="cuda", dtype=torch.float64)
        hi, lo = list(at), list(at)
        hi[k], lo[k] = at[k] + 1e-5 * v, at[k] - 1e-5 * v
        diff = (loss(*hi) - loss(*lo)) / 2e-5
        mag = dy.double().abs().sum() if k == 0 else (dy.double().abs().sum(0) * v.abs()).sum()
        assert abs((grad.double() * v).sum() - diff) <= 1e-5 * float(mag) * 10


def test_constant_and_offset_rows():
    """A constant row has xhat = 0 exactly; a large offset leaves the variance's digits that fp32 x holds."""
    s = lib()
    x = torch.full((3, 500), 7.25, device="cuda")
    y, mean, rstd = s.layer_norm(x, stats=True)
    assert not y.any() and (mean == 7.25).all()
    torch.testing.assert_close(rstd, torch.full_like(rstd, EPS ** -0.5), rtol=1e-6, atol=0)
    base = (torch.arange(512, device="cuda") % 2).float() * 2 - 1  # exact at any offset below 2^23
    for off in (1024.0, 65536.0):
        y = s.layer_norm((base + off).repeat(4, 1), eps=0.0)
        torch.testing.assert_close(y, base.repeat(4, 1), rtol=1e-6, atol=0)
    y = s.layer_norm(torch.zeros(2, 64, device="cuda"), eps=0.0)  # 0 * inf
    assert torch.isnan(y).all()


def test_no_rows():
    s = lib()
    x = torch.empty(0, 48, device="cuda")
    y, mean, rstd = s.layer_norm(x, stats=True)
    assert y.shape == (0, 48) and mean.numel() == rstd.numel() == 0
    dx, dg, db = s.layer_norm_backward(x, x, mean, rstd)
    assert s.device_status() == 0
    assert dx.shape == (0, 48) and not dg.any() and not db.any()


def test_non_finite_rows_stay_alone():
    s, g = lib(), F.gen(8)
    for cols in (40, 1500):
        x, dy = F.matrix(g, 6, cols), F.matrix(g, 6, cols)
        x[1, 3], x[4, cols - 1] = float("inf"), float("nan")
        y, mean, rstd = s.layer_norm(x, stats=True)
        bad = ~torch.isfinite(y)
        assert bad[1].any() and bad[4].all() and not bad[[0, 2, 3, 5]].any()
        dx, _, _ = s.layer_norm_backward(dy, x, mean, rstd)
        bad = ~torch.isfinite(dx)
        assert bad[1].any() and bad[4].all() and not bad[[0, 2, 3, 5]].any()


def test_in_place():
    s, g = lib(), F.gen(12)
    for cols in (200, 3000, 40000):
        x = F.matrix(g, 5, cols, FP32)
        want, mean, rstd = s.layer_norm(x, stats=True)
        dy, dres = F.matrix(g, 5, cols, FP32), F.matrix(g, 5, cols, FP32)
        y = x.clone()
        s.layer_norm(y, out=y)
        assert torch.equal(y, want)


def test_rows_far_apart():
    s, g = lib(), F.gen(13)
    ld = (1 << 30) + 8
    far = torch.empty(3 * ld, dtype=BF16, device="cuda").view(3, ld)[:, :520]
    x = F.matrix(g, 3, 520)
    far.copy_(x)
    want = s.layer_norm(x, stats=True)
    got = s.layer_norm(far, stats=True)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    dy = F.matrix(g, 3, 520)
    a, b = (s.layer_norm_backward(dy, t, want[1], want[2]) for t in (x, far))
    assert s.device_status() == 0
    assert all(torch.equal(p, q) for p, q in zip(a, b))
