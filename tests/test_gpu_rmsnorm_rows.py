"""RMS norm: 1/rms to the last digit, and more rows than the grid takes at once."""
import pytest
import torch

from _ffn import BF16, FP32, U32, check, gen, guard, matrix, rounded, untouched
from _q8 import E4M3, check8
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("cols", [1, 256, 4096, 16384, 65536])
def test_rstd_is_rounded_once(cols):
    """One number in a row of 4^k: its square, the average and the average's root are exact in fp32, so
    2^k / |x| rounded once is what a rounded root and quotient give."""
    x = torch.zeros(1000, cols, device="cuda")
    x[:, cols // 3] = torch.arange(3096, 4096, 1, device="cuda")[:1000] / 64.0
    _, rstd = sadmm.rms_norm(x, eps=0.0, out_dtype=FP32, stats=True)
    assert torch.equal(rstd, (cols ** 0.5 / x[:, cols // 3].double()).float())
    assert sadmm.device_status() == 0


def plain(x, residual, gamma):
    """h as it is kept, 1/rms and y in 64 bits."""
    h = x if residual is None else (x.float() + residual.float()).to(residual.dtype)
    rstd = (h.double().square().mean(1) + 1e-5) ** -0.5
    return h, rstd, h.double() * rstd[:, None] * gamma.double()


# more rows than CTAs and their warps take at once: 8 a CTA up to 512 columns, then one, of 64 to 1024 threads
MANY = [(6001, 130), (6001, 400), (2501, 513), (701, 8192), (1001, 8200), (401, 20001)]


@pytest.mark.parametrize("layout", ["dense", "padded"])
@pytest.mark.parametrize("rows,cols", MANY)
def test_more_rows_than_a_grid(rows, cols, layout):
    """Bounds as in test_gpu_rmsnorm.py: 44 U32 of 1/rms, 48 of y."""
    g = gen(rows + cols)
    gamma = torch.randn(cols, generator=g, device="cuda")
    for xt, rt, out in [(BF16, FP32, E4M3), (FP32, FP32, E4M3), (BF16, BF16, BF16), (FP32, None, FP32), (BF16, None, E4M3)]:
        x = matrix(g, rows, cols, xt, layout, 1.5, 0.25)
        r = None if rt is None else matrix(g, rows, cols, rt, layout, 2.0)
        h, rstd, y = plain(x, r, gamma)
        got = sadmm.rms_norm(x, gamma, r, 1e-5, out, True)
        check(got[-1], rstd, 44 * U32 * rstd, "rstd")
        if r is not None:
            assert torch.equal(got[-2], h)
        e = y.abs() * 48 * U32 + 2.0 ** -126
        if out == E4M3:
            check8(got[0], got[1], y, e, "y")
        else:
            check(got[0], y, rounded(y, e, out), "y")
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("layout", ["dense", "padded", "offset"])
@pytest.mark.parametrize("rows,cols", MANY)
def test_in_place_with_more_rows_than_a_grid(rows, cols, layout):
    """y in x's place, and the sum in the residual's or in x's, while the next rows are already on their way."""
    g = gen(rows * 3 + cols)
    gamma = torch.randn(cols, generator=g, device="cuda")
    x, r = matrix(g, rows, cols, BF16, layout), matrix(g, rows, cols, FP32, layout)
    h, rstd, y = plain(x, r, gamma)
    want = sadmm.rms_norm(x, gamma, r, 1e-5, E4M3)
    before = guard(r)
    q, s, got = sadmm.rms_norm(x, gamma, r, 1e-5, E4M3, sum_out=r)
    assert got.data_ptr() == r.data_ptr() and torch.equal(r, h) and untouched(r, before)
    assert torch.equal(q.float(), want[0].float()) and torch.equal(s, want[1])
    check8(q, s, y, y.abs() * 48 * U32 + 2.0 ** -126, "y")
    r = matrix(g, rows, cols, BF16, layout)
    h, rstd, y = plain(x, r, gamma)
    before, kept = guard(x), x.clone()
    got, total = sadmm.rms_norm(x, gamma, r, 1e-5, FP32, sum_out=x)
    assert total.data_ptr() == x.data_ptr() and torch.equal(x, h) and untouched(x, before)
    check(got, y, rounded(y, y.abs() * 48 * U32 + 2.0 ** -126, FP32), "y")
    x.copy_(kept)
    h, rstd, y = plain(x, None, gamma)
    assert sadmm.rms_norm(x, gamma, out=x).data_ptr() == x.data_ptr() and untouched(x, before)
    check(x, y, rounded(y, y.abs() * 48 * U32 + 2.0 ** -126, BF16), "y")
    assert sadmm.device_status() == 0
