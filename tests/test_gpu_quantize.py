"""The quantiser against its definition, bit for bit."""
import pytest
import torch

from _ffn import BF16, FP32, gen, guard, matrix
from _q8 import E4M3, quantized, values
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu


def same(q, want):
    assert q.dtype == E4M3 and q.shape == want.shape
    a, b = q.float(), want.float()
    assert torch.equal(torch.isnan(a), torch.isnan(b))
    assert torch.equal(torch.nan_to_num(a), torch.nan_to_num(b))


def run(x, tiles):
    q, s, qt, st = sadmm.quantize(x, tiles=tiles, transposed=True)
    for (a, b), m in (((q, s), x), ((qt, st), x.t())):
        want, scale = quantized(m, tiles)
        same(a, want)
        assert torch.equal(b, scale)
    alone = sadmm.quantize(x, tiles=tiles)
    assert torch.equal(alone[0].view(torch.uint8), q.view(torch.uint8)) and torch.equal(alone[1], s)
    turned = sadmm.quantize(x, tiles=tiles, transposed=True, want_q=False)
    assert torch.equal(turned[0].view(torch.uint8), qt.view(torch.uint8)) and torch.equal(turned[1], st)
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("layout", ["dense", "padded", "odd", "offset"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 127), (128, 128), (129, 130), (300, 513), (7, 1153), (1000, 8),
                                       (257, 256)])
def test_matrices(rows, cols, layout, dtype):
    g = gen(rows + cols)
    x = matrix(g, rows, cols, dtype, layout, 3.0)
    run(x, False)
    run(x, True)


def test_ends_of_the_range():
    """Zeros, the smallest and the largest numbers, and values on the borders between two of e4m3's."""
    x = torch.zeros(130, 384, device="cuda")
    x[1] = 1e-30
    x[2, 5], x[3, 7] = 2.0 ** -149, -3.4e38
    x[4] = torch.arange(384, device="cuda") * 0.125 - 20
    x[4, ::128] = 448.0  # scale 1: what stands between two values of e4m3 is there as it is
    x[5] = 2.0 ** -96 * torch.linspace(-1, 1, 384, device="cuda")
    x[6] = torch.linspace(-1, 1, 384, device="cuda") * 2.0 ** -100
    run(x, False)
    run(x, True)
    run(x.to(BF16), False)
    q, s = sadmm.quantize(x)
    assert float(s[0, 0]) == float(torch.tensor(2.0 ** -96) / torch.tensor(448.0)) and not q[0].float().any()
    assert float(q[3, 7]) == -448.0


def test_the_quotient_is_an_fp32_division():
    """4 million quotients of random digits, and those of 8-bit digits, which meet borders often."""
    g = gen(9)
    x = torch.randn(2048, 2048, generator=g, device="cuda")
    run(x, False)
    run((x * 1e-20).contiguous(), False)
    run(x.to(BF16), False)


def test_values_that_are_not_finite():
    """They become NaN; the rest of their block keeps the scale of its finite values."""
    g = gen(3)
    x = torch.randn(140, 300, generator=g, device="cuda")
    x[0, 0], x[5, 129], x[5, 130], x[139, 299] = float("inf"), float("nan"), float("-inf"), float("nan")
    x[7] = float("inf")
    for tiles in (False, True):
        run(x, tiles)
        q, s = sadmm.quantize(x, tiles=tiles)
        assert torch.isnan(q.float()).sum() == 304 and torch.isfinite(s).all()


def test_shapes_and_layouts_of_the_results():
    x = torch.randn(2, 3, 257, device="cuda")
    q, s, qt, st = sadmm.quantize(x, transposed=True)
    assert q.shape == (2, 3, 257) and s.shape == (2, 3, 3) and qt.shape == (257, 6) and st.shape == (257, 1)
    assert q.stride(-2) % 32 == 0 and qt.stride(0) % 32 == 0 and s.stride()[-2] == 1
    q, s, qt, st = sadmm.quantize(x, tiles=True, transposed=True)
    assert q.shape == (6, 257) and s.shape == (1, 3) and qt.shape == (257, 6) and st.shape == (3, 1)
    assert torch.equal(values(q, s), values(qt, st).t())
    empty = sadmm.quantize(x[:0], transposed=True)
    assert [t.shape for t in empty] == [(0, 3, 257), (0, 3, 3), (257, 0), (257, 0)]


def test_nothing_is_written_beside_the_matrix():
    """The bytes between rows (of the C call's outputs) stay as they were."""
    rows, cols = 131, 77
    g = gen(4)
    x = matrix(g, rows, cols, BF16, "odd")
    for ld, ldt in ((80, 136), (77, 131), (79, 133)):
        q = torch.full((rows, ld), 0x55, dtype=torch.uint8, device="cuda")
        qt = torch.full((cols, ldt), 0x55, dtype=torch.uint8, device="cuda")
        s, st = torch.full((rows, 3), 7.0, device="cuda"), torch.full((cols, 5), 7.0, device="cuda")
        a = sadmm.QuantizeArgs(rows, cols, x.data_ptr(), x.stride(0), sadmm.SADMM_BF16, 0,
                               sadmm.Q8Out(q.data_ptr(), ld, s.data_ptr(), 3, 1),
                               sadmm.Q8Out(qt.data_ptr(), ldt, st.data_ptr(), 5, 2))
        assert sadmm.sadmm_quantize(a, torch.cuda.current_stream().cuda_stream) == 0
        want, scale = quantized(x)
        same(q.view(E4M3)[:, :cols], want)
        assert torch.equal(s[:, :1], scale) and (s[:, 1:] == 7).all() and (q[:, cols:] == 0x55).all()
        want, scale = quantized(x.t())
        same(qt.view(E4M3)[:, :rows], want)
        assert torch.equal(st[:, 0:3:2], scale) and (st[:, [1, 3, 4]] == 7).all() and (qt[:, rows:] == 0x55).all()
