"""The 8-bit linear product, forward and backward, against 64 bits."""
import pytest
import torch

from _ffn import ACT_U, ACTS, BF16, FP32, LIPSCHITZ, U32, act, check, column_sum, gen, guard, matrix, rounded, slope_grad, untouched
from _q8 import E4M3, operand, place, product, quantized, rounded8, strided, values
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu


def forward(g, tokens, n_in, n_out, name="none", bias=False, residual=False, out=BF16, layout="padded", scales="blocks",
            tiles=True, save=False):
    x = operand(g, tokens, n_in, False, layout, scales)
    W = operand(g, n_out, n_in, tiles, layout, "rows" if scales == "blocks" else scales, n_in ** -0.5)
    b = torch.randn(n_out, generator=g, device="cuda") if bias else None
    r = matrix(g, tokens, n_out, out, layout) if residual else None
    got = sadmm.linear8(*x, *W, b, residual=r, act=ACTS[name], out_dtype=out, save=save)
    z, ez = product(x, W)
    if bias:
        z = z + b.double()
        ez = ez + U32 * z.abs()
    if save:
        got, kept = got
        check(kept, z, rounded(z, ez, BF16), "z")
    y = act(name, z)[0]
    ey = ez * LIPSCHITZ + (0 if name == "none" else ACT_U * (z.abs() + 1))
    if residual:
        y = y + r.double()
        ey = ey + U32 * y.abs()
    check(got, y, rounded(y, ey, out), "y")
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("tokens", [1, 2, 7, 16, 17, 33, 64, 65, 129, 300])
@pytest.mark.parametrize("n_in,n_out", [(1, 1), (31, 16), (128, 128), (129, 127), (333, 257), (1153, 640)])
def test_sizes(tokens, n_in, n_out):
    g = gen(tokens * 7 + n_in)
    forward(g, tokens, n_in, n_out)
    forward(g, tokens, n_in, n_out, "gelu", True, True, FP32, "dense", "rows", False, True)


@pytest.mark.parametrize("layout", ["dense", "padded", "odd", "offset"])
@pytest.mark.parametrize("scales", ["rows", "blocks", "apart"])
@pytest.mark.parametrize("tiles", [False, True])
def test_layouts(layout, scales, tiles):
    for tokens, n_in, n_out in ((3, 200, 96), (48, 257, 131), (260, 1000, 300)):
        forward(gen(tokens), tokens, n_in, n_out, "silu", True, True, BF16, layout, scales, tiles)


@pytest.mark.parametrize("name", list(ACTS))
@pytest.mark.parametrize("out", [BF16, FP32])
def test_epilogues(name, out):
    for tokens in (5, 40, 200):
        forward(gen(tokens), tokens, 300, 200, name, True, True, out, save=True)
        forward(gen(tokens), tokens, 300, 200, name, False, False, out)


@pytest.mark.parametrize("tokens,n_in,n_out", [(512, 4096, 1024), (1000, 640, 5000), (4099, 384, 770), (2048, 2048, 2048),
                                               (130, 16384, 256)])
def test_large(tokens, n_in, n_out):
    forward(gen(tokens), tokens, n_in, n_out, "silu", True, False, BF16)
    forward(gen(tokens), tokens, n_in, n_out, "none", False, True, FP32, tiles=False, scales="rows")


def test_exact_sums():
    """Whole numbers small enough that every sum is exact: the result has to be theirs."""
    g = gen(11)
    for tokens, n_in, n_out in ((3, 300, 100), (70, 1000, 300), (600, 2000, 512)):
        x = torch.randint(-3, 4, (tokens, n_in), generator=g, device="cuda").float()
        W = torch.randint(-3, 4, (n_out, n_in), generator=g, device="cuda").float()
        xs = torch.exp2(torch.randint(-3, 4, (tokens, (n_in + 127) // 128), generator=g, device="cuda").float())
        Ws = torch.exp2(torch.randint(-3, 4, ((n_out + 127) // 128, (n_in + 127) // 128), generator=g, device="cuda").float())
        xq, Wq = place(x.to(E4M3), "padded"), place(W.to(E4M3), "padded")
        y = sadmm.linear8(xq, xs, Wq, Ws, out_dtype=FP32)
        want = values(xq, xs) @ values(Wq, Ws).t()
        assert torch.equal(y.double(), want)


def test_nan_and_infinity_stay_in_their_rows_and_columns():
    g = gen(12)
    for tokens in (4, 50, 300):
        x, W = operand(g, tokens, 300), operand(g, 200, 300, True)
        clean = sadmm.linear8(*x, *W, out_dtype=FP32)
        x[0][2, 130] = float("nan")
        W[0][77, 3] = float("nan")
        y = sadmm.linear8(*x, *W, out_dtype=FP32)
        bad = torch.zeros_like(y, dtype=torch.bool)
        bad[2], bad[:, 77] = True, True
        assert torch.equal(torch.isnan(y), bad) and torch.equal(y[~bad], clean[~bad])


def test_residual_in_place_and_nothing_beside():
    g = gen(13)
    for tokens in (6, 90, 400):
        x, W = operand(g, tokens, 384, layout="offset"), operand(g, 131, 384, True)
        r = matrix(g, tokens, 131, FP32, "odd")
        want = sadmm.linear8(*x, *W, residual=r)
        before = guard(r)
        got = sadmm.linear8(*x, *W, residual=r, out=r)
        assert got.data_ptr() == r.data_ptr() and torch.equal(got, want) and untouched(r, before)


@pytest.mark.parametrize("tokens,n_in,n_out", [(5, 300, 200), (300, 300, 200), (1100, 640, 1500)])
def test_tiles_for_tokens_and_rows_for_weights(tokens, n_in, n_out):
    """Either operand's scales may be of rows or of tiles, forward and backward."""
    g = gen(tokens)
    for xt, wt in ((True, True), (True, False), (False, False)):
        x, W = operand(g, tokens, n_in, xt), operand(g, n_out, n_in, wt, scale=n_in ** -0.5)
        z, ez = product(x, W)
        check(sadmm.linear8(*x, *W, out_dtype=FP32), z, rounded(z, ez, FP32), "y")
        xT, WT = operand(g, n_in, tokens, xt), operand(g, n_in, n_out, wt)
        dy = matrix(g, tokens, n_out, BF16, "padded", 0.01)
        dx, dW, _ = sadmm.linear8_backward(dy, *xT, *WT, dx_dtype=FP32, dw_dtype=FP32)
        for got, d, other in ((dx, dy.double(), WT), (dW, dy.double().t(), xT)):
            v, e = product(quantized(d.float()), other)
            check(got, v, rounded(v, e, FP32), "gradient")
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("tokens", [3, 100, 600])
def test_one_scale_for_a_whole_matrix(tokens):
    """Scales of stride zero."""
    g = gen(tokens)
    x, W = operand(g, tokens, 512), operand(g, 768, 512, True)
    one = torch.full((1, 1), 0.25, device="cuda")
    xs, Ws = one.expand(tokens, 4), one.expand(6, 4)
    z, ez = product((x[0], xs), (W[0], Ws))
    y = sadmm.linear8(x[0], xs, W[0], Ws, out_dtype=FP32)
    check(y, z, rounded(z, ez, FP32), "y")


@pytest.mark.parametrize("tokens,n_out", [(700, 1000), (2300, 520), (513, 4097), (600, 4092), (1111, 2050)])
def test_large_outputs_leave_the_rest_of_their_buffers(tokens, n_out):
    """Whose rows start on 16-byte boundaries (written by the tensor-memory accelerator), with room behind each."""
    g = gen(tokens)
    x, W, Wr = operand(g, tokens, 384), operand(g, n_out, 384, True), operand(g, n_out, 384, False)
    for out in (BF16, FP32):
        for w in (W, Wr):
            y, r = matrix(g, tokens, n_out, out, "padded"), matrix(g, tokens, n_out, out, "padded")
            before = guard(y)
            got, z = sadmm.linear8(*x, *w, residual=r, out=y, save=True)
            assert got.data_ptr() == y.data_ptr() and untouched(y, before)
            v, e = product(x, w)
            check(z, v, rounded(v, e, BF16), "z")
            v, e = v + r.double(), e + U32 * (v + r.double()).abs()
            check(y, v, rounded(v, e, out), "y")


@pytest.mark.parametrize("tokens,n_out", [(19622, 256), (19712, 250), (256, 19622), (250, 19712)])
def test_a_few_tiles_more_than_rounds(tokens, n_out):
    """Tiles of 256 x 256 on 76 pairs of CTAs: the last ones may be computed apart."""
    forward(gen(tokens), tokens, 4096, n_out, "gelu", True, True, BF16, save=True)
    forward(gen(tokens), tokens, 4096, n_out, "none", True, True, FP32, "odd", "rows", True)
    forward(gen(tokens), tokens, 4096, n_out, "silu", True, False, FP32, scales="apart", tiles=False)


@pytest.mark.parametrize("n_out,n_in,tokens", [(512, 9856, 2048), (500, 9850, 2050), (39000, 120, 2100), (2048, 5120, 4096)])
def test_weight_gradients_of_a_few_tiles_more_than_rounds(n_out, n_in, tokens):
    """Tiles of 512 x 128."""
    g = gen(n_out)
    dy = matrix(g, tokens, n_out, BF16, "padded", 0.01)
    xT = operand(g, n_in, tokens, False)
    _, dW, _ = sadmm.linear8_backward(dy, *xT, None, None, want_dx=False, dw_dtype=FP32)
    v, e = product(quantized(dy.double().t().float()), xT)
    check(dW, v, rounded(v, e, FP32), "dW")
    assert sadmm.device_status() == 0


def test_what_is_kept_does_not_change_the_result():
    g = gen(21)
    for tokens in (4, 60, 900):
        x, W = operand(g, tokens, 700), operand(g, 900, 700, True)
        y, _ = sadmm.linear8(*x, *W, act=3, save=True)
        assert torch.equal(y, sadmm.linear8(*x, *W, act=3))
        q = sadmm.gated8(*x, *W, *W)
        k = sadmm.gated8(*x, *W, *W, save=True)
        assert torch.equal(q[0].view(torch.uint8), k[0].view(torch.uint8)) and torch.equal(q[1], k[1])


def test_same_bits_and_leading_dimensions():
    g = gen(14)
    x, W = operand(g, 6, 256), operand(g, 64, 256, True)
    y = sadmm.linear8(*x, *W)
    x3 = x[0].view(2, 3, 256), x[1].reshape(2, 3, 2)
    assert torch.equal(sadmm.linear8(*x3, *W), y.view(2, 3, 64)) and torch.equal(sadmm.linear8(*x, *W), y)


def test_no_tokens():
    g = gen(15)
    W = operand(g, 64, 256, True)
    x = torch.empty(0, 256, dtype=E4M3, device="cuda"), torch.empty(0, 2, device="cuda")
    assert sadmm.linear8(*x, *W).shape == (0, 64)
    xt = torch.empty(256, 0, dtype=E4M3, device="cuda"), torch.empty(256, 0, device="cuda")
    Wt = W[0].t().contiguous(), W[1].t()
    dx, dW, db = sadmm.linear8_backward(torch.empty(0, 64, device="cuda"), *xt, *Wt)
    assert dx.shape == (0, 256) and dW.shape == (64, 256) and not dW.any() and not db.any()


def backward(g, tokens, n_in, n_out, name="none", dy_dtype=BF16, dx_dtype=None, dw_dtype=None, layout="padded"):
    xt = operand(g, n_in, tokens, False, layout)
    Wt = operand(g, n_in, n_out, True, layout)
    dy = matrix(g, tokens, n_out, dy_dtype, layout, 0.01)
    z = matrix(g, tokens, n_out, BF16, layout) if name != "none" else None
    dx, dW, db = sadmm.linear8_backward(dy, *xt, *Wt, z=z, act=ACTS[name], dx_dtype=dx_dtype, dw_dtype=dw_dtype)
    dz, edz = slope_grad(dy, name, z)
    v, e = column_sum(dz, edz)
    check(db, v, e, "db")
    for got, d, ed, other, what in ((dx, dz, edz, Wt, "dx"), (dW, dz.t(), edz.t(), xt, "dW")):
        if name in ("none", "relu"):  # dz is exact, and with it its 8-bit form
            v, e = product(quantized(d.float()), other)
        else:
            o = values(*other)
            v = d @ o.t()
            e = (d.shape[1] / 16 + 32) * U32 * (d.abs() @ o.abs().t()) * 1.1 + rounded8(d, ed) @ o.abs().t()
        check(got, v, rounded(v, e, got.dtype), what)
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("tokens,n_in,n_out", [(1, 1, 1), (2, 40, 129), (128, 128, 128), (131, 257, 96), (300, 1000, 333),
                                               (1000, 130, 2000)])
@pytest.mark.parametrize("name", ["none", "relu", "gelu"])
def test_backward(tokens, n_in, n_out, name):
    backward(gen(tokens + n_in), tokens, n_in, n_out, name)
    backward(gen(tokens), tokens, n_in, n_out, name, FP32, FP32, FP32, "dense")
    backward(gen(tokens), tokens, n_in, n_out, name, BF16, FP32, BF16, "odd")


def test_backward_of_a_batch():
    backward(gen(1), 2048, 1024, 1280, "none", BF16, None, FP32)
    backward(gen(2), 1500, 2048, 1031, "relu")


def test_backward_parts_alone():
    """Each gradient alone has the same bits, and needs none of the others' operands."""
    g = gen(16)
    xt, Wt = operand(g, 200, 77), operand(g, 200, 130, True)
    dy = matrix(g, 77, 130)
    dx, dW, db = sadmm.linear8_backward(dy, *xt, *Wt)
    assert torch.equal(sadmm.linear8_backward(dy, None, None, *Wt, want_dw=False, want_db=False)[0], dx)
    assert torch.equal(sadmm.linear8_backward(dy, *xt, None, None, want_dx=False, want_db=False)[1], dW)
    assert torch.equal(sadmm.linear8_backward(dy, None, None, None, None, want_dx=False, want_dw=False)[2], db)


def test_gradient_is_the_differences():
    """sum(c * y) of operands and gradients that 8 bits hold exactly is linear in x and W: its differences are the gradients."""
    g = gen(17)
    tokens, n_in, n_out = 37, 150, 140

    def whole(r, c):
        return torch.randint(-4, 5, (r, c), generator=g, device="cuda").double()

    def ones(r, c):
        return torch.ones(r, (c + 127) // 128, device="cuda")

    x, W, c = whole(tokens, n_in), whole(n_out, n_in), whole(tokens, n_out)
    c[:, ::64], c[::32] = 7, 7  # (each block's largest: q = 64 c, s = 7 / 448)
    dx, dW, db = sadmm.linear8_backward(c.float(), place(x.t().to(E4M3), "padded"), ones(n_in, tokens),
                                        place(W.t().to(E4M3), "padded"), ones(n_in, n_out), dx_dtype=FP32, dw_dtype=FP32)

    def loss(x, W):
        return (c * (x @ W.t())).sum()

    for i, j in ((0, 0), (36, 149), (5, 131)):
        e = torch.zeros_like(x)
        e[i, j] = 1
        assert float(dx[i, j]) == float((loss(x + e, W) - loss(x - e, W)) / 2)
    for i, j in ((0, 0), (139, 149), (70, 131)):
        e = torch.zeros_like(W)
        e[i, j] = 1
        assert float(dW[i, j]) == float((loss(x, W + e) - loss(x, W - e)) / 2)
    assert torch.equal(db.double(), c.sum(0))
