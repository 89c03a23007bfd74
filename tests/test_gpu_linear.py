"""sadmm_linear_fwd / _bwd and sadmm_gated_fwd / _bwd against 64-bit forms: every
orientation of the tiles, ragged sizes, row strides and alignments, types,
activations, empty batches, and gradients against differences."""
import pytest
import torch

import _ffn as F
from _ffn import BF16, FP32

pytestmark = pytest.mark.gpu


def lib():
    from paper_1807_11091_gb300 import sadmm
    return sadmm


def done():
    assert lib().device_status() == 0


# tokens, in, out, act, bias, residual, out dtype, save, layout
LINEAR = [
    (1, 64, 128, "none", False, False, BF16, False, "dense"),
    (1, 1, 1, "none", True, True, FP32, True, "dense"),
    (1, 2731, 515, "silu", True, True, BF16, True, "dense"),
    (2, 1000, 130, "relu", True, False, FP32, True, "odd"),
    (7, 520, 300, "gelu", False, True, FP32, False, "padded"),
    (16, 4096, 64, "none", True, False, BF16, False, "dense"),
    (17, 640, 1023, "silu", True, True, BF16, True, "offset"),
    (33, 72, 40, "none", False, False, FP32, False, "dense"),
    (64, 1536, 256, "gelu", True, False, BF16, True, "dense"),
    (65, 63, 129, "relu", True, True, FP32, True, "odd"),
    (127, 8, 2000, "none", True, True, BF16, False, "padded"),
    (130, 65, 127, "silu", False, True, BF16, True, "offset"),
    (257, 1024, 384, "gelu", True, True, FP32, True, "dense"),
    (300, 2048, 96, "none", False, True, FP32, False, "dense"),
    (1000, 333, 777, "none", True, False, BF16, False, "odd"),
    (513, 128, 1, "relu", True, True, BF16, True, "dense"),
    (1537, 512, 1200, "silu", True, False, BF16, True, "padded"),
    (2100, 320, 2600, "gelu", True, True, BF16, True, "dense"),
    (4500, 130, 2310, "none", True, True, FP32, True, "dense"),
]


@pytest.mark.parametrize("T,K,N,act,bias,res,dt,save,layout", LINEAR)
def test_linear(T, K, N, act, bias, res, dt, save, layout):
    s, g = lib(), F.gen(T * 7 + K)
    x, W = F.matrix(g, T, K, layout=layout), F.matrix(g, N, K, layout=layout, scale=K ** -0.5)
    b = torch.randn(N, generator=g, device="cuda") if bias else None
    r = F.matrix(g, T, N, dt, layout) if res else None
    out = F.matrix(g, T, N, dt, layout)
    before = F.guard(out)
    got = s.linear(x, W, b, residual=r, act=F.ACTS[act], save=save, out=out)
    done()
    y, z = got if save else (got, None)
    wy, ey, wz, ez = F.linear(x, W, b, r, act)
    F.check(y, wy, F.rounded(wy, ey, dt), "y")
    if save:
        F.check(z, wz, F.rounded(wz, ez, BF16), "z")
    assert F.untouched(out, before)
    again = s.linear(x, W, b, residual=r, act=F.ACTS[act], out_dtype=dt)
    assert torch.equal(again, y)


def test_linear_in_place_residual():
    s, g = lib(), F.gen(3)
    x, W, r = F.matrix(g, 40, 200), F.matrix(g, 90, 200, scale=0.07), F.matrix(g, 40, 90, FP32)
    want = s.linear(x, W, residual=r)
    s.linear(x, W, residual=r, out=r)
    done()
    assert torch.equal(want, r)


# tokens, in, out, act, dy dtype, dx dtype, dW dtype, layout
LINEAR_BWD = [
    (1, 64, 64, "none", BF16, BF16, BF16, "dense"),
    (1, 515, 2731, "silu", BF16, FP32, BF16, "dense"),
    (5, 300, 1, "relu", FP32, BF16, FP32, "odd"),
    (16, 1, 70, "gelu", BF16, BF16, BF16, "offset"),
    (64, 1000, 520, "none", BF16, FP32, FP32, "padded"),
    (65, 129, 130, "silu", FP32, BF16, BF16, "odd"),
    (200, 700, 333, "gelu", BF16, BF16, FP32, "dense"),
    (1025, 256, 385, "none", FP32, FP32, FP32, "offset"),
    (2100, 2600, 320, "relu", BF16, BF16, BF16, "dense"),
    (3000, 520, 1100, "none", BF16, BF16, FP32, "dense"),
]


@pytest.mark.parametrize("T,K,N,act,ydt,xdt,wdt,layout", LINEAR_BWD)
def test_linear_backward(T, K, N, act, ydt, xdt, wdt, layout):
    s, g = lib(), F.gen(T * 5 + K)
    dy, x = F.matrix(g, T, N, ydt, layout, 0.01), F.matrix(g, T, K, layout=layout)
    W, z = F.matrix(g, N, K, layout=layout, scale=K ** -0.5), F.matrix(g, T, N, layout=layout)
    args = dict(z=z, act=F.ACTS[act], dx_dtype=xdt, dw_dtype=wdt)
    dx, dw, db = s.linear_backward(dy, x, W, **args)
    done()
    dz, ez = F.slope_grad(dy, act, z)
    exact = act == "none" and ydt == BF16
    v, e = F.grad_product(dz, ez, W.t(), exact)
    F.check(dx, v, F.rounded(v, e, xdt), "dx")
    v, e = F.grad_product(dz.t(), ez.t(), x.t(), exact)
    F.check(dw, v, F.rounded(v, e, wdt), "dW")
    F.check(db, *F.column_sum(dz, ez), "db")
    assert dw.stride(0) == W.stride(0) or N == 1
    # each output alone gives the same bits
    for k, want in (("dx", dx), ("dw", dw), ("db", db)):
        only = s.linear_backward(dy, x, W, **args, **{f"want_{o}": o == k for o in ("dx", "dw", "db")})
        assert torch.equal([t for t in only if t is not None][0], want)


# tokens, in, hidden, act, bias, save, layout
GATED = [
    (1, 64, 64, "silu", False, False, "dense"),
    (1, 1, 1, "gelu", True, True, "dense"),
    (3, 2048, 555, "silu", True, True, "padded"),
    (8, 1000, 200, "relu", False, False, "dense"),
    (33, 257, 300, "none", True, True, "odd"),
    (64, 320, 65, "silu", False, True, "offset"),
    (65, 96, 640, "gelu", True, False, "padded"),
    (300, 777, 129, "silu", True, True, "dense"),
    (1030, 512, 700, "relu", False, True, "odd"),
    (2500, 192, 1300, "silu", True, True, "dense"),
    (2304, 640, 1411, "gelu", False, False, "padded"),
]


@pytest.mark.parametrize("T,K,H,act,bias,save,layout", GATED)
def test_gated(T, K, H, act, bias, save, layout):
    s, gn = lib(), F.gen(T * 3 + H)
    x = F.matrix(gn, T, K, layout=layout)
    Wg, Wu = (F.matrix(gn, H, K, layout=layout, scale=K ** -0.5) for _ in range(2))
    bg, bu = (torch.randn(H, generator=gn, device="cuda") if bias else None for _ in range(2))
    out = F.matrix(gn, T, H, layout=layout)
    before = F.guard(out)
    got = s.gated(x, Wg, Wu, bg, bu, act=F.ACTS[act], save=save, out=out)
    done()
    h = got[0] if save else got
    _, _, g, eg = F.linear(x, Wg, bg, None, "none")
    _, _, u, eu = F.linear(x, Wu, bu, None, "none")
    a = F.act(act, g)[0]
    ea = eg * F.LIPSCHITZ + F.ACT_U * (g.abs() + 1)
    F.check(h, a * u, F.rounded(a * u, ea * u.abs() + eu * a.abs() + ea * eu, BF16), "h")
    if save:
        F.check(got[1], g, F.rounded(g, eg, BF16), "g")
        F.check(got[2], u, F.rounded(u, eu, BF16), "u")
    assert F.untouched(out, before)
    assert torch.equal(s.gated(x, Wg, Wu, bg, bu, act=F.ACTS[act]), h)


GATED_BWD = [
    (1, 64, 128, "silu", BF16, BF16, "dense"),
    (1, 77, 501, "gelu", FP32, FP32, "odd"),
    (9, 400, 130, "relu", BF16, BF16, "offset"),
    (64, 130, 65, "none", FP32, BF16, "padded"),
    (130, 1, 70, "silu", BF16, FP32, "dense"),
    (515, 320, 333, "silu", BF16, BF16, "odd"),
    (2100, 260, 1290, "gelu", BF16, BF16, "padded"),
    (1100, 2304, 517, "silu", BF16, BF16, "dense"),
]


@pytest.mark.parametrize("T,K,H,act,xdt,wdt,layout", GATED_BWD)
def test_gated_backward(T, K, H, act, xdt, wdt, layout):
    s, gn = lib(), F.gen(T + 11 * H)
    x, dh = F.matrix(gn, T, K, layout=layout), F.matrix(gn, T, H, layout=layout, scale=0.02)
    Wg, Wu = (F.matrix(gn, H, K, layout=layout, scale=K ** -0.5) for _ in range(2))
    g, u = F.matrix(gn, T, H, layout=layout, scale=1.5), F.matrix(gn, T, H, layout=layout)
    args = dict(act=F.ACTS[act], dx_dtype=xdt, dw_dtype=wdt)
    dx, dwg, dwu, dbg, dbu = s.gated_backward(dh, x, Wg, Wu, g, u, want_db=True, **args)
    done()
    a, slope = F.act(act, g.double())
    ea = F.ACT_U * (g.double().abs() + 1)
    d, ud = dh.double(), u.double()
    dg, du = d * ud * slope, d * a
    eg, eu = d.abs() * (ud.abs() * ea + U_OPS * (ud * slope).abs()), d.abs() * (ea + U_OPS * a.abs())
    vg, e1 = F.grad_product(dg, eg, Wg.t(), False)
    vu, e2 = F.grad_product(du, eu, Wu.t(), False)
    # one contraction over both: its later additions act on the joint sum
    joint = (2 * H / 16 + 32) * F.U32 * (dg.abs() @ Wg.double().abs() + du.abs() @ Wu.double().abs())
    F.check(dx, vg + vu, F.rounded(vg + vu, e1 + e2 + joint, xdt), "dx")
    for what, got, dd, ee in (("dWg", dwg, dg, eg), ("dWu", dwu, du, eu)):
        v, e = F.grad_product(dd.t(), ee.t(), x.t(), False)
        F.check(got, v, F.rounded(v, e, wdt), what)
    F.check(dbg, *F.column_sum(dg, eg), "dbg")
    F.check(dbu, *F.column_sum(du, eu), "dbu")
    again = s.gated_backward(dh, x, Wg, Wu, g, u, **args)
    assert torch.equal(again[0], dx) and torch.equal(again[1], dwg) and torch.equal(again[2], dwu)
    assert again[3] is None and again[4] is None


U_OPS = 4 * F.U32  # a few fp32 products


def test_gated_gradients_against_differences():
    """<gradient, direction> against the 64-bit loss's central difference.  The gradient's own bound
    is that of test_gated_backward, here as roundings of every term: dg, du and the outputs to bf16
    (2 U16 of the terms' magnitudes), g and u to bf16 in the forward pass (their slopes and values
    move by at most 2 U16 of (1 + |g|) |u|); the difference itself is off by h^2 times a third
    derivative below 2 per unit, with h = 1e-4 far below the rest."""
    s, gn = lib(), F.gen(5)
    T, K, H = 24, 40, 56
    x, dh = F.matrix(gn, T, K), F.matrix(gn, T, H, scale=0.1)
    Wg, Wu = (F.matrix(gn, H, K, scale=K ** -0.5) for _ in range(2))
    _, g, u = s.gated(x, Wg, Wu, save=True)
    dx, dwg, dwu, _, _ = s.gated_backward(dh, x, Wg, Wu, g, u, dx_dtype=FP32, dw_dtype=FP32)
    done()

    def loss(x, Wg, Wu):
        return (dh.double() * F.act("silu", x @ Wg.t())[0] * (x @ Wu.t())).sum()

    at = [t.double() for t in (x, Wg, Wu)]
    gd, ud = at[0] @ at[1].t(), at[0] @ at[2].t()
    scale = dh.double().abs() * (1 + gd.abs()) * (1 + ud.abs())   # bounds every |dg|, |du| and their moves
    for k, grad in ((0, dx), (1, dwg), (2, dwu)):
        v = torch.randn(at[k].shape, generator=gn, device="cuda", dtype=torch.float64)
        hi, lo = list(at), list(at)
        hi[k], lo[k] = at[k] + 1e-4 * v, at[k] - 1e-4 * v
        diff = (loss(*hi) - loss(*lo)) / 2e-4
        if k == 0:
            mag = (scale @ at[1].abs() + scale @ at[2].abs()) * v.abs()
        else:
            mag = (scale.t() @ at[0].abs()) * v.abs()
        assert abs((grad.double() * v).sum() - diff) <= 6 * F.U16 * mag.sum()


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_linear_gradients_against_differences(act):
    """As above for the linear layer: z to bf16 in the forward pass moves the slope by at most
    U16 (1 + |z|) (a step of relu' where z crosses 0 cannot: rounding keeps the sign), dz to bf16."""
    s, gn = lib(), F.gen(6)
    T, K, N = 20, 48, 33
    x, W, dy = F.matrix(gn, T, K), F.matrix(gn, N, K, scale=K ** -0.5), F.matrix(gn, T, N)
    b = torch.randn(N, generator=gn, device="cuda")
    _, z = s.linear(x, W, b, act=F.ACTS[act], save=True)
    dx, dw, db = s.linear_backward(dy, x, W, z=z, act=F.ACTS[act], dx_dtype=FP32, dw_dtype=FP32)
    done()
    at = [x.double(), W.double(), b.double()]

    def loss(x, W, b):
        return (dy.double() * F.act(act, x @ W.t() + b)[0]).sum()

    zd = at[0] @ at[1].t() + at[2]
    h = 1e-6
    scale = dy.double().abs() * (1 + zd.abs())
    mags = (scale @ at[1].abs(), scale.t() @ at[0].abs(), scale.sum(0))
    for k, grad in enumerate((dx, dw, db)):
        v = torch.randn(at[k].shape, generator=gn, device="cuda", dtype=torch.float64)
        hi, lo = list(at), list(at)
        hi[k], lo[k] = at[k] + h * v, at[k] - h * v
        diff = (loss(*hi) - loss(*lo)) / (2 * h)
        assert abs((grad.double() * v).sum() - diff) <= 4 * F.U16 * (mags[k] * v.abs()).sum()


def test_no_tokens():
    s = lib()
    x, W = torch.empty(0, 40, dtype=BF16, device="cuda"), torch.ones(24, 40, dtype=BF16, device="cuda")
    dy = torch.empty(0, 24, dtype=BF16, device="cuda")
    assert s.linear(x, W).shape == (0, 24)
    assert s.gated(x, W, W).shape == (0, 24)
    dx, dw, db = s.linear_backward(dy, x, W, z=dy, act=s.SADMM_ACT_SILU, dw_dtype=FP32)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()
    dx, dwg, dwu, dbg, dbu = s.gated_backward(dy, x, W, W, dy, dy, want_db=True)
    done()
    assert dx.shape == (0, 40) and not (dwg.any() or dwu.any() or dbg.any() or dbu.any())


def test_non_finite_values_stay_in_their_rows():
    """An infinity or NaN of one token reaches that token's outputs and no other's, and one of a
    weight row that row's column alone; what lies beside the matrices (NaN) reaches nothing."""
    s, g = lib(), F.gen(9)
    for T in (3, 70, 700):
        x, W = F.matrix(g, T, 150, layout="padded"), F.matrix(g, 90, 150, layout="padded", scale=0.1)
        x[1, 77] = float("inf")
        x[2, 149] = float("nan")
        W[5, 3] = float("inf")
        for y in (s.linear(x, W), s.gated(x, W, W)):
            bad = ~torch.isfinite(y)
            assert bad[1].all() and bad[2].all() and bad[:, 5].all()
            bad[1] = bad[2] = False
            bad[:, 5] = False
            assert not bad.any()
    y = s.linear(x, W, act=s.SADMM_ACT_RELU)
    done()
    assert torch.isnan(y[2]).all()  # a NaN is not hidden by the ReLU


def test_rows_far_apart():
    """Offsets past 2^31 elements: three rows 2^30 + 8 apart."""
    s, g = lib(), F.gen(10)
    ld = (1 << 30) + 8
    far = [torch.empty(3 * ld, dtype=BF16, device="cuda").view(3, ld)[:, :n] for n in (72, 136)]
    x, W = F.matrix(g, 3, 72), F.matrix(g, 136, 72, scale=0.1)
    far[0].copy_(x)
    want = s.linear(x, W)
    s.linear(far[0], W, out=far[1])
    assert torch.equal(far[1], want)
    want = s.linear_backward(want, x, W)
    got = s.linear_backward(far[1], far[0], W)
    done()
    assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_leading_dimensions_and_streams():
    s, g = lib(), F.gen(11)
    x, W = F.matrix(g, 60, 128), F.matrix(g, 96, 128, scale=0.1)
    want = s.linear(x, W)
    y, z = s.linear(x.view(3, 4, 5, 128), W, save=True)
    assert y.shape == z.shape == (3, 4, 5, 96) and torch.equal(y.reshape(60, 96), want)
    assert torch.equal(s.linear(x[7], W), s.linear(x[7:8], W)[0])
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    odd = F.matrix(g, 300, 131)
    Wo = F.matrix(g, 96, 131, scale=0.1)
    ref = s.linear(odd, Wo)
    torch.cuda.synchronize()
    got = [s.linear(odd, Wo, stream=side) for _ in range(8)]  # each through a workspace of its own
    torch.cuda.current_stream().wait_stream(side)
    done()
    assert all(torch.equal(t, ref) for t in got)


def test_backward_passes_in_a_row():
    """More clusters than the device holds at once, each pass's kernels close behind the ones before,
    from an idle device: the products' clusters must not take the places of those that have not started."""
    s, g = lib(), F.gen(12)
    T, K, N = 1025, 1024, 2731
    dy, x = F.matrix(g, T, N, scale=0.01), F.matrix(g, T, K)
    W, z = F.matrix(g, N, K, scale=K ** -0.5), F.matrix(g, T, N)
    first = s.linear_backward(dy, x, W, z=z, act=s.SADMM_ACT_GELU)
    for i in range(600):
        got = s.linear_backward(dy, x, W, z=z, act=s.SADMM_ACT_GELU)
        if i % 8 == 0:
            torch.cuda.synchronize()
    done()
    assert all(torch.equal(a, b) for a, b in zip(got, first))
