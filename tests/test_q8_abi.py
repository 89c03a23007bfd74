"""The entry points of the operators with 8-bit operands check their arguments on the
host alone: a bad one gives its status before anything is enqueued (the pointers
here are never dereferenced)."""
import ctypes

import pytest

from paper_1807_11091_gb300 import sadmm
from paper_1807_11091_gb300.sadmm import Q8, Q8Out

P = [(i + 1) << 32 for i in range(24)]  # never dereferenced
E4M3, BF16, FP32 = sadmm.SADMM_E4M3, sadmm.SADMM_BF16, sadmm.SADMM_FP32


def q8(i, ld, **kw):
    return Q8(**{**dict(q=P[i], ld=ld, s=P[i + 1], s_row=1, s_block=512, tile=0), **kw})


def out8(i, ld, **kw):
    return Q8Out(**{**dict(q=P[i], ld=ld, s=P[i + 1], s_row=1, s_block=512), **kw})


def rmsnorm_fwd(**kw):
    return sadmm.RmsNormFwdArgs(**{**dict(rows=4, cols=300, x=P[0], ldx=300, residual=P[1], ldr=300, h=P[2], ldh=300,
                                          gamma=P[3], eps=1e-5, ydt=E4M3, y8=out8(4, 300), rstd=P[6]), **kw})


def rmsnorm_bwd(**kw):
    return sadmm.RmsNormBwdArgs(**{**dict(rows=4, cols=300, h=P[0], ldh=300, dy=P[1], lddy=300, gamma=P[2], rstd=P[3],
                                          dres=P[4], lddres=300, dx=P[5], lddx=300, dgamma=P[6]), **kw})


def quantize(**kw):
    return sadmm.QuantizeArgs(**{**dict(rows=40, cols=300, x=P[0], ldx=300, out=out8(1, 300), out_t=out8(3, 40)), **kw})


def linear8_fwd(**kw):
    return sadmm.Linear8FwdArgs(**{**dict(tokens=4, n_in=300, n_out=32, x=q8(0, 304), w=q8(2, 304), bias=P[4], residual=P[5],
                                          ldr=32, act=1, y=P[6], ldy=32, z=P[7], ldz=32), **kw})


def linear8_bwd(**kw):
    return sadmm.Linear8BwdArgs(**{**dict(tokens=4, n_in=300, n_out=32, dy=P[0], lddy=32, xt=q8(1, 16), wt=q8(3, 32), z=P[5],
                                          ldz=32, act=1, dx=P[6], lddx=300, dw=P[7], lddw=300, db=P[8]), **kw})


def gated8_fwd(**kw):
    return sadmm.Gated8FwdArgs(**{**dict(tokens=4, n_in=300, n_hidden=200, x=q8(0, 304), wg=q8(2, 304), wu=q8(4, 304), bg=P[6],
                                         bu=P[7], act=3, hdt=E4M3, h8=out8(8, 200), g=P[10], ldg=200, u=P[11], ldu=200),
                                  **kw})


def gated8_bwd(**kw):
    return sadmm.Gated8BwdArgs(**{**dict(tokens=4, n_in=300, n_hidden=200, dh=P[0], lddh=200, xt=q8(1, 16), wgt=q8(3, 208),
                                         wut=q8(5, 208), g=P[7], ldg=200, u=P[8], ldu=200, act=3, dx=P[9], lddx=300,
                                         dwg=P[10], lddwg=300, dwu=P[11], lddwu=300, dbg=P[12], dbu=P[13]), **kw})


MAKERS = [rmsnorm_fwd, rmsnorm_bwd, quantize, linear8_fwd, linear8_bwd, gated8_fwd, gated8_bwd]


def call(make, a):
    f = getattr(sadmm, f"sadmm_{make.__name__}")
    return f(a, None) if make in (rmsnorm_fwd, quantize) else f(a, None, 0, None)


INVALID = [
    (rmsnorm_fwd, dict(rows=-1)), (rmsnorm_fwd, dict(cols=0)), (rmsnorm_fwd, dict(x=None)), (rmsnorm_fwd, dict(xdt=2)),
    (rmsnorm_fwd, dict(rdt=2)), (rmsnorm_fwd, dict(ydt=3)), (rmsnorm_fwd, dict(ldx=299)), (rmsnorm_fwd, dict(ldr=1)),
    (rmsnorm_fwd, dict(ldh=1)), (rmsnorm_fwd, dict(residual=None)), (rmsnorm_fwd, dict(eps=-1.0)),
    (rmsnorm_fwd, dict(eps=float("nan"))), (rmsnorm_fwd, dict(gamma=P[3] + 2)), (rmsnorm_fwd, dict(rstd=P[6] + 1)),
    (rmsnorm_fwd, dict(y8=out8(4, 299))), (rmsnorm_fwd, dict(y8=out8(4, 300, q=None))),
    (rmsnorm_fwd, dict(y8=out8(4, 300, s=None))), (rmsnorm_fwd, dict(y8=out8(4, 300, s=P[5] + 2))),
    (rmsnorm_fwd, dict(y8=out8(4, 300, s_row=0))), (rmsnorm_fwd, dict(y8=out8(4, 300, s_block=0))),
    (rmsnorm_fwd, dict(y8=out8(4, 300, s_block=3))), (rmsnorm_fwd, dict(y8=out8(4, 300, s_row=-1))),
    (rmsnorm_fwd, dict(y8=out8(4, 300, s_row=2, s_block=1))), (rmsnorm_fwd, dict(y8=out8(4, 300, s_block=1 << 38))),
    (rmsnorm_fwd, dict(ydt=BF16, y=None)), (rmsnorm_fwd, dict(ydt=BF16, y=P[9], ldy=299)),
    (rmsnorm_fwd, dict(h=P[1], ldh=301)), (rmsnorm_fwd, dict(h=P[0], rdt=FP32)), (rmsnorm_fwd, dict(x=P[0] + 1)),
    (rmsnorm_bwd, dict(rows=-1)), (rmsnorm_bwd, dict(cols=0)), (rmsnorm_bwd, dict(h=None)), (rmsnorm_bwd, dict(dy=None)),
    (rmsnorm_bwd, dict(rstd=None)), (rmsnorm_bwd, dict(hdt=2)), (rmsnorm_bwd, dict(dydt=-1)),
    (rmsnorm_bwd, dict(dx=None, dres=None, dgamma=None)), (rmsnorm_bwd, dict(dx=None)), (rmsnorm_bwd, dict(lddx=1)),
    (rmsnorm_bwd, dict(dx=P[4], lddx=304)),
    (quantize, dict(rows=-1)), (quantize, dict(cols=0)), (quantize, dict(x=None)), (quantize, dict(xdt=2)),
    (quantize, dict(ldx=299)), (quantize, dict(out=Q8Out(), out_t=Q8Out())), (quantize, dict(out=out8(1, 299))),
    (quantize, dict(out_t=out8(3, 39))), (quantize, dict(out_t=out8(3, 40, s_block=0, s_row=0))),
    (quantize, dict(out=out8(1, 300, s_block=39))),
    (linear8_fwd, dict(tokens=-1)), (linear8_fwd, dict(n_in=0)), (linear8_fwd, dict(n_out=0)),
    (linear8_fwd, dict(x=q8(0, 299))), (linear8_fwd, dict(w=q8(2, 299))), (linear8_fwd, dict(x=q8(0, 304, q=None))),
    (linear8_fwd, dict(w=q8(2, 304, s=None))), (linear8_fwd, dict(w=q8(2, 304, s=P[3] + 1))),
    (linear8_fwd, dict(x=q8(0, 304, s_row=-1))), (linear8_fwd, dict(x=q8(0, 304, s_block=1 << 38))),
    (linear8_fwd, dict(act=4)), (linear8_fwd, dict(ydt=2)), (linear8_fwd, dict(y=None)), (linear8_fwd, dict(ldy=31)),
    (linear8_fwd, dict(ldr=31)), (linear8_fwd, dict(ldz=31)), (linear8_fwd, dict(bias=P[4] + 2)),
    (linear8_fwd, dict(y=P[5], ldy=33)), (linear8_fwd, dict(x=q8(0, 1 << 38))),
    (linear8_bwd, dict(tokens=-1)), (linear8_bwd, dict(dx=None, dw=None, db=None)), (linear8_bwd, dict(dy=None)),
    (linear8_bwd, dict(xt=q8(1, 3))), (linear8_bwd, dict(wt=q8(3, 31))), (linear8_bwd, dict(z=None)),
    (linear8_bwd, dict(dxdt=2)), (linear8_bwd, dict(dwdt=2)), (linear8_bwd, dict(lddw=1)), (linear8_bwd, dict(db=P[8] + 2)),
    (linear8_bwd, dict(xt=Q8())), (linear8_bwd, dict(wt=Q8())),
    (gated8_fwd, dict(hdt=FP32)), (gated8_fwd, dict(hdt=BF16)), (gated8_fwd, dict(wg=q8(2, 1))), (gated8_fwd, dict(wu=Q8())),
    (gated8_fwd, dict(h8=out8(8, 199))), (gated8_fwd, dict(h8=out8(8, 200, s_block=3))), (gated8_fwd, dict(ldg=199)),
    (gated8_fwd, dict(bu=P[7] + 1)), (gated8_fwd, dict(act=-1)),
    (gated8_bwd, dict(dwg=None)), (gated8_bwd, dict(dh=None)), (gated8_bwd, dict(g=None)), (gated8_bwd, dict(ldu=1)),
    (gated8_bwd, dict(wgt=Q8())), (gated8_bwd, dict(xt=Q8())), (gated8_bwd, dict(lddx=299)),
    (gated8_bwd, dict(dx=None, dwg=None, dwu=None, dbg=None, dbu=None)),
]


@pytest.mark.parametrize("make,bad", INVALID, ids=lambda v: v.__name__ if callable(v) else "-".join(v))
def test_a_bad_argument_is_refused(make, bad):
    a = make(**bad)
    assert call(make, a) == sadmm.SADMM_EINVAL
    if make not in (rmsnorm_fwd, quantize):
        assert getattr(sadmm, f"sadmm_{make.__name__}_workspace_size")(a) == 0


@pytest.mark.parametrize("make", MAKERS, ids=lambda m: m.__name__)
def test_no_arguments_at_all(make):
    lib = sadmm.load()
    f = getattr(lib, f"sadmm_{make.__name__}")
    assert (f(None, None) if make in (rmsnorm_fwd, quantize) else f(None, None, 0, None)) == sadmm.SADMM_EINVAL


@pytest.mark.parametrize("make", MAKERS, ids=lambda m: m.__name__)
def test_more_than_the_kernels_hold(make):
    for field in ("rows", "tokens", "cols", "n_in"):
        a = make()
        if not hasattr(a, field):
            continue
        setattr(a, field, 0x7fffff01 if field in ("rows", "tokens") else (1 << 28) + 1)
        assert call(make, a) == sadmm.SADMM_EUNSUPPORTED


def pointers(a, prefix=""):
    """The paths of a struct's pointers."""
    for name, kind in a._fields_:
        if kind is ctypes.c_void_p:
            yield prefix + name
        elif kind in (Q8, Q8Out):
            yield from pointers(getattr(a, name), f"{prefix}{name}.")


def get(a, path):
    for p in path.split("."):
        a = getattr(a, p)
    return a


def put(a, path, v):
    *head, last = path.split(".")
    setattr(get(a, ".".join(head)) if head else a, last, v)


OUTPUTS = {rmsnorm_fwd: "h y8.q y8.s rstd", rmsnorm_bwd: "dx dgamma", quantize: "out.q out.s out_t.q out_t.s",
           linear8_fwd: "y z", linear8_bwd: "dx dw db", gated8_fwd: "h8.q h8.s g u", gated8_bwd: "dx dwg dwu dbg dbu"}
ALLOWED = {(rmsnorm_fwd, "h", "residual"), (rmsnorm_fwd, "h", "x"), (rmsnorm_bwd, "dx", "dres"),
           (linear8_fwd, "y", "residual")}
PAIRS = [(m, o, i) for m in MAKERS for o in OUTPUTS[m].split() for i in pointers(m())
         if o != i and (m, o, i) not in ALLOWED and get(m(), i)]


@pytest.mark.parametrize("make,out,other", PAIRS, ids=lambda v: v.__name__ if callable(v) else v)
def test_an_output_at_another_argument_is_refused(make, out, other):
    a = make()
    put(a, out, get(a, other))
    assert call(make, a) == sadmm.SADMM_EINVAL


def test_workspaces():
    """None where the operands lie on 16-byte boundaries, copies otherwise; too little or unaligned scratch is refused."""
    assert sadmm.sadmm_linear8_fwd_workspace_size(linear8_fwd()) == 0
    a = linear8_fwd(x=q8(0, 301))
    assert sadmm.sadmm_linear8_fwd_workspace_size(a) == (4 * 304 + 255) // 256 * 256
    assert sadmm.sadmm_linear8_fwd(a, None, 0, None) == sadmm.SADMM_EINVAL
    assert sadmm.sadmm_linear8_fwd(a, P[20] + 8, 1 << 20, None) == sadmm.SADMM_EINVAL
    assert sadmm.sadmm_linear8_fwd(a, P[20], 1000, None) == sadmm.SADMM_EINVAL
    for make in (linear8_bwd, gated8_bwd):
        a = make()
        n = getattr(sadmm, f"sadmm_{make.__name__}_workspace_size")(a)
        assert n > 0 and getattr(sadmm, f"sadmm_{make.__name__}")(a, P[20], n - 1, None) == sadmm.SADMM_EINVAL


def test_no_rows_need_nothing():
    """(No launch either: this runs without a GPU.)"""
    assert sadmm.sadmm_rmsnorm_fwd(rmsnorm_fwd(rows=0, x=None, residual=None, h=None, y8=Q8Out()), None) == 0
    assert sadmm.sadmm_quantize(quantize(rows=0, x=None), None) == 0
    assert sadmm.sadmm_linear8_fwd_workspace_size(linear8_fwd(tokens=0, x=q8(0, 301, q=None))) == 0
