"""The feed-forward entry points' checks of their arguments, on the host alone: a
bad argument gives its status before anything is enqueued (the pointers here
are never dereferenced)."""
import ctypes
import os
import re

import pytest

from paper_1807_11091_gb300 import sadmm

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = [(i + 1) << 32 for i in range(12)]  # never dereferenced
BIG = 1 << 50


def make(cls, **kw):
    return cls(**kw)


def ln_fwd(**kw):
    return make(sadmm.LayerNormFwdArgs, **{**dict(rows=4, cols=64, x=P[0], ldx=64, xdt=0, eps=1e-5, y=P[1], ldy=64,
                                                  ydt=0), **kw})


def ln_bwd(**kw):
    return make(sadmm.LayerNormBwdArgs, **{**dict(rows=4, cols=64, x=P[0], ldx=64, xdt=0, dy=P[1], lddy=64, dydt=0,
                                                  mean=P[2], rstd=P[3], dx=P[4], lddx=64, dgamma=P[5], dbeta=P[6]),
                                           **kw})


def linear_fwd(**kw):
    return make(sadmm.LinearFwdArgs, **{**dict(tokens=4, n_in=64, n_out=32, x=P[0], ldx=64, w=P[1], ldw=64, y=P[2],
                                               ldy=32, ydt=0), **kw})


def linear_bwd(**kw):
    return make(sadmm.LinearBwdArgs, **{**dict(tokens=4, n_in=64, n_out=32, dy=P[0], lddy=32, x=P[1], ldx=64, w=P[2],
                                               ldw=64, dx=P[3], lddx=64, dw=P[4], lddw=64, db=P[5]), **kw})


def gated_fwd(**kw):
    return make(sadmm.GatedFwdArgs, **{**dict(tokens=4, n_in=64, n_hidden=32, x=P[0], ldx=64, wg=P[1], ldwg=64,
                                              wu=P[2], ldwu=64, act=3, h=P[3], ldh=32), **kw})


def gated_bwd(**kw):
    return make(sadmm.GatedBwdArgs, **{**dict(tokens=4, n_in=64, n_hidden=32, dh=P[0], lddh=32, x=P[1], ldx=64,
                                              wg=P[2], ldwg=64, wu=P[3], ldwu=64, g=P[4], ldg=32, u=P[5], ldu=32,
                                              act=3, dx=P[6], lddx=64, dwg=P[7], lddwg=64, dwu=P[8], lddwu=64), **kw})


INVALID = [
    (ln_fwd, dict(rows=-1)), (ln_fwd, dict(cols=0)), (ln_fwd, dict(x=None)), (ln_fwd, dict(y=None)),
    (ln_fwd, dict(ldx=63)), (ln_fwd, dict(ldy=63)), (ln_fwd, dict(xdt=2)), (ln_fwd, dict(ydt=-1)),
    (ln_fwd, dict(eps=-1.0)), (ln_fwd, dict(eps=float("nan"))), (ln_fwd, dict(eps=float("inf"))),
    (ln_fwd, dict(x=P[0] + 1)), (ln_fwd, dict(xdt=1, x=P[0] + 2)), (ln_fwd, dict(gamma=P[2] + 2)),
    (ln_fwd, dict(mean=P[2] + 1)), (ln_fwd, dict(ldx=1 << 38)),
    (ln_bwd, dict(mean=None)), (ln_bwd, dict(rstd=None)), (ln_bwd, dict(dy=None)), (ln_bwd, dict(x=None)),
    (ln_bwd, dict(dx=None, dgamma=None, dbeta=None)), (ln_bwd, dict(dres=P[7], lddres=10)),
    (ln_bwd, dict(dres=P[7], lddres=64, dx=None)), (ln_bwd, dict(dx=P[0])), (ln_bwd, dict(dx=P[1])),
    (ln_bwd, dict(dydt=9)), (ln_bwd, dict(lddx=1)),
    (linear_fwd, dict(tokens=-1)), (linear_fwd, dict(n_in=0)), (linear_fwd, dict(n_out=0)),
    (linear_fwd, dict(x=None)), (linear_fwd, dict(w=None)), (linear_fwd, dict(y=None)), (linear_fwd, dict(act=4)),
    (linear_fwd, dict(act=-1)), (linear_fwd, dict(ydt=2)), (linear_fwd, dict(ldw=63)), (linear_fwd, dict(ldy=31)),
    (linear_fwd, dict(residual=P[3], ldr=31)), (linear_fwd, dict(z=P[3], ldz=31)), (linear_fwd, dict(y=P[0])),
    (linear_fwd, dict(y=P[1])), (linear_fwd, dict(z=P[2], ldz=32)), (linear_fwd, dict(bias=P[4] + 2)),
    (linear_fwd, dict(x=P[0] + 1)), (linear_fwd, dict(ydt=1, y=P[2] + 2)),
    (linear_bwd, dict(dx=None, dw=None, db=None)), (linear_bwd, dict(act=2)), (linear_bwd, dict(dy=None)),
    (linear_bwd, dict(w=None)), (linear_bwd, dict(x=None)), (linear_bwd, dict(dxdt=5)), (linear_bwd, dict(dwdt=5)),
    (linear_bwd, dict(dydt=5)), (linear_bwd, dict(dx=P[0])), (linear_bwd, dict(dw=P[2])), (linear_bwd, dict(dw=P[3])),
    (linear_bwd, dict(db=P[5] + 1)), (linear_bwd, dict(lddw=3)),
    (gated_fwd, dict(wg=None)), (gated_fwd, dict(wu=None)), (gated_fwd, dict(h=None)), (gated_fwd, dict(act=7)),
    (gated_fwd, dict(g=P[4], ldg=31)), (gated_fwd, dict(u=P[3], ldu=32)), (gated_fwd, dict(g=P[4], u=P[4], ldg=32, ldu=32)),
    (gated_fwd, dict(h=P[1])), (gated_fwd, dict(bu=P[5] + 1)), (gated_fwd, dict(ldwu=10)),
    (gated_bwd, dict(dwg=None)), (gated_bwd, dict(dwu=None)), (gated_bwd, dict(g=None)), (gated_bwd, dict(u=None)),
    (gated_bwd, dict(dh=None)), (gated_bwd, dict(dx=None, dwg=None, dwu=None)), (gated_bwd, dict(wg=None)),
    (gated_bwd, dict(x=None)), (gated_bwd, dict(dwu=P[7])), (gated_bwd, dict(dx=P[4])), (gated_bwd, dict(dbg=P[9] + 3)),
    (gated_bwd, dict(dwdt=3)), (gated_bwd, dict(ldu=1)),
]
CALLS = {ln_fwd: "layernorm_fwd", ln_bwd: "layernorm_bwd", linear_fwd: "linear_fwd", linear_bwd: "linear_bwd",
         gated_fwd: "gated_fwd", gated_bwd: "gated_bwd"}


def call(make_args, a, ws=P[11], nbytes=BIG):
    f = getattr(sadmm, "sadmm_" + CALLS[make_args])
    return f(a, None) if make_args is ln_fwd else f(a, ws, nbytes, None)


@pytest.mark.parametrize("make_args,bad", INVALID, ids=lambda v: CALLS.get(v, None) if callable(v) else str(v))
def test_bad_arguments_are_refused(make_args, bad):
    a = make_args(**bad)
    assert call(make_args, a) == sadmm.SADMM_EINVAL
    if make_args is not ln_fwd:
        assert getattr(sadmm, f"sadmm_{CALLS[make_args]}_workspace_size")(a) == 0


@pytest.mark.parametrize("make_args,wide", [(ln_fwd, dict(rows=1 << 31)), (linear_fwd, dict(tokens=1 << 31)),
                                            (gated_bwd, dict(tokens=1 << 31)), (linear_bwd, dict(n_in=1 << 29)),
                                            (gated_fwd, dict(n_hidden=1 << 29))])
def test_too_large_is_unsupported(make_args, wide):
    assert call(make_args, make_args(**wide)) == sadmm.SADMM_EUNSUPPORTED


@pytest.mark.parametrize("make_args", [linear_bwd, gated_bwd, ln_bwd])
def test_workspace_is_checked(make_args):
    a = make_args(act=1, z=P[6], ldz=32) if make_args is linear_bwd else make_args()
    need = getattr(sadmm, f"sadmm_{CALLS[make_args]}_workspace_size")(a)
    assert need > 0
    for ws, nbytes in ((None, need), (P[11], need - 1), (P[11] + 16, need)):
        assert call(make_args, a, ws, nbytes) == sadmm.SADMM_EINVAL


def test_workspace_sizes():
    """Aligned matrices are read where they lie; any other is copied, its rows to multiples of 8,
    except for a few tokens, which are read as they are."""
    size = sadmm.sadmm_linear_fwd_workspace_size
    assert size(linear_fwd(tokens=40)) == 0
    assert size(linear_fwd(tokens=40, ldx=68)) == 40 * 64 * 2
    assert size(linear_fwd(tokens=40, x=P[0] + 2)) == 40 * 64 * 2
    assert size(linear_fwd(tokens=40, n_in=61, ldx=61, ldw=61)) == 40 * 64 * 2 + 32 * 64 * 2
    assert size(linear_fwd(tokens=1, n_in=61, ldx=61, ldw=61)) == 0
    assert sadmm.sadmm_gated_fwd_workspace_size(gated_fwd(tokens=40, ldwu=65)) == 32 * 64 * 2
    assert sadmm.sadmm_gated_fwd_workspace_size(gated_fwd(tokens=1, ldwu=65)) == 0
    assert sadmm.sadmm_linear_bwd_workspace_size(linear_bwd()) == 0
    assert sadmm.sadmm_linear_bwd_workspace_size(linear_bwd(db=None, act=1, z=P[6], ldz=32)) == 4 * 32 * 2
    assert sadmm.sadmm_layernorm_bwd_workspace_size(ln_bwd(dgamma=None, dbeta=None)) == 0


def test_argument_structs_mirror_the_header():
    """Field names and kinds in order, from the header's text."""
    text = open(os.path.join(ROOT, "include", "sadmm.h")).read()
    text = re.sub(r"/\*.*?\*/", "", text, flags=re.S)
    kinds = {"long long": ctypes.c_longlong, "int": ctypes.c_int, "float": ctypes.c_float}
    for cls, name in ((sadmm.LayerNormFwdArgs, "layernorm_fwd"), (sadmm.LayerNormBwdArgs, "layernorm_bwd"),
                      (sadmm.LinearFwdArgs, "linear_fwd"), (sadmm.LinearBwdArgs, "linear_bwd"),
                      (sadmm.GatedFwdArgs, "gated_fwd"), (sadmm.GatedBwdArgs, "gated_bwd")):
        body = re.search(r"typedef struct \{([^{}]*)\} sadmm_%s_args;" % name, text).group(1)
        want = []
        for line in filter(None, (part.strip() for part in body.split(";"))):
            m = re.match(r"(const\s+)?(long long|int|float|void)\s*(\*?)\s*(.*)", line)
            for field in m.group(4).split(","):
                want.append((field.strip(), ctypes.c_void_p if m.group(3) else kinds[m.group(2)]))
        assert [tuple(f) for f in cls._fields_] == want
