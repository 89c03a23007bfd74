"""What the feed-forward functions refuse on tensors of the right device: types, shapes,
strides, outputs and options.  A refused call writes nothing and leaves the stream usable."""
import pytest
import torch

import _ffn as F
from _ffn import BF16, FP32

pytestmark = pytest.mark.gpu


def args_of(name):
    from paper_1807_11091_gb300 import sadmm as s
    g = F.gen(1)
    m = lambda r, c, dt=BF16: F.matrix(g, r, c, dt)  # noqa: E731
    vec = lambda n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    return getattr(s, name), {
        "layer_norm": lambda: dict(x=m(6, 64), gamma=vec(64), beta=vec(64), out=m(6, 64)),
        "layer_norm_backward": lambda: dict(dy=m(6, 64), x=m(6, 64), mean=vec(6), rstd=vec(6), gamma=vec(64), dres=m(6, 64)),
        "linear": lambda: dict(x=m(6, 64), W=m(32, 64), bias=vec(32), residual=m(6, 32), out=m(6, 32)),
        "linear_backward": lambda: dict(dy=m(6, 32), x=m(6, 64), W=m(32, 64), z=m(6, 32), act=s.SADMM_ACT_SILU),
        "gated": lambda: dict(x=m(6, 64), Wg=m(32, 64), Wu=m(32, 64), bg=vec(32), bu=vec(32), out=m(6, 32)),
        "gated_backward": lambda: dict(dh=m(6, 32), x=m(6, 64), Wg=m(32, 64), Wu=m(32, 64), g=m(6, 32), u=m(6, 32)),
    }[name]()


MATRICES = {"layer_norm": "x out", "layer_norm_backward": "dy x dres", "linear": "x W residual out",
            "linear_backward": "dy x W z", "gated": "x Wg Wu out", "gated_backward": "dh x Wg Wu g u"}
VECTORS = {"layer_norm": "gamma beta", "layer_norm_backward": "mean rstd gamma", "linear": "bias", "gated": "bg bu"}
PAIRS = [(f, a) for f, names in MATRICES.items() for a in names.split()]


def refused(name, error, **changed):
    from paper_1807_11091_gb300 import sadmm
    f, args = args_of(name)
    args.update(changed)
    out = args.get("out")
    before = F.guard(out) if out is not None else None
    with pytest.raises(error):
        f(**args)
    assert sadmm.device_status() == 0
    if before is not None:
        view = torch.int16 if out.element_size() == 2 else torch.int32 if out.element_size() == 4 else torch.int64
        assert torch.equal(F.guard(out).view(view), before.view(view))


@pytest.mark.parametrize("name,arg", PAIRS)
def test_types(name, arg):
    for dt in (torch.float16, torch.float64, torch.int32):
        t = args_of(name)[1][arg]
        refused(name, TypeError, **{arg: torch.zeros_like(t, dtype=dt)})


@pytest.mark.parametrize("name,arg", PAIRS)
def test_shapes(name, arg):
    t = args_of(name)[1][arg]
    r, c = t.shape
    if name not in ("linear", "gated") or arg not in ("x", "W", "Wg"):  # (there the rows are that argument's to choose)
        refused(name, (TypeError, ValueError), **{arg: torch.zeros(r + 1, c, dtype=t.dtype, device="cuda")})
    refused(name, (TypeError, ValueError), **{arg: torch.zeros(r, c + 8, dtype=t.dtype, device="cuda")})
    refused(name, (TypeError, ValueError), **{arg: torch.zeros((), dtype=t.dtype, device="cuda")})


@pytest.mark.parametrize("name,arg", PAIRS)
def test_strides(name, arg):
    t = args_of(name)[1][arg]
    r, c = t.shape
    across = torch.zeros(c, r, dtype=t.dtype, device="cuda").t()
    gaps = torch.zeros(r, 2 * c, dtype=t.dtype, device="cuda")[:, ::2]
    for bad in (across, gaps):
        assert bad.shape == t.shape
        refused(name, TypeError, **{arg: bad})
    one_row = torch.zeros(1, c, dtype=t.dtype, device="cuda").expand(r, c)  # rows that overlap
    refused(name, sadmm_error(), **{arg: one_row})


def sadmm_error():
    from paper_1807_11091_gb300 import sadmm
    return sadmm.SadmmError


def test_leading_dimensions_that_do_not_view_as_one():
    x = torch.zeros(4, 5, 64, dtype=BF16, device="cuda")[:, :3]
    refused("linear", TypeError, x=x, residual=None, out=None)


@pytest.mark.parametrize("name,arg", [(f, a) for f, names in VECTORS.items() for a in names.split()])
def test_vectors(name, arg):
    n = args_of(name)[1][arg].numel()
    for bad in (torch.zeros(n, dtype=BF16, device="cuda"), torch.zeros(n + 1, device="cuda"),
                torch.zeros(2 * n, device="cuda")[::2]):
        refused(name, TypeError, **{arg: bad})


def test_options():
    from paper_1807_11091_gb300 import sadmm as s
    err = s.SadmmError
    refused("layer_norm", err, eps=-1.0)
    refused("layer_norm", err, eps=float("nan"))
    refused("layer_norm", TypeError, eps="x")
    refused("layer_norm", TypeError, out=None, out_dtype=torch.float16)
    refused("layer_norm", TypeError, out=None, out_dtype="bf16")
    refused("layer_norm_backward", err, want_dx=False)  # dres has nowhere to go
    refused("layer_norm_backward", err, dres=None, want_dx=False, want_dgamma=False, want_dbeta=False)
    for act in (-1, 4, 5):
        refused("linear", err, act=act)
        refused("gated", err, act=act)
    refused("linear", TypeError, act="relu")
    refused("linear_backward", TypeError, z=None)
    refused("linear_backward", err, want_dx=False, want_dw=False, want_db=False)
    refused("linear_backward", TypeError, dw_dtype=torch.float16)
    refused("gated_backward", TypeError, dx_dtype=torch.float16)
    refused("gated_backward", err, want_dx=False, want_dw=False)


def test_outputs_in_an_arguments_place():
    from paper_1807_11091_gb300 import sadmm as s
    for name, args in (("linear", "x W"), ("gated", "x Wg Wu")):
        f, a = args_of(name)
        for arg in args.split():
            t = a[arg]
            wide = torch.as_strided(t, (6, 32), (t.stride(0), 1))  # out's shape at the argument's address
            with pytest.raises(s.SadmmError):
                f(**{**a, "out": wide})
    x = torch.randn(6, 64, device="cuda")
    with pytest.raises(s.SadmmError):  # in place, but as another type
        s.layer_norm(x, out=x.view(BF16)[:, :64])
    assert s.device_status() == 0
