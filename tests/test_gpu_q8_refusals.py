"""What the functions on 8-bit tensors refuse, and calls on other streams."""
import pytest
import torch

import _ffn as F
from _ffn import BF16, FP32
from _q8 import E4M3, operand

pytestmark = pytest.mark.gpu


def calls():
    from paper_1807_11091_gb300 import sadmm as s
    g = F.gen(1)
    m = lambda r, c, dt=BF16: F.matrix(g, r, c, dt)  # noqa: E731
    vec = lambda n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    x, W, U = operand(g, 6, 200), operand(g, 150, 200, True), operand(g, 150, 200, True)
    xt, Wt, Ut = operand(g, 200, 6), operand(g, 200, 150, True), operand(g, 200, 150, True)
    return {
        "rms_norm": (s.rms_norm, dict(x=m(6, 200), gamma=vec(200), residual=m(6, 200, FP32), out=m(6, 200), sum_out=m(6, 200, FP32))),
        "rms_norm_backward": (s.rms_norm_backward, dict(dy=m(6, 200), h=m(6, 200), rstd=vec(6), gamma=vec(200), dres=m(6, 200))),
        "quantize": (s.quantize, dict(x=m(6, 200))),
        "linear8": (s.linear8, dict(x=x[0], xs=x[1], W=W[0], Ws=W[1], bias=vec(150), residual=m(6, 150), out=m(6, 150))),
        "linear8_backward": (s.linear8_backward, dict(dy=m(6, 150), xt=xt[0], xts=xt[1], Wt=Wt[0], Wts=Wt[1], z=m(6, 150), act=1)),
        "gated8": (s.gated8, dict(x=x[0], xs=x[1], Wg=W[0], Wgs=W[1], Wu=U[0], Wus=U[1], bg=vec(150), bu=vec(150))),
        "gated8_backward": (s.gated8_backward, dict(dh=m(6, 150), xt=xt[0], xts=xt[1], Wgt=Wt[0], Wgts=Wt[1], Wut=Ut[0],
                                                    Wuts=Ut[1], g=m(6, 150), u=m(6, 150))),
    }


ARGS = [(f, a) for f, names in {
    "rms_norm": "x gamma residual out sum_out", "rms_norm_backward": "dy h rstd gamma dres", "quantize": "x",
    "linear8": "x xs W Ws bias residual out", "linear8_backward": "dy xt xts Wt Wts z",
    "gated8": "x xs Wg Wgs Wu Wus bg bu", "gated8_backward": "dh xt xts Wgt Wgts Wut Wuts g u"}.items() for a in names.split()]


def refused(name, error, **changed):
    from paper_1807_11091_gb300 import sadmm
    f, args = calls()[name]
    f(**args)
    args.update(changed)
    with pytest.raises(error):
        f(**args)
    assert sadmm.device_status() == 0


@pytest.mark.parametrize("name,arg", ARGS)
def test_wrong_tensors(name, arg):
    """Of another type, another size, on the host, or none."""
    t = calls()[name][1][arg]
    wrong = torch.float16 if t.dtype != E4M3 else torch.uint8
    refused(name, TypeError, **{arg: torch.zeros(t.shape, device="cuda", dtype=wrong)})
    refused(name, TypeError, **{arg: t.cpu()})
    refused(name, TypeError, **{arg: "text"})
    if (name, arg) in (("quantize", "x"),):
        return
    bigger = torch.zeros([n + 130 for n in t.shape], device="cuda", dtype=FP32).to(t.dtype)
    refused(name, (ValueError, TypeError), **{arg: bigger})


@pytest.mark.parametrize("name,arg", [(f, a) for f, a in ARGS if a not in ("xs", "Ws", "xts", "Wts", "Wgs", "Wus", "Wgts", "Wuts")])
def test_columns_that_are_no_neighbours(name, arg):
    t = calls()[name][1][arg]
    if t.dim() == 1:
        wrong = torch.zeros(2 * t.numel(), device="cuda")[::2]
    else:
        wrong = torch.zeros(t.shape[1], t.shape[0], device="cuda").to(t.dtype).t()
    refused(name, TypeError, **{arg: wrong})


def test_options():
    refused("quantize", ValueError, want_q=False)
    refused("gated8", TypeError, out_dtype=FP32)
    refused("linear8", TypeError, out=None, residual=None, out_dtype=E4M3)
    refused("rms_norm", ValueError, residual=None)           # sum_out of nothing
    refused("linear8_backward", TypeError, z=None)
    refused("linear8_backward", TypeError, Wt=None)
    from paper_1807_11091_gb300.sadmm import SadmmError
    refused("linear8", SadmmError, act=7)
    refused("rms_norm", SadmmError, eps=-1.0)
    refused("rms_norm_backward", SadmmError, want_dx=False)  # dres has no dx to go to
    refused("linear8_backward", SadmmError, want_dx=False, want_dw=False, want_db=False)


def test_outputs_in_an_inputs_place():
    from paper_1807_11091_gb300.sadmm import SadmmError
    x = torch.randn(6, 200, device="cuda")
    refused("rms_norm", SadmmError, x=x, residual=x, out=x, sum_out=x)
    refused("rms_norm", SadmmError, residual=x, out=x, sum_out=None)


@pytest.mark.parametrize("name", ["rms_norm", "rms_norm_backward", "quantize", "linear8", "linear8_backward", "gated8",
                                  "gated8_backward"])
def test_on_another_stream(name):
    """The bits of a call on the current stream, behind work that is still to come on the given one, with
    inputs and outputs whose memory is not handed out meanwhile."""
    f, args = calls()[name]
    args.pop("out", None), args.pop("sum_out", None)
    flat = lambda r: [t for t in (r if isinstance(r, tuple) else (r,)) if t is not None]  # noqa: E731
    want = [t.clone() for t in flat(f(**args))]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    f(**args, stream=side)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)
    got = flat(f(**args, stream=side))
    late = {k: v for k, v in args.items() if torch.is_tensor(v)}
    sizes = [v.untyped_storage().nbytes() for v in late.values()]
    args.clear(), late.clear()
    junk = [torch.full((n,), 0x7f, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(3)]
    side.synchronize()
    assert all(torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8)) for a, b in zip(got, want))
    del junk


def test_two_streams_at_once():
    """Calls that run at the same time, each with its own scratch."""
    from paper_1807_11091_gb300 import sadmm as s
    g = F.gen(2)
    x, W = operand(g, 300, 333, layout="offset"), operand(g, 500, 333, True, layout="offset")
    xt, Wt = operand(g, 333, 300), operand(g, 333, 500, True)
    dy = [F.matrix(g, 300, 500, BF16, "odd", 0.01) for _ in range(2)]
    want = [(s.linear8(*x, *W),) + s.linear8_backward(d, *xt, *Wt) for d in dy]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(5):
        got = []
        for st, d in zip(streams, dy):
            with torch.cuda.stream(st):
                got.append((s.linear8(*x, *W),) + s.linear8_backward(d, *xt, *Wt))
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert all(torch.equal(p, q) for p, q in zip(a, b))
    assert s.device_status() == 0
