"""What the feed-forward functions refuse before they look at any memory, on the host
alone: the tensors are torch's fake ones of two CUDA devices, which have none."""
import pytest
import torch
from torch._subclasses.fake_tensor import FakeTensorMode

BF16, FP32 = torch.bfloat16, torch.float32

pytestmark = pytest.mark.skipif(torch.cuda.is_available() and torch.cuda.device_count() < 2,
                                reason="a fake tensor of a second device needs two devices, or none")


def fake(*shape, dtype=BF16, device="cuda:0"):
    with FakeTensorMode():
        return torch.empty(*shape, dtype=dtype, device=device)


def calls():
    from paper_1807_11091_gb300 import sadmm as s
    t, vec = fake, lambda n: fake(n, dtype=FP32)
    return {
        "layer_norm": (s.layer_norm, dict(x=t(4, 64), gamma=vec(64), beta=vec(64), out=t(4, 64))),
        "layer_norm_backward": (s.layer_norm_backward, dict(dy=t(4, 64), x=t(4, 64), mean=vec(4), rstd=vec(4),
                                                            gamma=vec(64), dres=t(4, 64))),
        "linear": (s.linear, dict(x=t(4, 64), W=t(32, 64), bias=vec(32), residual=t(4, 32), out=t(4, 32))),
        "linear_backward": (s.linear_backward, dict(dy=t(4, 32), x=t(4, 64), W=t(32, 64), z=t(4, 32), act=1)),
        "gated": (s.gated, dict(x=t(4, 64), Wg=t(32, 64), Wu=t(32, 64), bg=vec(32), bu=vec(32), out=t(4, 32))),
        "gated_backward": (s.gated_backward, dict(dh=t(4, 32), x=t(4, 64), Wg=t(32, 64), Wu=t(32, 64), g=t(4, 32),
                                                  u=t(4, 32))),
    }


CASES = [(f, k) for f, ks in (("layer_norm", "gamma beta out"), ("layer_norm_backward", "dy mean rstd gamma dres"),
                              ("linear", "W bias residual out"), ("linear_backward", "dy W z"),
                              ("gated", "Wg Wu bg bu out"), ("gated_backward", "dh Wg Wu g u")) for k in ks.split()]


@pytest.mark.parametrize("name,arg", CASES)
def test_a_tensor_on_another_device_is_refused(name, arg):
    f, args = calls()[name]
    t = args[arg]
    with pytest.raises(ValueError, match=f"{arg} is on cuda:1, x on cuda:0"):
        f(**{**args, arg: fake(*t.shape, dtype=t.dtype, device="cuda:1")})


@pytest.mark.parametrize("name,arg", CASES + [(f, "x") for f in sorted({f for f, _ in CASES})])
def test_a_host_tensor_or_none_at_all_is_refused(name, arg):
    f, args = calls()[name]
    for wrong in (torch.empty(4, 64), "text"):
        with pytest.raises(TypeError, match=f"{arg} must be a"):
            f(**{**args, arg: wrong})
