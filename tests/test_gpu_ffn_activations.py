"""The activations and slopes value by value, far into the tails where they are small:
every bf16 number of magnitude 2^-20 to 12.5 as a pre-activation."""
import pytest
import torch

import _ffn as F
from _ffn import BF16, FP32, U32

pytestmark = pytest.mark.gpu

ACTS = ("relu", "gelu", "silu")


def values():
    z = torch.arange(0, 1 << 15, dtype=torch.int32).to(torch.int16).view(BF16)
    z = z[(z.float() >= 2.0 ** -20) & (z.float() <= 12.5)]
    return torch.cat((z, -z, torch.zeros(1, dtype=BF16))).cuda()


def nearest(want):
    return (want.to(BF16).double() - want).abs() + want.abs() * 2.0 ** -13 + 2.0 ** -126


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("T", [1, 8, 40, 200])
@pytest.mark.parametrize("dt", [BF16, FP32])
def test_activation(name, T, dt):
    """Each kernel that serves these token counts: x [T][1] of ones, W [N][1] the values.  fp32: eight
    operations' error (CUDA's functions err by at most five units).  bf16: no further off than the
    nearest bf16 number is, but for 2^-13 of the value, 1/32 of a rounding, for the function."""
    from paper_1807_11091_gb300 import sadmm
    z = values()
    x = torch.zeros(T, 8, dtype=BF16, device="cuda")[:, :1]
    x.fill_(1)
    W = torch.zeros(z.numel(), 8, dtype=BF16, device="cuda")[:, :1]
    W.copy_(z[:, None])
    y = sadmm.linear(x, W, act=F.ACTS[name], out_dtype=dt)
    assert sadmm.device_status() == 0
    want = F.act(name, z.double())[0].expand(T, -1)
    bound = 8 * U32 * want.abs() + 2.0 ** -126 if dt == FP32 else nearest(want)
    over = (y.double() - want).abs() - bound
    at = int(over.argmax())
    assert (over <= 0).all(), (float(z[at % z.numel()]), float(y.flatten()[at]), float(want.flatten()[at]))


@pytest.mark.parametrize("name", ACTS)
@pytest.mark.parametrize("T", [1, 40, 600])
def test_activation_of_fp32_values(name, T):
    """Pre-activations with all of fp32's digits: x is zero, the bias the values.  As above for fp32; the
    functions' arguments enter products that the tail enlarges, and must not lose digits there."""
    from paper_1807_11091_gb300 import sadmm
    z = torch.rand(20000, generator=F.gen(3), device="cuda") * 25 - 12.5
    x, W = torch.zeros(T, 8, dtype=BF16, device="cuda"), torch.zeros(z.numel(), 8, dtype=BF16, device="cuda")
    y = sadmm.linear(x, W, z, act=F.ACTS[name], out_dtype=FP32)
    assert sadmm.device_status() == 0
    want = F.act(name, z.double())[0].expand(T, -1)
    over = (y.double() - want).abs() - (8 * U32 * want.abs() + 2.0 ** -126)
    assert (over <= 0).all(), float(z[int(over.argmax()) % z.numel()])


@pytest.mark.parametrize("name", ACTS)
def test_slope(name):
    """db of one token is dy act'(z) before any rounding to bf16: within 2^-16 of the slope's terms
    (1/128 of the rounding that dz takes)."""
    from paper_1807_11091_gb300 import sadmm
    z = values()[None]
    one = torch.ones_like(z)
    x, W = torch.ones(1, 8, dtype=BF16, device="cuda"), torch.ones(z.numel(), 8, dtype=BF16, device="cuda")
    db = sadmm.linear_backward(one, x, W, z=z, act=F.ACTS[name], want_dx=False, want_dw=False)[2]
    assert sadmm.device_status() == 0
    zd = z[0].double()
    a, s = F.act(name, zd)
    terms = s.abs() + (a / zd.where(zd != 0, torch.ones_like(zd))).abs()  # sigmoid or Phi, and what is added to it
    over = (db.double() - s).abs() - (2.0 ** -16 * terms + 2.0 ** -126)
    assert (over <= 0).all(), float(zd[int(over.argmax())])


def test_gated_value():
    """du of the pair is dh act(g), rounded once: as the activation in bf16."""
    from paper_1807_11091_gb300 import sadmm
    z = values()[None]
    one = torch.ones_like(z)
    W = torch.ones(z.numel(), 8, dtype=BF16, device="cuda")
    x = torch.ones(1, 8, dtype=BF16, device="cuda")
    for name in ACTS:
        got = sadmm.gated_backward(one, x, W, W, z, one, act=F.ACTS[name], want_dx=False, dw_dtype=FP32)[2]
        want = F.act(name, z.double())[0][0]
        assert sadmm.device_status() == 0
        over = (got[:, 0].double() - want).abs() - nearest(want)
        assert (over <= 0).all(), (name, float(z[0][int(over.argmax())]))
