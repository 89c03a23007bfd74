"""The slopes of activations that become fp32 sums, at fp32's precision over the whole range of z.

With one token a bias's gradient is dy act'(z) itself.  Its terms are Phi(z) and z phi(z), or p and z p (1 - p):
an exponential (2 units), a quotient (2; of 1 + exp, one more), GELU's polynomial (4.4e-7, 4 units) and 5 roundings of
half a unit, no more than 12 U32 of the terms' magnitudes; and 1 - p, known to within 2 U32 of 1, which z p multiplies.
2^-120 covers what is below fp32's normal numbers (times z)."""
import math

import pytest
import torch

from _ffn import ACTS, BF16, U32, act, gen
from _q8 import operand
from paper_1807_11091_gb300 import sadmm

pytestmark = pytest.mark.gpu


def terms(name, z):
    """The magnitudes of the slope's terms."""
    if name == "gelu":
        return torch.special.erfc(-z / math.sqrt(2.0)) / 2 + z.abs() * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    p = torch.sigmoid(z)
    return p + (z * p).abs() * (1 - p) + (z * p).abs() / 6


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_bias_gradient_of_one_token(name):
    z = torch.linspace(-14, 14, 9000, device="cuda").to(BF16).unique()[None]
    one = torch.ones_like(z)
    _, _, db = sadmm.linear8_backward(one, None, None, None, None, z=z, act=ACTS[name], want_dx=False, want_dw=False)
    want = act(name, z.double())[1][0]
    bound = 12 * U32 * terms(name, z.double())[0] + 2.0 ** -120
    over = (db.double() - want).abs() / bound
    assert float(over.max()) <= 1, float(over.max())


@pytest.mark.parametrize("name", ["gelu", "silu"])
def test_gated_bias_gradients_of_one_token(name):
    """dg = dh u act'(g) and du = dh act(g), with dh = u = 1: act(g) = g Phi(g) or g p, whose terms are its own size."""
    g = torch.linspace(-14, 14, 9000, device="cuda").to(BF16).unique()[None]
    one, x = torch.ones_like(g), operand(gen(1), 3, 1)
    got = sadmm.gated8_backward(one, *x, None, None, None, None, g, one, act=ACTS[name], want_dx=False, want_db=True)
    a, slope = act(name, g.double())
    assert float(((got[3].double() - slope[0]).abs() / (12 * U32 * terms(name, g.double())[0] + 2.0 ** -120)).max()) <= 1
    assert float(((got[4].double() - a[0]).abs() / (12 * U32 * a[0].abs() + 2.0 ** -120)).max()) <= 1
