"""Plain 64-bit forms of the feed-forward operators, with bounds on what fp32
sums and one rounding may differ by, for the tests of the kernels.

Bounds, all per element and derived from the formats alone:
  U32 = 2^-23   one fp32 operation, truncation allowed for
  U16 = 2^-8    one rounding to bf16 (8 significant bits, to nearest)
A product of K terms is added up 16 at a time, so its error is at most
(K / 16 + 32) U32 times the sum of the terms' magnitudes; the 32 covers the
additions inside 16 terms, of a cut contraction's parts and of the bias.
"""
import math

import torch

U32, U16 = 2.0 ** -23, 2.0 ** -8
ACTS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
BF16, FP32 = torch.bfloat16, torch.float32


def matrix(g, rows, cols, dtype=BF16, layout="dense", scale=1.0, offset=0.0):
    """[rows][cols] of normal numbers inside a buffer of NaN: dense rows, rows padded to 32
    bytes, rows padded by an odd count, or the columns from 1 on of dense rows."""
    lead, ld = 0, cols
    if layout == "padded":
        ld = (cols + 15) // 16 * 16 + 16
    elif layout == "odd":
        ld = cols + 3 - cols % 2
    elif layout == "offset":
        lead, ld = 1, cols + 1
    buf = torch.full((rows * ld + 8,), float("nan"), dtype=dtype, device="cuda")
    m = buf[:rows * ld].view(rows, ld)[:, lead:lead + cols]
    m.copy_((torch.randn(rows, cols, generator=g, device="cuda") * scale + offset).to(dtype))
    return m


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def act(name, z):
    """The activation in 64 bits, its slope, and a bound on how far a value moves per unit of z."""
    if name == "relu":
        return z.clamp_min(0), (z > 0).double()
    if name == "gelu":
        p = torch.special.erfc(-z / math.sqrt(2.0)) / 2
        return z * p, p + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        p = torch.sigmoid(z)
        return z * p, p + z * p * (1 - p)
    return z, torch.ones_like(z)


LIPSCHITZ = 1.13  # of every activation here (gelu: 1.129) and, with 0.8 to spare, of gelu's and silu's slopes
ACT_U = 16 * U32  # evaluation of an activation or slope, per unit of |z| + 1


def product(a, b):
    """a b^T in 64 bits and the bound on an fp32 one: a [m][k], b [n][k], both exact."""
    a, b = a.double(), b.double()
    mag = a.abs() @ b.abs().t()
    return a @ b.t(), (a.shape[1] / 16 + 32) * U32 * mag


def rounded(v, err, dtype):
    """The bound after one rounding of v to dtype (fp32: one operation); 2^-126 covers denormals."""
    return err + (v.abs() + err) * (U16 if dtype == BF16 else U32) + 2.0 ** -126


def linear(x, W, bias, residual, name):
    """y and z in 64 bits, and their bounds before the final rounding."""
    z, ez = product(x, W)
    if bias is not None:
        z = z + bias.double()
        ez = ez + U32 * z.abs()
    y = act(name, z)[0]
    ey = ez * LIPSCHITZ + (0 if name == "none" else ACT_U * (z.abs() + 1))
    if residual is not None:
        y = y + residual.double()
        ey = ey + U32 * y.abs()
    return y, ey, z, ez


def slope_grad(dy, name, z):
    """dz = dy act'(z) in 64 bits, its fp32 error bound."""
    d = dy.double()
    if name == "none":
        return d, torch.zeros_like(d)
    z = z.double()
    return d * act(name, z)[1], d.abs() * ACT_U * (z.abs() + 1)


def grad_product(dz, edz, other, exact_operand):
    """dz @ other^T-like products where dz (bound edz) is rounded to bf16 first unless it already is."""
    v, e = product(dz, other)
    r = edz + (0 if exact_operand else (dz.abs() + edz) * U16 + 2.0 ** -126)
    if torch.is_tensor(r):
        e = e + r @ other.double().abs().t() * (1 + 1e-3)
    return v, e


def column_sum(d, ed):
    """Column sums of d in fp32: any order of `rows` additions."""
    return d.sum(0), ed.sum(0) + d.abs().sum(0) * (d.shape[0] + 8) * U32


def check(got, want, bound, what):
    got = got.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - want).abs() - bound
    assert (over <= 0).all(), f"{what}: {float(over.max()):.3e} past the bound at {int(over.argmax())}"


def guard(t):
    """A copy of the whole storage that t is a view of."""
    return torch.as_strided(t, (t.untyped_storage().nbytes() // t.element_size(),), (1,), 0).clone()


def untouched(t, before):
    """Whether nothing outside t's rows and columns changed in its storage."""
    after = guard(t)
    for s in (after, before):
        torch.as_strided(s, t.shape, t.stride(), t.storage_offset()).zero_()
    return torch.equal(after.view(torch.int16 if t.element_size() == 2 else torch.int32),
                       before.view(torch.int16 if t.element_size() == 2 else torch.int32))
