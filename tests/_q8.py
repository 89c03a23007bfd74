"""Plain 64-bit forms of the operators with 8-bit operands, and bounds, for the tests
of their kernels.

An 8-bit block has s = max(largest finite |x|, 2^-96) / 448 and q = e4m3(x / s), both
quotients in fp32.  A rounding to e4m3 is off by at most half a step: 2^-4 of the value,
or 2^-10 below 2^-6 (times the scale s).  So a value v known to within e comes out
as q s with |q s - v| <= (|v| + e) 2^-4 + s 2^-10 + e.

A product of K terms is added up 16 at a time inside the tensor cores and 128 at a
time outside: (K / 16 + 32) U32 times the sum of the terms' magnitudes bounds it, with
the scales' product (one rounding a block) and the multiply-add of a block's sum
(one more a block) in place of 8 of a block's additions.
"""
import torch

from _ffn import ACT_U, LIPSCHITZ, U32, act, gen, matrix  # noqa: F401

BF16, FP32, E4M3 = torch.bfloat16, torch.float32, torch.float8_e4m3fn
FLOOR = 2.0 ** -96
HALF, LEAST = 2.0 ** -4, 2.0 ** -10


def in_blocks(x, high):
    r, c = x.shape
    x = torch.nn.functional.pad(x, (0, -c % 128, 0, -r % high))
    return x.view(x.shape[0] // high, high, -1, 128)


def spread(s, rows, cols):
    """Scales for each element; they are of single rows or of tiles of 128."""
    if s.shape[0] != rows:
        s = s.repeat_interleave(128, 0)[:rows]
    return s.repeat_interleave(128, 1)[:, :cols]


def quantized(x, tiles=False):
    """(q, s) by the definition, in fp32 as it says."""
    r, c = x.shape
    b = in_blocks(x.float(), 128 if tiles else 1)
    size = torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b)).amax((1, 3))
    s = size.clamp_min(FLOOR) / torch.full_like(size, 448.0)
    v = b / s[:, None, :, None]
    v = torch.where(torch.isinf(v), torch.full_like(v, float("nan")), v)
    return v.to(E4M3).view(-1, b.shape[2] * 128)[:r, :c], s


def values(q, s):
    """The matrix that q and s stand for, in 64 bits."""
    return q.double() * spread(s.double(), *q.shape)


def place(q, layout):
    """q in a buffer of NaN bytes: dense rows, rows padded to 32 bytes, rows padded by an odd count,
    or the columns from 1 on of wider rows."""
    rows, cols = q.shape
    lead, ld = 0, cols
    if layout == "padded":
        ld = (cols + 31) // 32 * 32 + 32
    elif layout == "odd":
        ld = cols + 3 - cols % 2
    elif layout == "offset":
        lead, ld = 1, cols + 1
    buf = torch.full((rows * ld + 32,), 0x7f, dtype=torch.uint8, device=q.device).view(E4M3)
    m = buf[:rows * ld].view(rows, ld)[:, lead:lead + cols]
    m.copy_(q)
    return m


def strided(s, how):
    """Scales of rows after one another, of blocks after one another, or apart."""
    if how == "rows":
        return s.contiguous()
    if how == "blocks":
        return s.t().contiguous().t()
    buf = torch.full((s.shape[0], 2, s.shape[1], 3), float("nan"), device=s.device)
    buf[:, 1, :, 2] = s
    return buf[:, 1, :, 2]


def operand(g, rows, cols, tiles=False, layout="padded", scales="blocks", scale=1.0):
    """A random 8-bit matrix: (q, s)."""
    x = torch.randn(rows, cols, generator=g, device="cuda") * scale
    x *= torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))  # rows of different sizes
    q, s = quantized(x, tiles)
    return place(q, layout), strided(s, scales)


def product(a, b):
    """a b^T in 64 bits and its bound, of two 8-bit matrices."""
    a, b = values(*a), values(*b)
    return a @ b.t(), (a.shape[1] / 16 + 32) * U32 * (a.abs() @ b.abs().t())


def check8(q, s, v, e, what):
    """q and s against values v known to within e."""
    v, e = v.double(), e.double()
    assert q.dtype == E4M3 and s.dtype == FP32
    sx = spread(s.double(), *q.shape)
    top = in_blocks(v.abs(), 1).amax((1, 3)).clamp_min(FLOOR) / 448
    es = in_blocks(e, 1).amax((1, 3)) / 448 + 2 * U32 * top
    over = (s.double() - top).abs() - es
    assert (over <= 0).all(), f"{what}: scales {float(over.max()):.3e} past the bound"
    got = q.double() * sx
    assert torch.isfinite(got).all(), f"{what}: not finite"
    over = (got - v).abs() - ((v.abs() + e) * HALF * (1 + 8 * U32) + sx * LEAST + e)
    assert (over <= 0).all(), f"{what}: {float(over.max()):.3e} past the bound"


def rounded8(d, e):
    """What making d (known to within e) 8-bit by rows may change it by."""
    s = spread(in_blocks(d.abs() + e, 1).amax((1, 3)).clamp_min(FLOOR) / 448, *d.shape)
    return (d.abs() + e) * HALF * (1 + 8 * U32) + s * LEAST + e
