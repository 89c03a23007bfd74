"""The operators of a feed-forward block with 8-bit operands, as timed cases.

A pruned feed-forward block is a smaller dense block, and its products are what
a language model is served and retrained with.  Held in 8 bits (e4m3) with an
fp32 scale for each block of 128 values, weights and activations take half the
bytes of bf16 and twice its rate.  Such a block calls four operators and their
backward passes: the root-mean-square norm with the residual's addition
(``sadmm.rms_norm``), whose output may be 8-bit; the quantiser
(``sadmm.quantize``); the closing projection (``sadmm.linear8``); and the gated
pair of projections (``sadmm.gated8``), whose output is the next product's 8-bit
operand.  Each case is one such call.

A block's scale is s = max(largest finite |x|, 2^-96) / 448, and its values are
q = e4m3(x / s), the fp32 quotient rounded to nearest even; infinities and NaN
become NaN.  A block is 128 neighbouring columns of one row, or for ``tiles`` of
128 rows.  Products are the sums over blocks of both scales times the block's
sum of products of e4m3 values.

A case's ``op`` is one of
  rms_fwd      x (and the residual) -> y or its 8-bit form and scales, the sum, 1/rms where kept
  rms_bwd      dy, h, 1/rms (and the residual's gradient) -> dx, dgamma
  quantize     x -> q, s, and for ``both`` those of the transpose
  linear8_fwd  act(x W^T + bias) + residual -> y
  linear8_bwd  dy, x^T, W^T, z -> dx, dW, db; dy act'(z) becomes 8-bit by rows and by columns
  gated8_fwd   act(x Wg^T + bg) * (x Wu^T + bu) -> h (8-bit and scales, or bf16), both pre-activations where kept
  gated8_bwd   dh, x^T, Wg^T, Wu^T, g, u -> dx, dWg, dWu, dbg, dbu

``pad`` says that matrices lie in buffers whose rows start on 64-byte
boundaries, as a program that may choose its buffers has them; without it they
are dense, so that an odd width gives rows of every alignment.
"""
import math

import torch

own = False  # whether run() calls the framework's operators, or computes their plain forms

EPS = 1e-5
BLOCK = 128
LARGEST = 448.0  # of e4m3
FLOOR = 2.0 ** -96
E4M3 = torch.float8_e4m3fn
DT = {"bf16": torch.bfloat16, "fp32": torch.float32, "e4m3": E4M3}
SIZE = {"bf16": 2, "fp32": 4, "e4m3": 1}


# ------------------------------------------------------------------ cases --

def _rms(name, op, rows, cols, x, y, residual="none", stats=False, pad=True):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "x": x, "y": y, "residual": residual, "stats": stats,
            "pad": pad}


def _quantize(name, rows, cols, x, tiles, both, pad=True):
    return {"name": name, "op": "quantize", "rows": rows, "cols": cols, "x": x, "tiles": tiles, "both": both, "pad": pad}


def _linear(name, op, tokens, n_in, n_out, act, bias, residual, out, pad=True):
    return {"name": name, "op": op, "tokens": tokens, "in": n_in, "out": n_out, "act": act, "bias": bias,
            "residual": residual, "type": out, "pad": pad}


def _gated(name, op, tokens, n_in, hidden, act, bias, save, out="e4m3", pad=True):
    return {"name": name, "op": op, "tokens": tokens, "in": n_in, "hidden": hidden, "act": act, "bias": bias,
            "save": save, "type": out, "pad": pad}


def listed():
    return [
        # the newest token of four sequences on its way into an 8-bit product, where the call's own latency counts
        _rms("rms_fwd_4_tokens", "rms_fwd", 4, 4096, "bf16", "e4m3", "bf16"),
        # a training batch: a block's output added to the fp32 residual stream and normed into the next product's operand
        _rms("rms_fwd_batch", "rms_fwd", 16384, 4096, "bf16", "e4m3", "fp32", stats=True),
        # the same norm's backward pass, with the gradient that came along the residual
        _rms("rms_bwd_batch", "rms_bwd", 8192, 5120, "bf16", "bf16", "bf16"),
        # after an optimiser's step: a weight's tiles, for the forward product and transposed for the backward one
        _quantize("quantize_weight", 10240, 4096, "bf16", True, True),
        # activations of a ragged batch of odd width, by rows and by columns
        _quantize("quantize_ragged", 3001, 1153, "fp32", False, True, pad=False),
        # serving one sequence: the closing projection of one token, bound by the weights
        _linear("linear8_1_token", "linear8_fwd", 1, 5120, 4096, "none", False, True, "bf16"),
        # a prompt of odd length through a third of the hidden units, dense rows, fp32 residual stream
        _linear("linear8_ragged", "linear8_fwd", 777, 2731, 1025, "none", True, True, "fp32", pad=False),
        # training: a square projection with bias and activation on a whole batch
        _linear("linear8_batch", "linear8_fwd", 8192, 4096, 4096, "gelu", True, False, "bf16"),
        # retraining: the closing projection's gradients, the weights' in fp32
        _linear("linear8_bwd_batch", "linear8_bwd", 8192, 5120, 2048, "none", True, False, "fp32"),
        # serving sixteen sequences: the gated pair on their newest tokens, an odd number of units kept
        _gated("gated8_16_tokens", "gated8_fwd", 16, 4096, 5461, "silu", False, False),
        # training: the gated pair of a wide block on a whole batch, the most work here
        _gated("gated8_batch", "gated8_fwd", 8192, 4096, 10240, "silu", False, True),
        # retraining: its backward pass with an odd number of units kept
        _gated("gated8_bwd_batch", "gated8_bwd", 4096, 2048, 5461, "silu", True, False, "bf16"),
    ]


def _size(rng, lo, hi):
    """A size spread over the logarithm of lo..hi: odd or of a warp's or tile's multiple."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    step = rng.choice([1, 1, 1, 8, 128])
    return max(lo, min(hi, int(round(v / step)) * step if v >= step else int(round(v))))


def draw(rng):
    op = rng.choice(["rms_fwd", "rms_bwd", "quantize", "linear8_fwd", "linear8_fwd", "linear8_bwd", "gated8_fwd",
                     "gated8_fwd", "gated8_bwd"])
    pad = rng.random() < 0.7
    while True:
        if op.startswith("rms"):
            x = rng.choice(["bf16", "fp32"])
            residual = rng.choice(["none", "bf16", "fp32"]) if op == "rms_fwd" else rng.choice(["none", x])
            y = rng.choice(["bf16", "fp32", "e4m3", "e4m3"]) if op == "rms_fwd" else rng.choice(["bf16", "fp32"])
            c = _rms("", op, _size(rng, 1, 32768), _size(rng, 32, 8192), x, y, residual, rng.random() < 0.5, pad)
        elif op == "quantize":
            c = _quantize("", _size(rng, 1, 16384), _size(rng, 32, 8192), rng.choice(["bf16", "fp32"]),
                          rng.random() < 0.5, rng.random() < 0.5, pad)
        elif op.startswith("linear8"):
            c = _linear("", op, _size(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 64, 8192),
                        rng.choice(["none", "none", "relu", "gelu", "silu"]), rng.random() < 0.5, rng.random() < 0.5,
                        rng.choice(["bf16", "bf16", "fp32"]), pad)
            if op == "linear8_bwd" and c["act"] != "none":
                c["type"] = "bf16"
        else:
            c = _gated("", op, _size(rng, 1, 8192), _size(rng, 64, 4096), _size(rng, 64, 10240),
                       rng.choice(["relu", "gelu", "silu", "silu"]), rng.random() < 0.5, rng.random() < 0.5,
                       rng.choice(["e4m3", "e4m3", "bf16"]) if op == "gated8_fwd" else "bf16", pad)
        w = work(c)
        if w["flops"] <= 1.3e12 and w["bytes"] <= 4e8:
            del c["name"]
            return c


def _blocks(n):
    return -(-n // BLOCK)


def work(case):
    """The bytes that one pass has to read and write and the operations that it has to do."""
    c, op = case, case["op"]
    if op.startswith("rms"):
        n, m, x, y = c["rows"] * c["cols"], c["cols"], SIZE[c["x"]], SIZE[c["y"]]
        stats = 4 * c["rows"]
        if op == "rms_fwd":
            r = 2 * SIZE[c["residual"]] if c["residual"] != "none" else 0
            scales = 4 * c["rows"] * _blocks(m) * (c["y"] == "e4m3")
            return {"bytes": n * (x + y + r) + 4 * m + scales + stats * c["stats"], "flops": 6 * n}
        return {"bytes": n * (2 * x + y + x * (c["residual"] != "none")) + 8 * m + stats, "flops": 11 * n}
    if op == "quantize":
        r, m = c["rows"], c["cols"]
        if c["tiles"]:
            scales = _blocks(r) * _blocks(m) * (1 + c["both"])
        else:
            scales = r * _blocks(m) + m * _blocks(r) * c["both"]
        return {"bytes": r * m * (SIZE[c["x"]] + 1 + c["both"]) + 4 * scales, "flops": 3 * r * m}
    t, k = c["tokens"], c["in"]
    kb, tb = _blocks(k), _blocks(t)
    if op.startswith("linear8"):
        n, s = c["out"], SIZE[c["type"]]
        nb = _blocks(n)
        if op == "linear8_fwd":
            return {"bytes": t * k + n * k + 4 * (t * kb + nb * kb) + t * n * s * (1 + c["residual"]) + 4 * n * c["bias"],
                    "flops": 2 * t * k * n}
        z = c["act"] != "none"
        return {"bytes": t * k + n * k + 4 * (k * tb + kb * nb) + 2 * (t * k + t * n * (1 + z)) + s * n * k +
                4 * n * c["bias"], "flops": 4 * t * k * n}
    n = c["hidden"]
    nb = _blocks(n)
    if op == "gated8_fwd":
        h = t * n + 4 * t * nb if c["type"] == "e4m3" else 2 * t * n
        return {"bytes": t * k + 2 * n * k + 4 * (t * kb + 2 * nb * kb) + h + 4 * t * n * c["save"] + 8 * n * c["bias"],
                "flops": 4 * t * k * n}
    return {"bytes": t * k + 2 * n * k + 4 * (k * tb + 2 * kb * nb) + 2 * (t * k + 2 * n * k + 3 * t * n) +
            8 * n * c["bias"], "flops": 8 * t * k * n}


# ----------------------------------------------------------------- inputs --

def _rows(v, dtype, pad):
    """The matrix v in `dtype`, in a buffer of its own rows or of rows on 64-byte boundaries."""
    step = 64 // SIZE[next(k for k in DT if DT[k] == dtype)] if pad else 1
    rows, cols = v.shape
    buf = torch.zeros(rows, -(-cols // step) * step, dtype=dtype, device="cuda")
    buf[:, :cols].copy_(v)
    return buf[:, :cols]


def _matrix(g, rows, cols, dtype, pad, scale=1.0, offset=0.0):
    """[rows][cols] of N(offset, scale^2)."""
    return _rows(torch.empty(rows, cols, device="cuda").normal_(generator=g).mul_(scale).add_(offset), dtype, pad)


def _vector(g, n, scale=0.1, offset=0.0):
    return torch.empty(n, device="cuda").normal_(generator=g).mul_(scale).add_(offset)


def _in_blocks(x, tiles):
    """x padded with zeros to whole blocks, as [row blocks][rows of a block][column blocks][128]."""
    r, c = x.shape
    high = BLOCK if tiles else 1
    x = torch.nn.functional.pad(x, (0, -c % BLOCK, 0, -r % high))
    return x.view(x.shape[0] // high, high, -1, BLOCK)


def _quantized(x, tiles):
    """(q, s) of a matrix: e4m3 values, and the blocks' scales as fp32."""
    r, c = x.shape
    b = _in_blocks(x.float(), tiles)
    size = torch.where(torch.isfinite(b), b.abs(), torch.zeros_like(b)).amax((1, 3))
    s = size.clamp_min(FLOOR) / torch.full_like(size, LARGEST)  # (a division by a number is a product with its inverse)
    v = b / s[:, None, :, None]
    v = torch.where(torch.isinf(v), torch.full_like(v, math.nan), v)
    return v.to(E4M3).view(-1, b.shape[2] * BLOCK)[:r, :c], s


def _scales(s):
    """Scales as the quantiser leaves them: those of one column block are neighbours."""
    buf = torch.zeros(s.shape[1], -(-s.shape[0] // 4) * 4, device="cuda")
    buf[:, :s.shape[0]].copy_(s.t())
    return buf[:, :s.shape[0]].t()


def _operand(x, tiles, pad):
    """The 8-bit operand of a matrix that a user's program holds: (q, s)."""
    q, s = _quantized(x, tiles)
    return _rows(q, E4M3, pad), _scales(s)


def _outliers(x):
    """A residual stream's: one channel in 64 some 8 times as large as the others."""
    x[:, 7::64] *= 8
    return x


def prepare(case, seed):
    c, op = case, case["op"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if op.startswith("rms"):
        rows, cols, x, y = c["rows"], c["cols"], DT[c["x"]], DT[c["y"]]
        s["gamma"] = _vector(g, cols, 0.1, 1.0)
        if op == "rms_fwd":
            s["x"] = _outliers(_matrix(g, rows, cols, x, c["pad"], 0.7))
            s["residual"] = _outliers(_matrix(g, rows, cols, DT[c["residual"]], c["pad"], 1.5, 0.25)) \
                if c["residual"] != "none" else None
            return s
        s["h"] = _outliers(_matrix(g, rows, cols, x, c["pad"], 1.5, 0.25))
        s["rstd"] = (s["h"].float().square().mean(1) + EPS).rsqrt()
        s["dy"] = _matrix(g, rows, cols, y, c["pad"], 1e-2)
        s["dres"] = _matrix(g, rows, cols, x, c["pad"], 1e-2) if c["residual"] != "none" else None
        return s
    if op == "quantize":
        s["x"] = _outliers(_matrix(g, c["rows"], c["cols"], DT[c["x"]], c["pad"], 0.02 if c["tiles"] else 1.0))
        return s
    t, k, pad = c["tokens"], c["in"], c["pad"]
    x = _outliers(torch.empty(t, k, device="cuda").normal_(generator=g))
    if op.startswith("linear8"):
        n = c["out"]
        W = torch.empty(n, k, device="cuda").normal_(generator=g).mul_(k ** -0.5)
        if op == "linear8_fwd":
            s["x"], s["W"] = _operand(x, False, pad), _operand(W, True, pad)
            s["bias"] = _vector(g, n) if c["bias"] else None
            s["residual"] = _matrix(g, t, n, DT[c["type"]], pad) if c["residual"] else None
            return s
        # what the forward pass kept for this one: both operands' transposes
        s["xt"], s["Wt"] = _operand(x.t().contiguous(), False, pad), _operand(W.t().contiguous(), True, pad)
        s["dy"] = _matrix(g, t, n, torch.bfloat16, pad, 1e-2)
        s["z"] = _matrix(g, t, n, torch.bfloat16, pad) if c["act"] != "none" else None
        return s
    n = c["hidden"]
    Wg = torch.empty(n, k, device="cuda").normal_(generator=g).mul_(1.5 * k ** -0.5)
    Wu = torch.empty(n, k, device="cuda").normal_(generator=g).mul_(k ** -0.5)
    if op == "gated8_fwd":
        s["x"], s["Wg"], s["Wu"] = _operand(x, False, pad), _operand(Wg, True, pad), _operand(Wu, True, pad)
        s["bg"] = _vector(g, n) if c["bias"] else None
        s["bu"] = _vector(g, n) if c["bias"] else None
        return s
    s["xt"] = _operand(x.t().contiguous(), False, pad)
    s["Wgt"], s["Wut"] = _operand(Wg.t().contiguous(), True, pad), _operand(Wu.t().contiguous(), True, pad)
    # pre-activations as the forward pass leaves them
    s["g"] = _matrix(g, t, n, torch.bfloat16, pad, 1.5)
    s["u"] = _matrix(g, t, n, torch.bfloat16, pad)
    s["dh"] = _matrix(g, t, n, torch.bfloat16, pad, 1e-2)
    return s


# ------------------------------------------------------------ plain forms --

def _act(name, z):
    if name == "relu":
        return torch.where(z < 0, torch.zeros_like(z), z)
    if name == "gelu":
        return 0.5 * z * (1 + torch.erf(z * 0.5 ** 0.5))
    if name == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _dact(name, z):
    if name == "relu":
        return (z > 0).to(z.dtype)
    if name == "gelu":
        return 0.5 * (1 + torch.erf(z * 0.5 ** 0.5)) + z * torch.exp(-0.5 * z * z) * (2 * math.pi) ** -0.5
    if name == "silu":
        s = 1 / (1 + torch.exp(-z))
        return s * (1 + z * (1 - s))
    return torch.ones_like(z)


def _values(q, s, tiles):
    """The fp32 matrix that an 8-bit operand stands for."""
    r, c = q.shape
    return (_in_blocks(q.float(), tiles) * s[:, None, :, None]).view(-1, s.shape[1] * BLOCK)[:r, :c]


def _rounded(x, tiles=False):
    """x as its 8-bit form stands for it."""
    return _values(*_quantized(x, tiles), tiles)


def _one(out):
    """A single output comes by itself."""
    return out if len(out) > 1 else out[0]


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "rms_fwd":
        h = s["x"].float()
        out = ()
        if s["residual"] is not None:
            h = (h + s["residual"].float()).to(DT[c["residual"]])
            out = (h,)
            h = h.float()
        rstd = 1 / torch.sqrt(h.square().mean(1, keepdim=True) + EPS)
        y = h * rstd * s["gamma"]
        out = (_quantized(y, False) if c["y"] == "e4m3" else (y.to(DT[c["y"]]),)) + out
        return _one(out + (rstd[:, 0],) if c["stats"] else out)
    if op == "rms_bwd":
        rstd = s["rstd"][:, None]
        hhat, dy = s["h"].float() * rstd, s["dy"].float()
        d = dy * s["gamma"]
        dx = rstd * (d - hhat * (d * hhat).mean(1, keepdim=True))
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        return dx.to(DT[c["x"]]), (dy * hhat).sum(0)
    if op == "quantize":
        out = _quantized(s["x"], c["tiles"])
        return out + _quantized(s["x"].t(), c["tiles"]) if c["both"] else out
    if op == "linear8_fwd":
        z = _values(*s["x"], False) @ _values(*s["W"], True).t()
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _act(c["act"], z)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        return y.to(DT[c["type"]])
    if op == "linear8_bwd":
        dz = s["dy"].float()
        if s["z"] is not None:
            dz = dz * _dact(c["act"], s["z"].float())
        dx = (_rounded(dz) @ _values(*s["Wt"], True).t()).to(torch.bfloat16)
        dW = (_rounded(dz.t()) @ _values(*s["xt"], False).t()).to(DT[c["type"]])
        return (dx, dW, dz.sum(0)) if c["bias"] else (dx, dW)
    if op == "gated8_fwd":
        x = _values(*s["x"], False)
        g, u = x @ _values(*s["Wg"], True).t(), x @ _values(*s["Wu"], True).t()
        if s["bg"] is not None:
            g, u = g + s["bg"], u + s["bu"]
        h = _act(c["act"], g) * u
        out = _quantized(h, False) if c["type"] == "e4m3" else (h.to(torch.bfloat16),)
        return _one(out + (g.to(torch.bfloat16), u.to(torch.bfloat16)) if c["save"] else out)
    g, u, dh = s["g"].float(), s["u"].float(), s["dh"].float()
    dg, du = dh * u * _dact(c["act"], g), dh * _act(c["act"], g)
    dx = _rounded(dg) @ _values(*s["Wgt"], True).t() + _rounded(du) @ _values(*s["Wut"], True).t()
    x = _values(*s["xt"], False).t()
    out = dx.to(torch.bfloat16), (_rounded(dg.t()) @ x).to(torch.bfloat16), (_rounded(du.t()) @ x).to(torch.bfloat16)
    return out + (dg.sum(0), du.sum(0)) if c["bias"] else out


def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_1807_11091_gb300 import sadmm
    c, op = s["case"], s["case"]["op"]
    if op == "rms_fwd":
        return sadmm.rms_norm(s["x"], s["gamma"], residual=s["residual"], eps=EPS, out_dtype=DT[c["y"]],
                              stats=c["stats"])
    if op == "rms_bwd":
        return sadmm.rms_norm_backward(s["dy"], s["h"], s["rstd"], s["gamma"], dres=s["dres"])
    if op == "quantize":
        return sadmm.quantize(s["x"], tiles=c["tiles"], transposed=c["both"])
    act = getattr(sadmm, "SADMM_ACT_" + c["act"].upper())
    if op == "linear8_fwd":
        return sadmm.linear8(*s["x"], *s["W"], s["bias"], residual=s["residual"], act=act, out_dtype=DT[c["type"]])
    if op == "linear8_bwd":
        got = sadmm.linear8_backward(s["dy"], *s["xt"], *s["Wt"], z=s["z"], act=act, dw_dtype=DT[c["type"]],
                                     want_db=c["bias"])
        return got if c["bias"] else got[:2]
    if op == "gated8_fwd":
        return sadmm.gated8(*s["x"], *s["Wg"], *s["Wu"], s["bg"], s["bu"], act=act, out_dtype=DT[c["type"]],
                            save=c["save"])
    got = sadmm.gated8_backward(s["dh"], *s["xt"], *s["Wgt"], *s["Wut"], s["g"], s["u"], act=act, want_db=c["bias"])
    return got if c["bias"] else got[:3]


# ------------------------------------------------------------ in 64 bits --

def _exact_act(name, z):
    """The activation and its slope in 64 bits."""
    if name == "relu":
        return z.clamp_min(0), torch.heaviside(z, torch.zeros_like(z))
    if name == "gelu":
        p = torch.special.erfc(-z / math.sqrt(2.0)) / 2
        return z * p, p + z * torch.exp(-z ** 2 / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        p = (1 + torch.tanh(z / 2)) / 2
        return z * p, p + z * p * (1 - p)
    return z, torch.ones_like(z)


def _spread(s, rows, cols, high):
    """Scales of blocks of `high` rows and 128 columns, for each element."""
    return s.repeat_interleave(high, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :cols]


def _exact_quantized(x, high):
    """(values as e4m3 numbers in 64 bits, scales): blocks one after the other along the columns."""
    rows, cols = x.shape
    tops = [torch.nan_to_num(x[:, b:b + BLOCK].abs(), 0.0, 0.0, 0.0).amax(1) for b in range(0, cols, BLOCK)]
    top = torch.stack(tops, 1)
    if high > 1:
        top = torch.stack([top[b:b + high].amax(0) for b in range(0, rows, high)])
    s = torch.div(top.clamp(min=FLOOR), torch.full_like(top, LARGEST)).float()
    v = (x.float() / _spread(s, rows, cols, high)).double()  # the quotient is an fp32 number by definition
    # e4m3 has three digits after the leading one, down to steps of 2^-9
    power = torch.frexp(v)[1].long().sub(1).clamp(min=-6) - 3
    step = (power + 1023).bitwise_left_shift(52).view(torch.float64)  # 2^power, to the last digit
    return (torch.round(v / step) * step).clamp(-LARGEST, LARGEST), s.double()


def _exact_rounded(x):
    q, s = _exact_quantized(x, 1)
    return q * _spread(s, *x.shape, 1)


def _exact_operand(pair, high):
    q, s = pair
    return q.double() * _spread(s.double(), *q.shape, high)


def exact(case, seed):
    s = prepare(case, seed)
    c, op = case, case["op"]
    if op == "quantize":
        high, x = BLOCK if c["tiles"] else 1, s["x"].double()
        out = _exact_quantized(x, high)
        return out + _exact_quantized(x.t(), high) if c["both"] else out
    for name in ("x", "xt"):
        if isinstance(s.get(name), tuple):
            s[name] = _exact_operand(s[name], 1)
    for name in ("W", "Wt", "Wg", "Wu", "Wgt", "Wut"):
        if name in s:
            s[name] = _exact_operand(s[name], BLOCK)
    s = {k: v.double() if torch.is_tensor(v) else v for k, v in s.items()}
    if op == "rms_fwd":
        h, out = s["x"], ()
        if s["residual"] is not None:
            # what the norm reads is the sum as it is kept
            kept = (h + s["residual"]).to(DT[c["residual"]])
            h, out = kept.double(), (kept.double(),)
        rstd = (torch.linalg.vector_norm(h, dim=1) ** 2 / c["cols"] + EPS) ** -0.5
        y = torch.einsum("rc,r,c->rc", h, rstd, s["gamma"])
        out = (_exact_quantized(y, 1) if c["y"] == "e4m3" else (y,)) + out
        return _one(out + (rstd,) if c["stats"] else out)
    if op == "rms_bwd":
        # dL/dh from the norm's Jacobian, rstd (I - hhat hhat^T / n), applied to gamma * dy
        hhat = torch.einsum("rc,r->rc", s["h"], s["rstd"])
        d = torch.einsum("rc,c->rc", s["dy"], s["gamma"])
        along = torch.einsum("rc,rc->r", d, hhat) / c["cols"]
        dx = torch.einsum("r,rc->rc", s["rstd"], d - hhat * along.unsqueeze(1))
        if s["dres"] is not None:
            dx += s["dres"]
        return dx, torch.einsum("rc,rc->c", s["dy"], hhat)
    if op == "linear8_fwd":
        z = torch.einsum("tk,nk->tn", s["x"], s["W"])
        z = z if s["bias"] is None else z + s["bias"]
        y = _exact_act(c["act"], z)[0]
        return y if s["residual"] is None else y + s["residual"]
    if op == "linear8_bwd":
        dz = s["dy"] if s["z"] is None else s["dy"] * _exact_act(c["act"], s["z"])[1]
        out = (torch.einsum("tn,kn->tk", _exact_rounded(dz), s["Wt"]),
               torch.einsum("nt,kt->nk", _exact_rounded(dz.t()), s["xt"]))
        return out + (torch.einsum("tn->n", dz),) if c["bias"] else out
    if op == "gated8_fwd":
        g, u = torch.einsum("tk,nk->tn", s["x"], s["Wg"]), torch.einsum("tk,nk->tn", s["x"], s["Wu"])
        if s["bg"] is not None:
            g, u = g + s["bg"], u + s["bu"]
        h = _exact_act(c["act"], g)[0] * u
        out = _exact_quantized(h, 1) if c["type"] == "e4m3" else (h,)
        return _one(out + (g, u) if c["save"] else out)
    a, slope = _exact_act(c["act"], s["g"])
    dg, du = s["dh"] * s["u"] * slope, s["dh"] * a
    dx = (torch.einsum("tn,kn->tk", _exact_rounded(dg), s["Wgt"]) +
          torch.einsum("tn,kn->tk", _exact_rounded(du), s["Wut"]))
    out = dx, torch.einsum("nt,kt->nk", _exact_rounded(dg.t()), s["xt"]), torch.einsum(
        "nt,kt->nk", _exact_rounded(du.t()), s["xt"])
    return out + (torch.einsum("tn->n", dg), torch.einsum("tn->n", du)) if c["bias"] else out
