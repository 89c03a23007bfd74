"""The operators of a feed-forward block with pruned hidden units, as timed cases.

A transformer's feed-forward block is where structured pruning (StructADMM,
arXiv 1807.11091) takes the most weights from a language model: a hidden unit is
a row of the block's first products and a column of its last one, and a block
that keeps some of them is a smaller dense block of any width.  A program that
serves or retrains such a block calls three operators and their backward passes:
layer norm (``sadmm.layer_norm``), the gated pair of projections
(``sadmm.gated``) and the closing projection with bias, activation and residual
(``sadmm.linear``).  Each case is one such call.

A case's ``op`` is one of
  ln_fwd      x -> y, and the rows' mean and 1/std where they are kept
  ln_bwd      dy, x, mean, rstd (and the residual's gradient) -> dx, dgamma, dbeta
  linear_fwd  act(x W^T + bias) + residual -> y, and the pre-activation z where kept
  linear_bwd  dy, x, W, z -> dx, dW, db
  gated_fwd   act(x Wg^T + bg) * (x Wu^T + bu) -> h, and both pre-activations where kept
  gated_bwd   dh, x, Wg, Wu, g, u -> dx, dWg, dWu, dbg, dbu

``pad`` says that matrices lie in buffers whose rows start on 64-byte
boundaries, as a program that may choose its buffers has them; without it they
are dense, so that an odd width gives rows of every alignment.
"""
import math

import torch

own = False  # whether run() calls the framework's operators, or computes their plain forms

EPS = 1e-5
DT = {"bf16": torch.bfloat16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp32": 4}


# ------------------------------------------------------------------ cases --

def _ln(name, op, rows, cols, x, y, stats=False, dres=False, pad=False):
    return {"name": name, "op": op, "rows": rows, "cols": cols, "x": x, "y": y, "stats": stats, "dres": dres,
            "pad": pad}


def _linear(name, op, tokens, n_in, n_out, act, bias, residual, save, out, pad=True):
    return {"name": name, "op": op, "tokens": tokens, "in": n_in, "out": n_out, "act": act, "bias": bias,
            "residual": residual, "save": save, "type": out, "pad": pad}


def _gated(name, op, tokens, n_in, hidden, act, bias, save, pad=True):
    return {"name": name, "op": op, "tokens": tokens, "in": n_in, "hidden": hidden, "act": act, "bias": bias,
            "save": save, "pad": pad}


def listed():
    return [
        # the newest token of four sequences, where the call's own latency counts
        _ln("ln_fwd_4_tokens", "ln_fwd", 4, 2048, "bf16", "bf16"),
        # a training batch's residual stream in fp32, normed into the products' type
        _ln("ln_fwd_batch", "ln_fwd", 16384, 4096, "fp32", "bf16", stats=True),
        # the same norm's backward pass, with the gradient that came along the residual
        _ln("ln_bwd_batch", "ln_bwd", 8192, 4096, "bf16", "bf16", dres=True),
        # a ragged batch of a narrow model of odd width: rows of every alignment
        _ln("ln_bwd_ragged", "ln_bwd", 3001, 1153, "fp32", "bf16"),
        # serving one sequence: the closing projection of one token, bound by the weights
        _linear("linear_1_token", "linear_fwd", 1, 5120, 2048, "none", False, True, False, "bf16"),
        # training: a square projection with bias and activation, its pre-activation kept
        _linear("linear_batch", "linear_fwd", 4096, 4096, 4096, "gelu", True, False, True, "bf16"),
        # a prompt of odd length through a third of the hidden units, dense rows, fp32 residual stream
        _linear("linear_ragged", "linear_fwd", 777, 2731, 1025, "none", True, True, False, "fp32", pad=False),
        # retraining: the closing projection's gradients, the weights' in fp32
        _linear("linear_bwd_batch", "linear_bwd", 8192, 5120, 2048, "none", True, False, False, "fp32"),
        # retraining a small block of odd widths through its activation
        _linear("linear_bwd_ragged", "linear_bwd", 1025, 1024, 2731, "gelu", True, False, False, "bf16", pad=False),
        # serving eight sequences: the gated pair on their newest tokens, an odd number of units kept
        _gated("gated_8_tokens", "gated_fwd", 8, 2048, 5461, "silu", False, False),
        # training: the gated pair of a wide block on a whole batch, the most work here
        _gated("gated_batch", "gated_fwd", 8192, 4096, 10240, "silu", False, True),
        # retraining: its backward pass with an odd number of units kept
        _gated("gated_bwd_batch", "gated_bwd", 4096, 2048, 5461, "silu", True, False),
    ]


def _size(rng, lo, hi):
    """A size spread over the logarithm of lo..hi: odd or of a warp's or tile's multiple."""
    v = math.exp(rng.uniform(math.log(lo), math.log(hi)))
    step = rng.choice([1, 1, 1, 8, 64])
    return max(lo, min(hi, int(round(v / step)) * step if v >= step else int(round(v))))


def draw(rng):
    op = rng.choice(["ln_fwd", "ln_bwd", "linear_fwd", "linear_fwd", "linear_bwd", "gated_fwd", "gated_fwd", "gated_bwd"])
    pad = rng.random() < 0.6
    while True:
        if op.startswith("ln"):
            c = _ln("", op, _size(rng, 1, 32768), _size(rng, 32, 8192), rng.choice(["bf16", "fp32"]),
                    rng.choice(["bf16", "bf16", "fp32"]), rng.random() < 0.5, rng.random() < 0.5, pad)
        elif op.startswith("linear"):
            c = _linear("", op, _size(rng, 1, 8192), _size(rng, 64, 8192), _size(rng, 64, 8192),
                        rng.choice(["none", "relu", "gelu", "silu"]), rng.random() < 0.5, rng.random() < 0.5,
                        rng.random() < 0.3, rng.choice(["bf16", "bf16", "fp32"]), pad)
            if op == "linear_bwd" and c["act"] != "none":
                c["type"] = "bf16"
        else:
            c = _gated("", op, _size(rng, 1, 8192), _size(rng, 64, 4096), _size(rng, 64, 10240),
                       rng.choice(["relu", "gelu", "silu", "silu"]), rng.random() < 0.5, rng.random() < 0.5, pad)
        w = work(c)
        if w["flops"] <= 1.3e12 and w["bytes"] <= 4e8 and 3072 not in c.values():
            del c["name"]
            return c


def work(case):
    """The bytes that one pass has to read and write and the operations that it has to do."""
    c, op = case, case["op"]
    if op.startswith("ln"):
        n, m, x, y = c["rows"] * c["cols"], c["cols"], SIZE[c["x"]], SIZE[c["y"]]
        stats = 8 * c["rows"]
        if op == "ln_fwd":
            return {"bytes": n * (x + y) + 8 * m + stats * c["stats"], "flops": 8 * n}
        return {"bytes": n * (2 * x + y + x * c["dres"]) + 12 * m + stats, "flops": 14 * n}
    t, k = c["tokens"], c["in"]
    if op.startswith("linear"):
        n, s = c["out"], SIZE[c["type"]]
        if op == "linear_fwd":
            return {"bytes": 2 * (t * k + n * k) + t * n * (s + s * c["residual"] + 2 * c["save"]) + 4 * n * c["bias"],
                    "flops": 2 * t * k * n}
        z = c["act"] != "none"
        return {"bytes": 2 * (2 * t * k + n * k + t * n * (1 + z)) + s * n * k + 4 * n * c["bias"],
                "flops": 4 * t * k * n}
    n = c["hidden"]
    if op == "gated_fwd":
        return {"bytes": 2 * (t * k + 2 * n * k + t * n * (1 + 2 * c["save"])) + 8 * n * c["bias"],
                "flops": 4 * t * k * n}
    return {"bytes": 2 * (2 * t * k + 4 * n * k + 3 * t * n) + 8 * n * c["bias"], "flops": 8 * t * k * n}


# ----------------------------------------------------------------- inputs --

def _matrix(g, rows, cols, dtype, pad, scale=1.0, offset=0.0):
    """[rows][cols] of N(offset, scale^2), in a buffer of its own rows or of rows on 64-byte boundaries."""
    step = 64 // torch.empty((), dtype=dtype).element_size() if pad else 1
    ld = -(-cols // step) * step
    buf = torch.empty(rows, ld, dtype=torch.float32, device="cuda").normal_(generator=g).mul_(scale).add_(offset)
    return buf.to(dtype)[:, :cols]


def prepare(case, seed):
    c, op = case, case["op"]
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c}
    if op.startswith("ln"):
        rows, cols, x, y = c["rows"], c["cols"], DT[c["x"]], DT[c["y"]]
        # a residual stream: an offset of its own, and a channel in 64 some 8 times as large as the others
        s["x"] = _matrix(g, rows, cols, x, c["pad"], 1.5, 0.25)
        s["x"][:, 7::64] *= 8
        s["gamma"] = torch.empty(cols, device="cuda").normal_(generator=g).mul_(0.1).add_(1)
        s["beta"] = torch.empty(cols, device="cuda").normal_(generator=g).mul_(0.1)
        if op == "ln_bwd":
            f = s["x"].float()
            s["mean"] = f.mean(1)
            s["rstd"] = ((f - s["mean"][:, None]).square().mean(1) + EPS).rsqrt()
            s["dy"] = _matrix(g, rows, cols, y, c["pad"], 1e-2)
            s["dres"] = _matrix(g, rows, cols, x, c["pad"], 1e-2) if c["dres"] else None
        return s
    t, k, pad = c["tokens"], c["in"], c["pad"]
    s["x"] = _matrix(g, t, k, torch.bfloat16, pad)
    if op.startswith("linear"):
        n = c["out"]
        s["W"] = _matrix(g, n, k, torch.bfloat16, pad, k ** -0.5)
        s["bias"] = torch.empty(n, device="cuda").normal_(generator=g).mul_(0.1) if c["bias"] else None
        if op == "linear_fwd":
            s["residual"] = _matrix(g, t, n, DT[c["type"]], pad) if c["residual"] else None
        else:
            s["dy"] = _matrix(g, t, n, torch.bfloat16, pad, 1e-2)
            s["z"] = _matrix(g, t, n, torch.bfloat16, pad) if c["act"] != "none" else None
        return s
    n = c["hidden"]
    s["Wg"] = _matrix(g, n, k, torch.bfloat16, pad, 1.5 * k ** -0.5)
    s["Wu"] = _matrix(g, n, k, torch.bfloat16, pad, k ** -0.5)
    s["bg"] = torch.empty(n, device="cuda").normal_(generator=g).mul_(0.1) if c["bias"] else None
    s["bu"] = torch.empty(n, device="cuda").normal_(generator=g).mul_(0.1) if c["bias"] else None
    if op == "gated_bwd":
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


def _plain(s):
    c, op = s["case"], s["case"]["op"]
    if op == "ln_fwd":
        x = s["x"].float()
        mean = x.mean(1, keepdim=True)
        rstd = 1 / torch.sqrt((x - mean).square().mean(1, keepdim=True) + EPS)
        y = ((x - mean) * rstd * s["gamma"] + s["beta"]).to(DT[c["y"]])
        return (y, mean[:, 0], rstd[:, 0]) if c["stats"] else y
    if op == "ln_bwd":
        xhat = (s["x"].float() - s["mean"][:, None]) * s["rstd"][:, None]
        dy = s["dy"].float()
        d = dy * s["gamma"]
        dx = s["rstd"][:, None] * (d - d.mean(1, keepdim=True) - xhat * (d * xhat).mean(1, keepdim=True))
        if s["dres"] is not None:
            dx = dx + s["dres"].float()
        return dx.to(DT[c["x"]]), (dy * xhat).sum(0), dy.sum(0)
    x = s["x"].float()
    if op == "linear_fwd":
        z = x @ s["W"].float().t()
        if s["bias"] is not None:
            z = z + s["bias"]
        y = _act(c["act"], z)
        if s["residual"] is not None:
            y = y + s["residual"].float()
        y = y.to(DT[c["type"]])
        return (y, z.to(torch.bfloat16)) if c["save"] else y
    if op == "linear_bwd":
        dz = s["dy"].float()
        if s["z"] is not None:
            dz = dz * _dact(c["act"], s["z"].float())
        dx = (dz @ s["W"].float()).to(torch.bfloat16)
        dW = (dz.t() @ x).to(DT[c["type"]])
        return (dx, dW, dz.sum(0)) if c["bias"] else (dx, dW)
    if op == "gated_fwd":
        g, u = x @ s["Wg"].float().t(), x @ s["Wu"].float().t()
        if s["bg"] is not None:
            g, u = g + s["bg"], u + s["bu"]
        h = (_act(c["act"], g) * u).to(torch.bfloat16)
        return (h, g.to(torch.bfloat16), u.to(torch.bfloat16)) if c["save"] else h
    g, u, dh = s["g"].float(), s["u"].float(), s["dh"].float()
    dg, du = dh * u * _dact(c["act"], g), dh * _act(c["act"], g)
    dx = (dg @ s["Wg"].float() + du @ s["Wu"].float()).to(torch.bfloat16)
    out = dx, (dg.t() @ x).to(torch.bfloat16), (du.t() @ x).to(torch.bfloat16)
    return out + (dg.sum(0), du.sum(0)) if c["bias"] else out


def run(state):
    s = state
    if not own:
        return _plain(s)
    from paper_1807_11091_gb300 import sadmm
    c, op = s["case"], s["case"]["op"]
    if op == "ln_fwd":
        return sadmm.layer_norm(s["x"], s["gamma"], s["beta"], eps=EPS, out_dtype=DT[c["y"]], stats=c["stats"])
    if op == "ln_bwd":
        return sadmm.layer_norm_backward(s["dy"], s["x"], s["mean"], s["rstd"], s["gamma"], dres=s["dres"])
    act = getattr(sadmm, "SADMM_ACT_" + c["act"].upper())
    if op == "linear_fwd":
        return sadmm.linear(s["x"], s["W"], s["bias"], residual=s["residual"], act=act, out_dtype=DT[c["type"]],
                            save=c["save"])
    if op == "linear_bwd":
        got = sadmm.linear_backward(s["dy"], s["x"], s["W"], z=s["z"], act=act, dw_dtype=DT[c["type"]],
                                    want_db=c["bias"])
        return got if c["bias"] else got[:2]
    if op == "gated_fwd":
        return sadmm.gated(s["x"], s["Wg"], s["Wu"], s["bg"], s["bu"], act=act, save=c["save"])
    got = sadmm.gated_backward(s["dh"], s["x"], s["Wg"], s["Wu"], s["g"], s["u"], act=act, want_db=c["bias"])
    return got if c["bias"] else got[:3]


# ------------------------------------------------------------ in 64 bits --

def _normal_cdf(z):
    return torch.special.erfc(-z / math.sqrt(2.0)) / 2


def _exact_act(name, z):
    """The activation and its slope in 64 bits."""
    if name == "relu":
        return z.clamp_min(0), torch.heaviside(z, torch.zeros_like(z))
    if name == "gelu":
        p = _normal_cdf(z)
        return z * p, p + z * torch.exp(-z ** 2 / 2) / math.sqrt(2 * math.pi)
    if name == "silu":
        p = (1 + torch.tanh(z / 2)) / 2
        return z * p, p + z * p * (1 - p)
    return z, torch.ones_like(z)


def exact(case, seed):
    s = {k: v.double() if torch.is_tensor(v) else v for k, v in prepare(case, seed).items()}
    c, op = case, case["op"]
    if op == "ln_fwd":
        var, mean = torch.var_mean(s["x"], 1, correction=0)
        rstd = (var + EPS) ** -0.5
        y = torch.addcmul(s["beta"], (s["x"] - mean[:, None]) * rstd[:, None], s["gamma"])
        return (y, mean, rstd) if c["stats"] else y
    if op == "ln_bwd":
        # dL/dx from the norm's Jacobian, rstd/n (n I - 1 1^T - xhat xhat^T), applied to gamma * dy
        n = c["cols"]
        xhat = torch.einsum("rc,r->rc", s["x"] - s["mean"].unsqueeze(1), s["rstd"])
        d = torch.einsum("rc,c->rc", s["dy"], s["gamma"])
        along = torch.einsum("rc,rc->r", d, xhat)
        dx = torch.einsum("r,rc->rc", s["rstd"] / n, n * d - d.sum(1).unsqueeze(1) - xhat * along.unsqueeze(1))
        if s["dres"] is not None:
            dx += s["dres"]
        return dx, torch.einsum("rc,rc->c", s["dy"], xhat), torch.einsum("rc->c", s["dy"])
    if op == "linear_fwd":
        z = torch.einsum("tk,nk->tn", s["x"], s["W"])
        z = z if s["bias"] is None else z + s["bias"]
        y = _exact_act(c["act"], z)[0]
        y = y if s["residual"] is None else y + s["residual"]
        return (y, z) if c["save"] else y
    if op == "linear_bwd":
        dz = s["dy"] if s["z"] is None else s["dy"] * _exact_act(c["act"], s["z"])[1]
        out = torch.einsum("tn,nk->tk", dz, s["W"]), torch.einsum("tn,tk->nk", dz, s["x"])
        return out + (torch.einsum("tn->n", dz),) if c["bias"] else out
    if op == "gated_fwd":
        g, u = torch.einsum("tk,nk->tn", s["x"], s["Wg"]), torch.einsum("tk,nk->tn", s["x"], s["Wu"])
        if s["bg"] is not None:
            g, u = g + s["bg"], u + s["bu"]
        h = _exact_act(c["act"], g)[0] * u
        return (h, g, u) if c["save"] else h
    a, slope = _exact_act(c["act"], s["g"])
    dg, du = s["dh"] * s["u"] * slope, s["dh"] * a
    out = (torch.einsum("tn,nk->tk", dg, s["Wg"]) + torch.einsum("tn,nk->tk", du, s["Wu"]),
           torch.einsum("tn,tk->nk", dg, s["x"]), torch.einsum("tn,tk->nk", du, s["x"]))
    return out + (torch.einsum("tn->n", dg), torch.einsum("tn->n", du)) if c["bias"] else out
