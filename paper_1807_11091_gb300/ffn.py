"""Gated feed-forward blocks with their hidden units pruned, from this library's calls:
FeedForward in bf16, and FeedForward8 with 8-bit operands and an RMS norm.

    y = x + act(n Wg^T) * (n Wu^T) Wd^T + b,   n = layer norm of x

A hidden unit is a row of Wg, a row of Wu and a column of Wd.  Structured pruning
(StructADMM, arXiv 1807.11091, Sec. 4: keep the k groups of the largest Euclidean
norm) takes units as its groups: the three together are one filter of a 1x1
layer with 3 D channels, so ``sadmm_project_groups`` chooses them.  The kept
units make a smaller dense block of any width.
"""
from __future__ import annotations

from . import sadmm


class FeedForward:
    """The block's weights (bf16; vectors fp32) and what its backward pass needs.

    Wg, Wu [H][D] and Wd [D][H] are kept in buffers whose rows start on 32-byte
    boundaries, so that an odd number of units costs nothing.

    ``saved`` is what the last forward(train=True) of the object kept: its input
    and activations.  They live until the next such pass, or until ``saved`` is
    set to None.  A program with several passes in flight (micro-batches,
    threads) keeps each pass's own and hands it to its backward:

        y = block.forward(x, train=True); kept = block.saved
        ...
        dx, grads = block.backward(dy, saved=kept)

    (threads that share an object take its ``saved`` under the lock of their
    forward).  Nothing here is recorded for torch's autograd.
    """

    def __init__(self, gamma, beta, Wg, Wu, Wd, bias=None, act: int = sadmm.SADMM_ACT_SILU, eps: float = 1e-5):
        self.gamma, self.beta, self.bias, self.act, self.eps = gamma, beta, bias, act, eps
        self.Wg, self.Wu, self.Wd = (self._rows(w) for w in (Wg, Wu, Wd))
        self.saved = None

    @staticmethod
    def _rows(w):
        import torch
        ld = (w.shape[1] + 15) // 16 * 16
        out = torch.zeros((w.shape[0], ld), dtype=torch.bfloat16, device=w.device)[:, :w.shape[1]]
        out.copy_(w)
        return out

    @property
    def hidden(self) -> int:
        return self.Wg.shape[0]

    def kept_units(self, k: int):
        """The k units of the largest Euclidean norm, ascending (an int32 device tensor)."""
        import torch
        units = torch.cat((self.Wg, self.Wu, self.Wd.t()), 1).contiguous()
        h, c = units.shape
        desc16 = [1, c, 1, 1, 1, h, 1, 1, 1, 1, 1, 1, 1, 0, 0, 0]
        return sadmm.project_groups(desc16, units, k, sadmm.SADMM_COL_NONE, 0)[0]

    def pruned(self, k: int) -> "FeedForward":
        """The block of the k units that the projection keeps."""
        i = self.kept_units(k).long()
        return FeedForward(self.gamma, self.beta, self.Wg[i], self.Wu[i], self.Wd[:, i], self.bias, self.act, self.eps)

    def forward(self, x, train: bool = False):
        """x [tokens][D] (bf16 or fp32, the residual stream) -> y of the same type."""
        import torch
        if not train:
            n = sadmm.layer_norm(x, self.gamma, self.beta, self.eps, out_dtype=torch.bfloat16)
            h = sadmm.gated(n, self.Wg, self.Wu, act=self.act)
            return sadmm.linear(h, self.Wd, self.bias, residual=x)
        n, mean, rstd = sadmm.layer_norm(x, self.gamma, self.beta, self.eps, out_dtype=torch.bfloat16, stats=True)
        h, g, u = sadmm.gated(n, self.Wg, self.Wu, act=self.act, save=True)
        self.saved = (x, n, mean, rstd, h, g, u)
        return sadmm.linear(h, self.Wd, self.bias, residual=x)

    def backward(self, dy, dw_dtype=None, saved=None):
        """Gradients for dy (of x's shape and type) of the pass that `saved` is of, otherwise of the
        last forward(train=True): dx and a dict of the weights'."""
        saved = self.saved if saved is None else saved
        if saved is None:
            raise RuntimeError("backward needs a forward(train=True) before it")
        x, n, mean, rstd, h, g, u = saved
        if dy.shape != x.shape:
            raise ValueError(f"dy is {tuple(dy.shape)}, the pass's x {tuple(x.shape)}")
        dh, dWd, db = sadmm.linear_backward(dy, h, self.Wd, want_db=self.bias is not None, dw_dtype=dw_dtype)
        dn, dWg, dWu, _, _ = sadmm.gated_backward(dh, n, self.Wg, self.Wu, g, u, act=self.act, dw_dtype=dw_dtype)
        dx, dgamma, dbeta = sadmm.layer_norm_backward(dn, x, mean, rstd, self.gamma, dres=dy)
        return dx, {"gamma": dgamma, "beta": dbeta, "Wg": dWg, "Wu": dWu, "Wd": dWd, "bias": db}


class FeedForward8:
    """The block with 8-bit operands, after an RMS norm:

        y = x + act(n Wg^T) * (n Wu^T) Wd^T + b,   n = RMS norm of x

    Wg, Wu, Wd are kept in bf16 as FeedForward keeps them, for pruning and for
    updates, and in 8 bits with a scale for each 128 x 128 tile, as they are and
    transposed.  Whoever changes the bf16 weights calls ``quantize()`` afterwards.
    ``saved`` is as in FeedForward: what a backward pass reads of its forward(train=True).

    A training pass does not give the bits of a plain one: n and h are rounded to bf16 before
    they are made 8-bit (their transposes, which the gradients read, are made from bf16), where the
    plain pass makes them 8-bit from fp32.  The rounding is off by up to 2^-8, the 8-bit
    form by 2^-4 in either.
    """

    def __init__(self, gamma, Wg, Wu, Wd, bias=None, act: int = sadmm.SADMM_ACT_SILU, eps: float = 1e-5):
        self.gamma, self.bias, self.act, self.eps = gamma, bias, act, eps
        self.Wg, self.Wu, self.Wd = (FeedForward._rows(w) for w in (Wg, Wu, Wd))
        self.saved = None
        self.quantize()

    hidden, kept_units = FeedForward.hidden, FeedForward.kept_units

    def quantize(self) -> None:
        """Makes the 8-bit weights from the bf16 ones."""
        (*self.Wg8, qt, st), (*self.Wu8, ut, vt), (*self.Wd8, dt, et) = (
            sadmm.quantize(w, tiles=True, transposed=True) for w in (self.Wg, self.Wu, self.Wd))
        self.Wgt8, self.Wut8, self.Wdt8 = (qt, st), (ut, vt), (dt, et)

    def pruned(self, k: int) -> "FeedForward8":
        """The block of the k units that the projection keeps."""
        i = self.kept_units(k).long()
        return FeedForward8(self.gamma, self.Wg[i], self.Wu[i], self.Wd[:, i], self.bias, self.act, self.eps)

    def forward(self, x, delta=None, train: bool = False):
        """x [tokens][D] (bf16 or fp32, the residual stream) -> y of the same type.  With `delta`, the
        output of the layer before that is still to be added to it, that of x + delta (x itself stays as it is)."""
        import torch
        if not train:
            if delta is None:
                n = sadmm.rms_norm(x, self.gamma, eps=self.eps, out_dtype=torch.float8_e4m3fn)
            else:
                *n, x = sadmm.rms_norm(delta, self.gamma, residual=x, eps=self.eps, out_dtype=torch.float8_e4m3fn)
            h = sadmm.gated8(*n, *self.Wg8, *self.Wu8, act=self.act)
            return sadmm.linear8(*h, *self.Wd8, self.bias, residual=x)
        if delta is None:
            n, rstd = sadmm.rms_norm(x, self.gamma, eps=self.eps, out_dtype=torch.bfloat16, stats=True)
        else:
            n, x, rstd = sadmm.rms_norm(delta, self.gamma, residual=x, eps=self.eps, out_dtype=torch.bfloat16, stats=True)
        q, s, nt, nts = sadmm.quantize(n, transposed=True)
        h, g, u = sadmm.gated8(q, s, *self.Wg8, *self.Wu8, act=self.act, out_dtype=torch.bfloat16, save=True)
        q, s, ht, hts = sadmm.quantize(h, transposed=True)
        self.saved = (x, rstd, (nt, nts), g, u, (ht, hts))
        return sadmm.linear8(q, s, *self.Wd8, self.bias, residual=x)

    def backward(self, dy, dw_dtype=None, saved=None):
        """Gradients for dy (of x's shape and type) of the pass that `saved` is of, otherwise of the last
        forward(train=True): dx (delta's too) and a dict of the weights'."""
        saved = self.saved if saved is None else saved
        if saved is None:
            raise RuntimeError("backward needs a forward(train=True) before it")
        x, rstd, nt, g, u, ht = saved
        if dy.shape != x.shape:
            raise ValueError(f"dy is {tuple(dy.shape)}, the pass's x {tuple(x.shape)}")
        dh, dWd, db = sadmm.linear8_backward(dy, *ht, *self.Wdt8, want_db=self.bias is not None, dw_dtype=dw_dtype)
        dn, dWg, dWu, _, _ = sadmm.gated8_backward(dh, *nt, *self.Wgt8, *self.Wut8, g, u, act=self.act, dw_dtype=dw_dtype)
        dx, dgamma = sadmm.rms_norm_backward(dn, x, rstd, self.gamma, dres=dy)
        return dx, {"gamma": dgamma, "Wg": dWg, "Wu": dWu, "Wd": dWd, "bias": db}
