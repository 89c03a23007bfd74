"""A gated feed-forward block with its hidden units pruned, from this library's calls.

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
