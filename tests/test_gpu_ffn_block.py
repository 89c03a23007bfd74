"""The gated feed-forward block (ffn.py): its operators together, the units that the
projection keeps, and the command that runs it."""
import pytest
import torch

import _ffn as F
from _ffn import U16

pytestmark = pytest.mark.gpu


def reference(b, x, dy):
    """y, dx and the weights' gradients in 64 bits by torch's autograd, and y's branch alone."""
    p = {k: getattr(b, k).double().clone().requires_grad_() for k in ("gamma", "beta", "Wg", "Wu", "Wd", "bias")}
    x = x.double().clone().requires_grad_()
    n = torch.nn.functional.layer_norm(x, x.shape[1:], p["gamma"], p["beta"], b.eps)
    z = n @ p["Wg"].t()
    branch = (z * torch.sigmoid(z) * (n @ p["Wu"].t())) @ p["Wd"].t() + p["bias"]
    (x + branch).backward(dy.double())
    return branch.detach(), x.grad, {k: v.grad for k, v in p.items()}


@pytest.mark.parametrize("tokens,d,hidden,keep", [(1, 96, 200, 77), (40, 256, 512, 131), (700, 320, 1000, 501)])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_block_forward_and_backward(tokens, d, hidden, keep, dtype):
    """In norms: n, g, u, h, dh, dg and du are each rounded to bf16 (U16 / sqrt 3 of their norm when
    the roundings are independent) and so is each result; four such steps lie on the longest path to a
    gradient, and each output is held to 4 U16 of its norm."""
    from paper_1807_11091_gb300 import sadmm
    from paper_1807_11091_gb300.run_ffn import make_block
    b = make_block(d, hidden, seed=tokens).pruned(keep)
    assert b.hidden == keep
    g = F.gen(tokens)
    x = torch.randn(tokens, d, generator=g, device="cuda").to(dtype)
    dy = torch.randn(tokens, d, generator=g, device="cuda").to(dtype)
    y = b.forward(x)
    assert torch.equal(b.forward(x, train=True), y)
    dx, grads = b.backward(dy, dw_dtype=torch.float32)
    assert sadmm.device_status() == 0
    branch, wdx, want = reference(b, x, dy)
    assert (y.double() - x.double() - branch).norm() <= 4 * U16 * branch.norm() + U16 * y.double().norm() * (dtype != torch.float32)
    assert (dx.double() - wdx).norm() <= 4 * U16 * wdx.norm()
    for k, w in want.items():
        assert (grads[k].double() - w).norm() <= 4 * U16 * w.norm() + 1e-12, k


def test_kept_units_are_those_of_the_largest_norm():
    from paper_1807_11091_gb300.run_ffn import make_block
    b = make_block(64, 300, seed=3)
    norms = (b.Wg.double().square().sum(1) + b.Wu.double().square().sum(1) + b.Wd.double().square().sum(0))
    for k in (1, 150, 299, 300):
        want = norms.topk(k).indices.sort().values
        assert torch.equal(b.kept_units(k).long(), want)


def test_command():
    from paper_1807_11091_gb300 import run_ffn
    assert run_ffn.main(["--tokens", "300", "--d", "192", "--hidden", "400", "--keep", "0.33", "--reps", "1"]) == 0
