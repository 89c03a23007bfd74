"""The feed-forward block with 8-bit operands (ffn.FeedForward8): its operators together.

y is held to the plain formula in 64 bits, in norms: a rounding to e4m3 is off by at most 2^-4 of a value,
evenly spread 2^-4 / sqrt 3 = 0.036; on the path to y lie those of n, Wg and Wu, h and Wd, six at most, whose
independent errors add up to sqrt 6 * 0.036 = 0.09, and the branch is held to 2^-3.

A gradient's path has more of them, and slopes that enlarge an error.  So the gradients are held to the
same roundings taken in 64 bits: what is left are the intermediate results' roundings to bf16 that fall
the other way, each less than U16 of the norm, and the result's own: 4 U16 of its norm, as for FeedForward."""
import pytest
import torch

import _ffn as F
from _ffn import BF16, FP32, U16
from _q8 import E4M3, quantized, values
from paper_1807_11091_gb300 import run_ffn, sadmm
from paper_1807_11091_gb300.ffn import FeedForward8

pytestmark = pytest.mark.gpu
BOUND = 2.0 ** -3


def block(d, hidden, keep, seed):
    b = run_ffn.make_block(d, hidden, seed=seed, bits=8).pruned(keep)
    assert isinstance(b, FeedForward8) and b.hidden == keep
    return b


def plain(b, x):
    """The branch in 64 bits."""
    x = x.double()
    n = x * (x.square().mean(1, keepdim=True) + b.eps).rsqrt() * b.gamma.double()
    z = n @ b.Wg.double().t()
    return (z * torch.sigmoid(z) * (n @ b.Wu.double().t())) @ b.Wd.double().t() + b.bias.double()


def made8(v, tiles=False):
    return values(*quantized(v.float(), tiles))


def bf16(v):
    return v.float().to(BF16).double()


def rounded_pass(b, x, dy):
    """The training pass with its roundings, and everything between them in 64 bits: branch, dx and the
    weights' gradients."""
    x, dy = x.double(), dy.double()
    rstd = (x.square().mean(1, keepdim=True) + b.eps).rsqrt()
    xhat, gamma = x * rstd, b.gamma.double()
    n = bf16(xhat * gamma)
    Wg, Wu, Wd = (made8(w, True) for w in (b.Wg, b.Wu, b.Wd))
    g, u = made8(n) @ Wg.t(), made8(n) @ Wu.t()
    h = bf16(g * torch.sigmoid(g) * u)
    branch = made8(h) @ Wd.t() + b.bias.double()
    dh = bf16(made8(dy) @ Wd)
    g, u = bf16(g), bf16(u)
    p = torch.sigmoid(g)
    dg, du = dh * u * (p + g * p * (1 - p)), dh * g * p
    dn = bf16(made8(dg) @ Wg + made8(du) @ Wu)
    nt, ht = made8(n.t()), made8(h.t())
    grads = {"gamma": (dn * xhat).sum(0), "bias": dy.sum(0), "Wg": made8(dg.t()) @ nt.t(), "Wu": made8(du.t()) @ nt.t(),
             "Wd": made8(dy.t()) @ ht.t()}
    d = dn * gamma
    return branch, rstd * (d - xhat * (d * xhat).mean(1, keepdim=True)) + dy, grads


@pytest.mark.parametrize("tokens,d,hidden,keep", [(1, 96, 200, 77), (40, 256, 512, 131), (700, 320, 1000, 501)])
@pytest.mark.parametrize("dtype", [FP32, BF16])
def test_block_forward_and_backward(tokens, d, hidden, keep, dtype):
    b = block(d, hidden, keep, tokens)
    g = F.gen(tokens)
    x, dy = (torch.randn(tokens, d, generator=g, device="cuda").to(dtype) for _ in range(2))
    want = plain(b, x)
    step = U16 * x.double().norm() * (dtype == BF16)
    y = b.forward(x)
    assert y.dtype == dtype and (y.double() - x.double() - want).norm() <= BOUND * want.norm() + step
    y = b.forward(x, train=True)
    assert (y.double() - x.double() - want).norm() <= BOUND * want.norm() + step
    dx, grads = b.backward(dy, dw_dtype=FP32)
    assert sadmm.device_status() == 0
    branch, wdx, want = rounded_pass(b, x, dy)
    assert (y.double() - x.double() - branch).norm() <= 4 * U16 * branch.norm() + step
    assert dx.dtype == dtype and (dx.double() - wdx).norm() <= 4 * U16 * wdx.norm()
    for k, w in want.items():
        assert (grads[k].double() - w).norm() <= 4 * U16 * w.norm() + 1e-12, k


@pytest.mark.parametrize("tokens", [3, 200])
def test_with_the_last_layers_output_to_add(tokens):
    """x + delta, added on the way: the same as adding it before."""
    b = block(256, 512, 301, 5)
    g = F.gen(6)
    x, delta = torch.randn(tokens, 256, generator=g, device="cuda"), torch.randn(tokens, 256, generator=g, device="cuda").to(BF16)
    dy = torch.randn(tokens, 256, generator=g, device="cuda")
    s = x + delta.float()
    assert torch.equal(b.forward(x, delta), b.forward(s))
    y = b.forward(x, delta, train=True)
    got = b.backward(dy)
    assert torch.equal(y, b.forward(s, train=True))
    want = b.backward(dy)
    assert torch.equal(got[0], want[0]) and all(torch.equal(got[1][k], want[1][k]) for k in want[1])


def test_changed_weights_count_after_quantize():
    b = block(128, 300, 200, 7)
    x = torch.randn(10, 128, device="cuda")
    y = b.forward(x)
    b.Wd.mul_(2)
    assert torch.equal(b.forward(x), y)
    b.quantize()
    # a product with 2 is exact in every step, the bias aside
    assert torch.allclose(b.forward(x) - x - b.bias, 2 * (y - x - b.bias), rtol=0, atol=2e-5)


def test_passes_in_flight():
    b = block(96, 200, 77, 1)
    xs = [torch.randn(n, 96, device="cuda") for n in (40, 40, 7)]
    want, kept = [], []
    for x in xs:
        b.forward(x, train=True)
        want.append(b.backward(x))
    for x in xs:
        b.forward(x, train=True)
        kept.append(b.saved)
    for x, k, w in zip(xs, kept, want):
        dx, grads = b.backward(x, saved=k)
        assert torch.equal(dx, w[0]) and all(torch.equal(grads[n], w[1][n]) for n in grads)
    with pytest.raises(ValueError, match="dy is"):
        b.backward(xs[0], saved=kept[2])
    b.saved = None
    with pytest.raises(RuntimeError, match="forward"):
        b.backward(xs[0])


@pytest.mark.parametrize("tokens,d,hidden,keep", [(4, 96, 200, 77), (700, 320, 1000, 501), (2100, 513, 3000, 1501)])
def test_block_in_a_graph(tokens, d, hidden, keep):
    """Captured, and replayed on new inputs: the bits of plain calls.  A second graph of the same block, replayed on
    another stream at the same time, has memory of its own."""
    b = block(d, hidden, keep, tokens)
    g = F.gen(tokens)
    xs, dys = [[torch.empty(tokens, d, device="cuda") for _ in range(2)] for _ in range(2)]

    def step(i):
        y = b.forward(xs[i], train=True)
        dx, grads = b.backward(dys[i], dw_dtype=FP32)
        return [b.forward(xs[i]), y, dx] + [grads[k] for k in sorted(grads)]

    def fill():
        for t in xs + dys:
            t.normal_(generator=g)

    fill()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(0)
    torch.cuda.current_stream().wait_stream(side)
    graphs, got = [torch.cuda.CUDAGraph() for _ in range(2)], []
    for i in range(2):
        with torch.cuda.graph(graphs[i]):
            got.append(step(i))
    for _ in range(3):
        fill()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        for i in range(2):
            kept = [t.clone() for t in got[i]]
            want = step(i)
            assert all(torch.equal(p, q) for p, q in zip(kept, want))
    assert sadmm.device_status() == 0


def test_command():
    assert run_ffn.main(["--tokens", "300", "--d", "192", "--hidden", "400", "--keep", "0.33", "--reps", "1", "--bits", "8"]) == 0


def test_results_of_one_call_are_the_next_ones_operands_where_they_lie():
    """Rows on 32-byte boundaries, also of an odd width: no call in the chain has scratch for a copy."""
    x = torch.randn(5, 333, device="cuda").to(BF16)
    q, s = sadmm.rms_norm(x, out_dtype=E4M3)
    w = torch.randn(77, 333, device="cuda")
    (qw, sw), (qu, su) = sadmm.quantize(w, tiles=True), sadmm.quantize(w, tiles=True)
    h, hs = sadmm.gated8(q, s, qw, sw, qu, su)
    for t in (q, qw, h):
        assert t.stride(0) % 32 == 0 and t.data_ptr() % 32 == 0
    assert s.stride(0) == 1 and hs.stride(0) == 1
