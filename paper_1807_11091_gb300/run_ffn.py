"""Prunes one gated feed-forward block, runs its forward and backward pass, and times both.

    python -m paper_1807_11091_gb300.run_ffn --tokens 4096 --d 1024 --hidden 4096 --keep 0.5

Builds a seeded block, keeps the given share of its hidden units (the projection
of Sec. 4 with units as groups), runs forward and backward of the dense and of
the pruned block, checks the pruned one against plain fp32 torch, and prints the
time of each pass (CUDA events, median of `reps`).
"""
from __future__ import annotations

import argparse
import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)


def make_block(d: int, hidden: int, seed: int = 0):
    import torch

    from paper_1807_11091_gb300.ffn import FeedForward
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, scale=1.0):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    # units of different sizes, as training leaves them: the projection has something to choose by
    size = torch.exp(normal(hidden, 1, scale=0.5))
    return FeedForward(1 + normal(d, scale=0.1), normal(d, scale=0.1), normal(hidden, d, scale=d ** -0.5) * size,
                       normal(hidden, d, scale=d ** -0.5) * size, normal(d, hidden, scale=hidden ** -0.5) * size.t(),
                       normal(d, scale=0.1))


def plain(block, x):
    """The block in plain fp32 torch."""
    import torch
    x = x.float()
    m = x.mean(1, keepdim=True)
    n = (x - m) * ((x - m).square().mean(1, keepdim=True) + block.eps).rsqrt() * block.gamma + block.beta
    z = n @ block.Wg.float().t()
    return x + (z * torch.sigmoid(z) * (n @ block.Wu.float().t())) @ block.Wd.float().t() + block.bias


def timed(f, reps: int) -> float:
    import torch
    times = []
    for _ in range(reps + 3):
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        torch.cuda._sleep(200_000)
        a.record()
        f()
        b.record()
        torch.cuda.synchronize()
        times.append(a.elapsed_time(b) * 1e3)
    return sorted(times[3:])[reps // 2]


def main(argv=None) -> int:
    import torch

    from paper_1807_11091_gb300 import sadmm

    ap = argparse.ArgumentParser()
    ap.add_argument("--tokens", type=int, default=4096)
    ap.add_argument("--d", type=int, default=1024)
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--keep", type=float, default=0.5)
    ap.add_argument("--reps", type=int, default=5)
    args = ap.parse_args(argv)
    dense = make_block(args.d, args.hidden)
    block = dense.pruned(max(1, round(args.keep * args.hidden)))
    x = torch.randn(args.tokens, args.d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    dy = (x * 0.01).to(x.dtype)
    want, got = plain(block, x), block.forward(x)
    err = float((got - want).norm() / (want - x).norm())
    for name, b in (("dense", dense), (f"{block.hidden} units", block)):
        flops = 6.0 * args.tokens * args.d * b.hidden
        f = timed(lambda: b.forward(x), args.reps)
        t = timed(lambda: (b.forward(x, train=True), b.backward(dy)), args.reps)
        print(f"{name}: forward {f:.1f} us ({flops / f / 1e6:.0f} TFLOP/s), forward and backward {t:.1f} us "
              f"({3 * flops / t / 1e6:.0f} TFLOP/s)")
    print(f"pruned block against plain fp32: {err:.2e} of the branch's norm")
    return 1 if sadmm.device_status() != 0 or not err < 2e-2 else 0


if __name__ == "__main__":
    raise SystemExit(main())
