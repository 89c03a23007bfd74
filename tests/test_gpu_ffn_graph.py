"""The feed-forward calls captured in a CUDA graph: replays on new inputs give the bits of
plain calls."""
import pytest
import torch

import _ffn as F
from _ffn import FP32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("tokens,d,hidden,keep", [(4, 96, 200, 77), (12, 256, 512, 131), (700, 320, 1000, 501),
                                                  (2100, 513, 3000, 1501)])
def test_block_in_a_graph(tokens, d, hidden, keep):
    from paper_1807_11091_gb300 import sadmm
    from paper_1807_11091_gb300.run_ffn import make_block
    b = make_block(d, hidden, seed=tokens).pruned(keep)
    g = F.gen(tokens)
    x, dy = torch.empty(tokens, d, device="cuda"), torch.empty(tokens, d, device="cuda")

    def step():
        y = b.forward(x, train=True)
        dx, grads = b.backward(dy, dw_dtype=FP32)
        return [b.forward(x), y, dx] + [grads[k] for k in sorted(grads)]

    x.normal_(generator=g), dy.normal_(generator=g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step()
    for _ in range(3):
        x.normal_(generator=g), dy.normal_(generator=g)
        graph.replay()
        kept = [t.clone() for t in got]
        want = step()
        assert sadmm.device_status() == 0
        assert all(torch.equal(p, q) for p, q in zip(kept, want))
