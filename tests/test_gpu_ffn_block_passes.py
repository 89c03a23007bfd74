"""Passes of one feed-forward block: several in flight, none, and a dy of another pass's shape."""
import pytest
import torch

from _ffn import FP32


def test_backward_without_a_pass():
    from paper_1807_11091_gb300.ffn import FeedForward
    w = torch.ones(8, 4)
    b = FeedForward(torch.ones(4), torch.zeros(4), w, w, w.t())
    with pytest.raises(RuntimeError, match="forward"):
        b.backward(torch.ones(2, 4))


@pytest.mark.gpu
def test_passes_in_flight():
    from paper_1807_11091_gb300 import sadmm
    from paper_1807_11091_gb300.run_ffn import make_block
    b = make_block(96, 200, seed=1).pruned(77)
    xs = [torch.randn(n, 96, device="cuda") for n in (40, 40, 7)]
    dys = [torch.randn_like(x) for x in xs]
    want = []
    for x, dy in zip(xs, dys):
        b.forward(x, train=True)
        want.append(b.backward(dy, dw_dtype=FP32))
    kept = []
    for x in xs:
        b.forward(x, train=True)
        kept.append(b.saved)
    for i in (1, 0, 2):
        dx, grads = b.backward(dys[i], dw_dtype=FP32, saved=kept[i])
        assert torch.equal(dx, want[i][0]) and all(torch.equal(grads[k], v) for k, v in want[i][1].items())
    dx, _ = b.backward(dys[2])  # the last pass's, as before
    assert torch.equal(dx, want[2][0])
    with pytest.raises(ValueError, match="dy is"):
        b.backward(dys[0])
    b.saved = None
    with pytest.raises(RuntimeError):
        b.backward(dys[2])
    assert sadmm.device_status() == 0
