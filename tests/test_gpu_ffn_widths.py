"""Rows wider than the 65535 x 1024 columns that one launch's third dimension counts."""
import pytest
import torch

import _ffn as F
from _ffn import BF16, FP32, U32

pytestmark = pytest.mark.gpu


def test_linear_of_very_wide_unaligned_rows():
    """Some 3000 terms of each row are not zero, and adding a zero rounds nothing: the sums' error is
    that of 3000 terms at most."""
    from paper_1807_11091_gb300 import sadmm
    T, K, N = 9, 65535 * 1024 + 1, 3
    g = F.gen(1)
    at = torch.cat((torch.randint(0, K, (3000,), generator=g, device="cuda"),
                    torch.tensor([0, 1, 1023, 1024, 65534 * 1024 + 1023, 65535 * 1024], device="cuda")))
    x = torch.zeros(T * K, dtype=BF16, device="cuda").view(T, K)  # an odd stride: rows off 16-byte boundaries
    W = torch.zeros(N, K + 7, dtype=BF16, device="cuda")[:, :K]
    x[:, at] = torch.randn(T, len(at), generator=g, device="cuda").to(BF16)
    W[:, at] = torch.randn(N, len(at), generator=g, device="cuda").to(BF16)
    y = sadmm.linear(x, W, out_dtype=FP32)
    assert sadmm.device_status() == 0
    at = at.unique()
    a, b = x[:, at].double(), W[:, at].double()
    assert ((y.double() - a @ b.t()).abs() <= (len(at) + 32) * U32 * (a.abs() @ b.abs().t())).all()
