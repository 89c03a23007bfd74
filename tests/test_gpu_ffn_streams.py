"""Calls on a stream that is not torch's current one: no block of memory that another
stream's pending kernels use is handed to the call, and none that the call uses or
returns is handed out while it is in use.  Work is kept pending by a sleeping kernel
in front of it."""
import pytest
import torch

import _ffn as F

pytestmark = pytest.mark.gpu

SLEEP = 200_000_000  # cycles, some 100 ms


def lib():
    from paper_1807_11091_gb300 import sadmm
    return sadmm


def problem():
    g = F.gen(1)
    x, W = F.matrix(g, 1000, 515), F.matrix(g, 2048, 515, scale=0.05)  # odd rows: the call has scratch for both
    return x, W


def warm(side):
    """Both streams' pools empty, the kernels loaded."""
    x, W = problem()
    lib().linear(x, W)
    lib().linear(x, W, stream=side)
    torch.cuda.synchronize()
    del x, W
    torch.cuda.empty_cache()


def test_freed_memory_of_the_current_stream_is_not_taken():
    s, side = lib(), torch.cuda.Stream()
    warm(side)
    x, W = problem()
    ref = s.linear(x, W)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    # blocks of the output's and the scratch's sizes, written late by the current stream; the given stream has had
    # its own, so that the call need not ask the device for memory, which waits for the device
    a = torch.empty(1000 * 2048 * 2, dtype=torch.uint8, device="cuda")
    b = torch.empty((1000 + 2048) * 520 * 2, dtype=torch.uint8, device="cuda")
    at, done = a.data_ptr(), torch.cuda.Event()
    s.linear(x, W, stream=side)
    a.fill_(0), b.fill_(0)  # (a kernel's first launch may wait for the device too)
    torch.cuda._sleep(1)
    torch.cuda.synchronize()
    torch.cuda._sleep(SLEEP)
    a.fill_(255), b.fill_(255)
    done.record()
    del a, b
    y = s.linear(x, W, stream=side)
    side.synchronize()
    assert not done.query()  # the call did not wait for the current stream either
    assert y.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(y, ref) and s.device_status() == 0


def test_inputs_freed_early_are_kept_for_the_given_stream():
    s, side = lib(), torch.cuda.Stream()
    warm(side)
    x, W = problem()
    ref = s.linear(x, W)
    torch.cuda.synchronize()
    at, size = x.untyped_storage().data_ptr(), x.untyped_storage().nbytes()
    with torch.cuda.stream(side):
        torch.cuda._sleep(SLEEP)
    y = s.linear(x, W, stream=side)
    del x
    z = torch.empty(size, dtype=torch.uint8, device="cuda")
    assert z.data_ptr() != at
    z.fill_(255)
    torch.cuda.synchronize()
    assert torch.equal(y, ref) and s.device_status() == 0


def test_outputs_freed_early_are_kept_for_the_current_stream():
    s, side = lib(), torch.cuda.Stream()
    warm(side)
    x, W = problem()
    ref = s.linear(x, W)
    torch.cuda.synchronize()
    y = s.linear(x, W, stream=side)
    at = y.data_ptr()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda._sleep(SLEEP)
    copy = y.clone()
    del y
    again = s.linear(x, W, stream=side)
    assert again.data_ptr() != at
    torch.cuda.synchronize()
    assert torch.equal(copy, ref) and torch.equal(again, ref) and s.device_status() == 0


@pytest.mark.parametrize("given", ["same", "default"])
def test_the_current_or_default_stream_by_name(given):
    s = lib()
    x, W = problem()
    ref = s.linear(x, W)
    torch.cuda.synchronize()
    name = torch.cuda.current_stream() if given == "same" else torch.cuda.default_stream()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side if given == "default" else name):
        y = s.linear(x, W, stream=name)
    torch.cuda.synchronize()
    assert torch.equal(y, ref)


def test_an_argument_that_is_not_read_may_lie_anywhere():
    """z without an activation is ignored, on a given stream too."""
    s, side = lib(), torch.cuda.Stream()
    g = F.gen(2)
    dy, x, W = F.matrix(g, 40, 64), F.matrix(g, 40, 128), F.matrix(g, 64, 128)
    want = s.linear_backward(dy, x, W)
    side.wait_stream(torch.cuda.current_stream())
    got = s.linear_backward(dy, x, W, z=torch.zeros(3), stream=side)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and s.device_status() == 0
