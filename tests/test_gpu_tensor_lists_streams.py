"""Calls on lists on other streams than the current one, while that one is busy.  (Streams may share a hardware queue, and then one waits for the
other: what is checked holds either way.)"""
from __future__ import annotations

import math

import pytest
import torch

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BUSY = 200_000_000   # cycles: about a tenth of a second


def test_records_made_for_a_call_on_another_stream():
    """The call is ordered behind what the current stream had to do before it, and nothing of its own is left to the current stream."""
    x = torch.full((100_000,), 2.0, device=DEV)
    lst = B.make_tensor_list([x])
    norm = 2.0 * math.sqrt(x.numel())
    side = torch.cuda.Stream()
    for _ in range(3):
        x.fill_(2.0)
        side.wait_stream(torch.cuda.current_stream())
        torch.cuda._sleep(BUSY)
        records = B.normtest_clip_grad_norm(lst, 1.0, stream=side)
        torch.cuda.synchronize()
        r = B.read_norms(records)[0]
        assert abs(r.norm - norm) <= 1e-12 * norm and r.clipped and r.elements == x.numel()
        assert bool(((x - 2.0 / norm).abs() <= 1e-6 * 2.0 / norm).all())


def test_a_list_made_on_another_stream_and_dropped():
    """Its table stays until the call has run, also where the plan was made on the call's stream."""
    x, y = torch.full((50_000,), 2.0, device=DEV), torch.zeros(50_000, device=DEV)
    src = B.make_tensor_list([x])
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        dst = B.make_tensor_list([y], like=src)
    at, size = dst.table.data_ptr(), dst.table.numel()
    B.normtest_accumulate(dst, src, beta=0.0)   # kernels are loaded by their first launch, which takes longer than the wait below
    torch.cuda.synchronize()
    torch.cuda._sleep(BUSY)
    B.normtest_accumulate(dst, src, beta=0.0, scale=0.5)
    del dst
    with torch.cuda.stream(side):
        given = [torch.empty(size, dtype=torch.uint8, device=DEV) for _ in range(64)]
    if not torch.cuda.current_stream().query():   # the call has not run, or not long ago
        assert at not in [t.data_ptr() for t in given]
    torch.cuda.synchronize()
    assert bool((y == 1.0).all())


def test_refresh_behind_a_call_on_another_stream():
    old, new, y = torch.full((50_000,), 2.0, device=DEV), torch.full((50_000,), 3.0, device=DEV), torch.zeros(50_000, device=DEV)
    src = B.make_tensor_list([old])
    dst = B.make_tensor_list([y], like=src)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(BUSY)
        B.normtest_accumulate(dst, src)
    src.refresh([new])
    B.normtest_accumulate(dst, src)
    torch.cuda.synchronize()
    assert bool((y == 5.0).all())


@pytest.mark.parametrize("native", [False, True])
def test_a_tensor_that_is_another_one_at_the_same_address(monkeypatch, native):
    """What the table on the device says no longer holds, so no call takes it, until the list is refreshed."""
    if not native:
        monkeypatch.setattr(B, "_fast", None)
    x, y = torch.full((60, 80), 2.0, device=DEV), torch.zeros(60, 80, device=DEV)
    src = B.make_tensor_list([x])
    dst = B.make_tensor_list([y], like=src)
    for new in (y.data[:30], y.data.view(torch.bfloat16), y.data.view(80, 60), y.data.view(-1).as_strided((60, 80), (1, 60))):
        was, y.data = y.data, new
        with pytest.raises(RuntimeError, match="refresh"):
            B.normtest_accumulate(dst, src)
        y.data = was
        B.normtest_accumulate(dst, src)
    y.data = y.data.view(80, 60)
    B.normtest_accumulate(dst.refresh(), src)
    assert bool((y == 10.0).all())
