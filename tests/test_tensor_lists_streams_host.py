"""Which stream the memory of lists belongs to and who waits for whom, seen without a GPU: tensors are host tensors, streams are stand-ins that
note what is asked of them, and the library's calls are noted instead of made."""
import contextlib

import pytest
import torch
from torch.utils._python_dispatch import TorchDispatchMode

from paper_2412_21124_amd import binding as B


class Stream:
    def __init__(self, handle):
        self.cuda_stream, self.waited = handle, []

    def wait_stream(self, other):
        self.waited.append(other.cuda_stream)


class Streams:
    """current: torch's current stream; called: the streams that calls were made on; owner: {address: stream that its memory was allocated on};
    held: {address: other streams that it is kept for}."""
    def __init__(self):
        self.current, self.called, self.owner, self.held = Stream(0), [], {}, {}

    @contextlib.contextmanager
    def on(self, stream):
        before, self.current = self.current, stream
        yield
        self.current = before

    def kept_for(self, tensor):
        """Streams whose work may still use the memory when the tensor is dropped."""
        return {self.owner[tensor.data_ptr()], *self.held.get(tensor.data_ptr(), [])}


class Allocations(TorchDispatchMode):
    """Notes whose memory a tensor is, and what else is run: (operator, current stream)."""
    def __init__(self, streams):
        super().__init__()
        self.streams, self.ran = streams, []

    def __torch_dispatch__(self, func, types, args=(), kwargs=None):
        out = func(*args, **(kwargs or {}))
        if str(func).startswith(("aten.empty", "aten.zeros")):
            self.streams.owner[out.data_ptr()] = self.streams.current.cuda_stream
        if not str(func).startswith("aten.empty"):
            self.ran.append((str(func), self.streams.current.cuda_stream))
        return out


@pytest.fixture
def streams(monkeypatch):
    s = Streams()
    B.lib()
    monkeypatch.setattr(B, "_fast", None)
    monkeypatch.setattr(B, "_check_listed", lambda tensors, device: None)
    monkeypatch.setattr(B, "_stream_handle", lambda stream, dev: (stream or s.current).cuda_stream)
    monkeypatch.setattr(B, "_call", lambda dev, fn, *args: s.called.append(args[-1]) or B.NT_OK)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: s.current)
    monkeypatch.setattr(torch.cuda, "stream", s.on)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda t, stream: s.held.setdefault(t.data_ptr(), []).append(stream.cuda_stream))
    with Allocations(s) as s.allocations:
        yield s


def test_records_made_for_a_call_on_another_stream(streams):
    """The call's stream does not wait for the current one: the records are its own memory, which nothing on the current stream writes, and are
    kept for both."""
    lst = B.make_tensor_list([torch.zeros(5), torch.zeros(3)], groups=[0, 1])
    side = Stream(7)
    for call in (lambda: B.normtest_grad_norm(lst, stream=side), lambda: B.normtest_clip_grad_norm(lst, 1.0, stream=side)):
        streams.called.clear()
        streams.allocations.ran.clear()
        norms = call()
        assert set(streams.called) == {7} and not [x for x in streams.allocations.ran if x[1] != 7]
        assert norms.dtype == torch.uint8 and norms.numel() == 2 * B.NORM_BYTES
        assert streams.owner[norms.data_ptr()] == 7 and streams.kept_for(norms) == {0, 7}
    assert streams.kept_for(B.normtest_grad_norm(lst)) == {0}
