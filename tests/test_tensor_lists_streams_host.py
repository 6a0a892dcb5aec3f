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


@pytest.mark.parametrize("on", [0, 7, 9])
def test_memory_of_lists_that_were_made_on_several_streams(streams, on):
    """A plan of stream 0, lists of streams 0, 7 and 9: whatever stream a call runs on, the tables and the plan are kept until it has run."""
    def make(like=None):
        return B.make_tensor_list([torch.zeros(5), torch.zeros(3)], like=like)
    grads = make()
    lists = {0: [grads, make(grads)]}
    for handle in (7, 9):
        with streams.on(Stream(handle)):
            lists[handle] = [make(grads), make(grads)]
    norms = B.make_norms(grads)
    for a in (0, 7, 9):
        for b in (0, 7, 9):
            x, y, z, u, v = lists[a][0], lists[b][1], lists[b][0], lists[a][1], lists[0][0]
            for call, used in [(lambda **k: B.normtest_grad_norm(x, norms, **k), (x,)), (lambda **k: B.normtest_clip_grads(x, norms, out=y, **k), (x, y)),
                               (lambda **k: B.normtest_accumulate(y, x, **k), (x, y)),
                               (lambda **k: B.normtest_adamw_tensors(x, y, z, u, B.make_hyper(), copy=v, **k), (x, y, z, u, v))]:
                for own in (False, True):   # the current stream, or one that is named
                    streams.held.clear()
                    if own:
                        call(stream=Stream(on))
                    else:
                        with streams.on(Stream(on)):
                            call()
                    assert streams.called[-1] == on
                    for memory in (grads.plan.image, *[lst.table for lst in used]):
                        assert on in streams.kept_for(memory)


def test_the_native_path_is_given_lists_of_their_plans_stream_only(streams, monkeypatch):
    """It keeps no memory for a stream: it takes a call where the plan and every list were made on the call's stream."""
    class Fast:
        def make_list(self, *args):
            return args
    monkeypatch.setattr(B, "_fast", Fast())
    grads = B.make_tensor_list([torch.zeros(5)])
    alike = B.make_tensor_list([torch.zeros(5)], like=grads)
    assert grads.native[-1] == alike.native[-1] == 0
    with streams.on(Stream(7)):
        assert not B.make_tensor_list([torch.zeros(5)], like=grads).native
        grads.refresh()
        assert grads.native[-1] == 0   # its memory is still the first stream's


def test_refresh_waits_for_calls_on_other_streams(streams):
    """The table is written in place (a captured graph reads it there), so it is written behind every call that may still read it."""
    ran = streams.allocations.ran

    class Waiting(Stream):
        def wait_stream(self, other):
            ran.append(("wait", self.cuda_stream, other.cuda_stream))

    def refreshed(lst, on):
        ran.clear()
        with streams.on(Waiting(on)):
            table = lst.table.data_ptr()
            lst.refresh([torch.ones(5)])
            assert lst.table.data_ptr() == table
        at = next(i for i, x in enumerate(ran) if x[0].startswith("aten.copy_"))
        assert all(x[1] == on for x in ran if x[0] == "wait")
        assert not [x for x in ran[at:] if x[0] == "wait"]
        return {x[2] for x in ran if x[0] == "wait"}
    lst = B.make_tensor_list([torch.zeros(5)])
    norms = B.make_norms(lst)
    B.normtest_grad_norm(lst, norms)
    assert refreshed(lst, 0) == set()             # its own stream: in order
    assert refreshed(lst, 5) == {0}
    B.normtest_grad_norm(lst, norms, stream=Stream(7))
    with streams.on(Stream(9)):
        B.normtest_clip_grads(lst, norms)
    assert refreshed(lst, 0) == {7, 9}
    assert refreshed(lst, 0) == set()             # which it has waited for
    with streams.on(Stream(7)):
        other = B.make_tensor_list([torch.zeros(5)], like=lst)
    B.normtest_accumulate(lst, other)
    assert refreshed(other, 7) == {0}             # not what the plan's stream does, but what the list was used on


def changed_in_place():
    """What a program may put at a listed tensor's address: (name, function of a (6, 8) tensor)."""
    def data(new):
        def change(t):
            t.data = new(t.data)
        return change
    return [("shorter", data(lambda x: x[:3])), ("another type", data(lambda x: x.view(torch.bfloat16))),
            ("another type of the same size", data(lambda x: x.view(torch.int32))), ("another shape", data(lambda x: x.view(8, 6))),
            ("other strides", data(lambda x: x.view(-1).as_strided((6, 8), (1, 6)))), ("transposed", lambda t: t.t_()),
            ("resized", lambda t: t.resize_(2, 8))]


@pytest.mark.parametrize("change", [c for _, c in changed_in_place()], ids=[n for n, _ in changed_in_place()])
@pytest.mark.parametrize("native", [False, True])
def test_a_tensor_that_is_another_one_at_the_same_address(streams, monkeypatch, change, native):
    """The table on the device still says what was there: a call would read and write it in the old type and length."""
    monkeypatch.setattr(B, "_fast", B._load_callpath() if native else None)
    t = torch.zeros(6, 8)
    lst = B.make_tensor_list([torch.zeros(5), t])
    like = B.make_tensor_list([torch.zeros(5), torch.zeros(6, 8)], like=lst)
    assert bool(lst.held) == native and lst.unchanged()
    norms = B.make_norms(lst)
    at = t.data_ptr()
    change(t)
    assert t.data_ptr() == at
    hyper = B.make_hyper()
    for call in (lambda: B.normtest_grad_norm(lst, norms), lambda: B.normtest_clip_grads(like, norms, out=lst), lambda: B.normtest_accumulate(like, lst),
                 lambda: B.normtest_accumulate(lst, like), lambda: B.normtest_adamw_tensors(like, like, like, lst, hyper)):
        with pytest.raises(RuntimeError, match="refresh"):
            call()
    assert streams.called == []


def test_no_two_tensors_of_a_list_share_elements(streams):
    """A tied weight that is listed twice would be updated by two blocks at once."""
    flat, wide = torch.zeros(1000), torch.zeros(20, 50)
    a, b = flat[:300], flat[300:]
    apart = [[a, b], [b, a], [a, torch.zeros(0), torch.zeros(0), b], [flat[:0], flat, flat[1000:]], [wide[:, :20], wide[:, 20:]],
             [wide[:, 30:], wide[:, :30], wide[:0]], [wide[:10], wide[10:]], [wide[:10, :20], wide[10:, :20], wide[:, 20:]], [wide[::2], wide[1::2]],
             [wide[:10, 40:], wide[10:, :5]], [wide[:, 3:4], wide[:, 4:5]], [wide.view(-1)[::2], wide.view(-1)[1::2]]]
    shared = [[a, a], [flat, a], [a, torch.zeros(3), flat[299:301]], [flat, flat.view(10, 100)], [flat, flat.view(torch.bfloat16)[1999:]],
              [wide[:, :20], wide[:, 19:]], [wide, wide[3:4, 7:8]], [wide[:, :20], wide.view(-1)[949:952]], [wide[5:, :30], wide[:6, 29:31]],
              [wide[:, 3:4], wide[:, 3:4]], [wide.view(-1)[::2], wide.view(-1)[::2]], [wide[:, :20].t(), wide[0, 19:30]]]
    for tensors in apart:
        B.make_tensor_list(tensors).refresh(tensors[::1])
    for tensors in shared:
        with pytest.raises(ValueError, match="share memory"):
            B.make_tensor_list(tensors)
        lst = B.make_tensor_list([t.clone(memory_format=torch.contiguous_format) for t in tensors])
        if all(t.is_contiguous() for t in tensors):
            with pytest.raises(ValueError, match="share memory"):
                B.make_tensor_list(tensors, like=lst)
            with pytest.raises(ValueError, match="share memory"):
                lst.refresh(tensors)


def test_group_numbers_past_32_bits(streams):
    """They would be another group's in the library's records."""
    for kw in (dict(groups=[1 << 32]), dict(num_groups=(1 << 32) + 1), dict(groups=[(1 << 31) - 1])):
        with pytest.raises(ValueError, match="2\\^31"):
            B.make_tensor_list([torch.zeros(3)], **kw)
