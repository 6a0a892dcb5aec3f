"""Results of one quantisation that share memory, on the CPU: refused before anything is enqueued."""
import pytest
import torch
from test_mx_replaced_host import OnDevice, bytes_

from paper_2412_21124_amd import binding as B


@pytest.mark.parametrize("shared", ["matrix", "codes", "scales"])
def test_refused(monkeypatch, shared):
    B.lib()
    monkeypatch.setattr(B, "_call", lambda *a: pytest.fail("enqueued"))
    monkeypatch.setattr(B, "_stream_handle", lambda *a: 0)
    codes, scales = bytes_(32, 32), bytes_(32, 32)
    out = B.MxTensor(codes, scales, 32, B.NT_MX_E4M3)
    out_t = out if shared == "matrix" else B.MxTensor(codes if shared == "codes" else bytes_(32, 32), scales if shared == "scales" else bytes_(32, 32), 32, B.NT_MX_E4M3)
    x = torch.zeros(32, 32).as_subclass(OnDevice)
    for fast in (B._fast, None):
        with monkeypatch.context() as m:
            m.setattr(B, "_fast", fast)
            with pytest.raises(ValueError, match="share memory"):
                B.normtest_mx_quantize(x, out, out_t)


def test_empty_ones_are_taken(monkeypatch):
    called = []
    B.lib()
    monkeypatch.setattr(B, "_call", lambda dev, fn, *a: called.append(fn) or B.NT_OK)
    monkeypatch.setattr(B, "_stream_handle", lambda *a: 0)
    codes, scales = bytes_(0, 32), bytes_(0, 32)
    B.normtest_mx_quantize(torch.zeros(0, 0).as_subclass(OnDevice), B.MxTensor(codes, scales, 0, B.NT_MX_E4M3), B.MxTensor(codes, scales, 0, B.NT_MX_E4M3))
    assert len(called) == 1
