"""A microscaled matrix whose tensors take other memory or another shape: every call on it raises, through either call path, and writes nothing."""
import pytest
import torch

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


def square():
    codes = torch.full((64, 64), 0x38, dtype=torch.uint8, device=DEV)
    return B.MxTensor(codes, torch.full((64, 64), 127, dtype=torch.uint8, device=DEV), 64, B.NT_MX_E4M3)


CHANGES = {"turned": lambda t: t.t_(), "fewer rows": lambda t: t.resize_(32, 64), "fewer columns": lambda t: t.as_strided_((64, 32), (64, 1)),
           "rows nearer": lambda t: t.as_strided_((64, 64), (32, 1)), "other memory": lambda t: t.set_(torch.zeros_like(t)),
           "other memory behind it": lambda t: setattr(t, "data", torch.zeros_like(t)), "another dimension": lambda t: t.unsqueeze_(0)}


@pytest.mark.parametrize("path", ["native", "python"])
@pytest.mark.parametrize("which", ["codes", "scales"])
@pytest.mark.parametrize("change", CHANGES)
def test_every_call_raises(monkeypatch, path, which, change):
    B.lib()
    m, other = square(), square()
    assert m.native
    x, out = torch.ones(64, 64, device=DEV), torch.full((64, 64), 7.0, device=DEV)
    kept = m.codes.untyped_storage(), m.scales.untyped_storage()   # the memory that it was made of
    before = [torch.tensor([], dtype=torch.uint8, device=DEV).set_(k).clone() for k in kept]
    CHANGES[change](getattr(m, which))
    if path == "python":
        monkeypatch.setattr(B, "_fast", None)
    for call in (lambda: B.normtest_mx_quantize(x, m), lambda: B.normtest_mx_quantize(x, None, m), lambda: B.normtest_mx_dequantize(m, out),
                 lambda: B.normtest_mx_matmul(m, other, out), lambda: B.normtest_mx_matmul(other, m, out), lambda: B.normtest_rms_norm(x, None, out_mx=m),
                 lambda: B.normtest_mx_matmul(m, other, out, full_sums=True)):
        with pytest.raises(RuntimeError, match="other memory or another shape"):
            call()
    assert (out == 7.0).all()
    assert all(torch.equal(torch.tensor([], dtype=torch.uint8, device=DEV).set_(k), b) for k, b in zip(kept, before))


def test_bytes_may_change():
    m, other = square(), square()
    out = torch.empty(64, 64, device=DEV)
    B.normtest_mx_matmul(m, other, out)
    assert (out == 64.0).all()
    m.scales.fill_(128)
    m.codes[0] = 0
    B.normtest_mx_matmul(m, other, out)
    assert (out[0] == 0).all() and (out[1:] == 128.0).all()
    with pytest.raises(AttributeError, match="make another"):
        m.scales = m.scales.clone()
    B.normtest_mx_quantize(torch.zeros(64, 64, device=DEV), m)
    assert not m.codes.any()
