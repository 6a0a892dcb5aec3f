"""Results of one quantisation that share memory: refused through either call path, with nothing written; different matrices are taken."""
import pytest
import torch
from test_gpu_mx import DEV

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("path", ["native", "python"])
def test_refused(monkeypatch, path):
    B.lib()
    if path == "python":
        monkeypatch.setattr(B, "_fast", None)
    x, a, b = torch.ones(32, 32, device=DEV), B.make_mx(32, 32, B.NT_MX_E4M3, DEV), B.make_mx(32, 32, B.NT_MX_E4M3, DEV)
    for out, out_t in ((a, a), (a, B.MxTensor(a.codes, b.scales, 32, B.NT_MX_E4M3)), (B.MxTensor(b.codes, a.scales, 32, B.NT_MX_E4M3), a)):
        with pytest.raises(ValueError, match="share memory"):
            B.normtest_mx_quantize(x, out, out_t)
    assert not a.codes.any() and not b.codes.any() and not a.scales.any()
    B.normtest_mx_quantize(x, a, b)
    assert a.codes.all() and torch.equal(a.codes, b.codes)
