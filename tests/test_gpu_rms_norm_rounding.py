"""The RMS norm's roundings: its result once to fp32, and from there to the type and to codes."""
import mx_reference as R
import numpy as np
import pytest
import torch
from test_gpu_mx import DEV, FORMS, TYPES, matrix
from test_gpu_rms_norm import EPS, SHAPES, STEP

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES + [(300, 700)], ids=str)
def test_forward(rows, cols, dtype):
    t = TYPES[dtype]
    half = torch.finfo(t).eps / 2
    x, r = matrix(rows, cols, t, cols, pad=3), matrix(rows, cols, t, cols + 1)
    w = 1 + 0.1 * torch.randn(cols, device=DEV)
    for weight, form, fit in ((w, "e4m3", False), (None, "e2m1", True), (w, "e2m1", False), (w, "e4m3", True)):
        h, out, rstd = torch.empty_like(x), torch.empty_like(x), torch.empty(rows, device=DEV)
        mx = B.make_mx(rows, cols, FORMS[form], DEV)
        B.normtest_rms_norm(x, weight, out, residual=r, eps=EPS, sum_out=h, out_mx=mx, rstd=rstd, fit=fit)
        # the same rows in fp32: the squares' order is the shape's, so that rstd and the result are the same numbers
        y, again = torch.empty(rows, cols, device=DEV), torch.empty(rows, device=DEV)
        B.normtest_rms_norm(h.float(), weight, y, eps=EPS, rstd=again)
        assert torch.equal(rstd, again)
        assert torch.equal(out, y.to(t))
        grid, scales = R.quantize(R.wide(y), FORMS[form], fit)
        blocks = scales.shape[1]
        assert np.array_equal(mx.scales.cpu().numpy()[:, :blocks], scales)
        assert np.array_equal(R.decode(mx.codes.cpu().numpy()[:, :blocks * R.BYTES[mx.format]], mx.format), grid)
        # and how far all of it is from 64 bits.  A square is exact in fp64, and its sum's additions of 2^-53 each, at most 32768 of them, are 2^-38; the reciprocal
        # root is then off by half a step, and the result by another one of its own, 2^-40 for what the second words leave
        wide = R.wide(h)
        exact = 1 / np.sqrt((wide ** 2).mean(1) + np.float32(EPS))
        assert (np.abs(R.wide(rstd) - exact) <= STEP * exact * (1 + 2.0 ** -12)).all()
        want = wide * exact[:, None] * (R.wide(w) if weight is not None else 1.0)
        off = STEP * np.abs(want) * (1 + 2.0 ** -12)
        assert (np.abs(R.wide(y) - want) <= off).all()
        assert (np.abs(R.wide(out) - want) <= off + half * (np.abs(want) + off) + (2.0 ** -25 if dtype == "f16" else 0)).all()
