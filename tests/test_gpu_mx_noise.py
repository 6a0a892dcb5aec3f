"""Random rounding on the GPU, over all 256 bytes: without bias where nothing is clamped, which `fit` sees to; both directions."""
import itertools

import mx_reference as R
import numpy as np
import pytest
import torch
from test_gpu_mx import DEV, FORMS, TYPES

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("form,dtype", itertools.product(FORMS, TYPES))
def test_mean(form, dtype):
    grid = R.GRID[FORMS[form]]
    tops = [2.0 ** R.TOP[FORMS[form]] * x for x in (1.0, 1.25, 1.5, 1.51, 1.75, 1.77, 1.9921875)]
    row = torch.tensor([[top * share for share in (1.0, -1.0, 0.9, -0.55, 0.3, 0.07, 0.003)] + [0.0] * 25 for top in tops], device=DEV).to(TYPES[dtype]).reshape(1, -1)
    x = row.repeat(256, 1)
    noise = torch.arange(256, dtype=torch.uint8, device=DEV)[:, None].repeat(1, x.shape[1])
    wide = R.wide(row)[0]
    for fit in (True, False):
        mx = B.make_mx(*x.shape, FORMS[form], DEV)
        B.normtest_mx_quantize(x, mx, fit=fit, noise=noise)
        scale = np.repeat(np.exp2(mx.scales.cpu().numpy()[0, :len(tops)].astype(float) - 127), 32)
        a = np.abs(wide) / scale
        clamped = a > grid[-1]
        assert clamped.any() == (not fit)
        step = np.diff(grid)[np.minimum(np.searchsorted(grid, a, side="right") - 1, len(grid) - 2)] * scale
        mean = R.numbers(mx).mean(0)
        assert (np.abs(mean - wide) <= step / 512 * (1 + 1e-12))[~clamped].all()
        assert (mean == np.sign(wide) * grid[-1] * scale)[clamped].all()
        # the transpose: a column for every byte, so a block has the same element 32 times; its means are over eight blocks
        column = row[0, :7].repeat_interleave(256)[:, None].contiguous()
        turned = B.make_mx(1, column.shape[0], FORMS[form], DEV)
        B.normtest_mx_quantize(column, None, turned, fit=fit, noise=torch.arange(256, dtype=torch.uint8, device=DEV).repeat(7)[:, None].contiguous())
        scale = np.exp2(turned.scales.cpu().numpy()[0, ::8][:7].astype(float) - 127)
        a = np.abs(wide[:7]) / scale
        step = np.diff(grid)[np.minimum(np.searchsorted(grid, a, side="right") - 1, len(grid) - 2)] * scale
        mean = R.numbers(turned).reshape(7, 256).mean(1)
        assert (np.abs(mean - wide[:7]) <= step / 512 * (1 + 1e-12))[a <= grid[-1]].all()
