"""Random rounding in the 64-bit reference: its mean over all bytes is the element where nothing is clamped, and the largest code where it is."""
import mx_reference as R
import numpy as np
import pytest

ALL = np.arange(256)[:, None]


def mean(row, form, fit):
    """Over the 256 bytes, of a row of elements (each with the same byte)."""
    rows = np.repeat(np.array([row]), 256, 0)
    return R.quantized(rows, form, fit, np.repeat(ALL, len(row), 1)).mean(0)


@pytest.mark.parametrize("form,top", [(R.E2M1, 7.9), (R.E2M1, 6.01), (R.E2M1, 4.0), (R.E4M3, 1.99 * 256), (R.E4M3, 449.0), (R.E4M3, 256.0)])
def test_mean(form, top):
    row = [top, -top, 0.7 * top, -0.31 * top, 0.11 * top]
    grid = R.GRID[form]
    unit = 2.0 if top > grid[-1] else 1.0              # of the scale that fits; without fit it is 1
    step = np.array([np.diff(grid)[min(np.searchsorted(grid, abs(v) / unit, side="right") - 1, len(grid) - 2)] for v in row]) * unit
    assert (np.abs(mean(row, form, True) - row) <= step / 512 * (1 + 1e-12)).all()
    got = mean(row, form, False)
    clamped = np.abs(row) > grid[-1]
    assert (got[clamped] == np.sign(np.array(row))[clamped] * grid[-1]).all()
    step = np.array([np.diff(grid)[min(np.searchsorted(grid, abs(v), side="right") - 1, len(grid) - 2)] for v in row])
    assert (np.abs(got - row) <= step / 512 * (1 + 1e-12))[~clamped].all()


def test_how_much_is_lost():
    assert abs(mean([7.9], R.E2M1, False)[0] / 7.9 - 6 / 7.9) < 1e-15 and abs(mean([1.99 * 256], R.E4M3, False)[0] / (1.99 * 256) - 448 / (1.99 * 256)) < 1e-15
    for form, most in ((R.E2M1, 0.25), (R.E4M3, 0.125)):      # up to a quarter and an eighth
        top = 2.0 ** (R.TOP[form] + 1) * (1 - 2.0 ** -20)
        assert most - 1e-5 < 1 - mean([top], form, False)[0] / top < most
