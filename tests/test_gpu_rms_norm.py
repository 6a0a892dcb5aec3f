"""The RMS norm with the residual's addition and its backward pass on the GPU against 64-bit references."""
import itertools

import mx_reference as R
import numpy as np
import pytest
import torch
from test_gpu_mx import DEV, FORMS, TYPES, matrix

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu

EPS = 1e-5
STEP = 2.0 ** -24            # half a step of fp32
SHAPES = [(1, 1), (1, 5), (3, 31), (2, 64), (5, 512), (7, 513), (4, 768), (9, 1024), (3, 1111), (2, 2048), (2, 2049), (5, 4096), (2, 5003), (3, 8192),
          (1, 8200), (2, 16384), (2, 16391), (1, 32768)]


def adds(cols):
    """Additions on the way to a row's sum: a thread's own elements, then lanes and waves."""
    return min(cols, 40) + 6 + 16


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES, ids=str)
def test_forward(rows, cols, dtype):
    t = TYPES[dtype]
    half = torch.finfo(t).eps / 2
    for k, (form, fit, residual, weighted) in enumerate([("e4m3", False, True, True), ("e2m1", True, True, True), ("e4m3", True, False, True), ("e2m1", False, True, False)]):
        x = matrix(rows, cols, t, 10 * cols + k, pad=(0, 3, 8, 1)[k])
        r = matrix(rows, cols, t, 20 * cols + k, pad=(1, 0, 8, 3)[k]) if residual else None
        w = 1 + 0.1 * torch.randn(cols, device=DEV) if weighted else None
        total = torch.full((rows, cols + 4), 7.0, dtype=t, device=DEV)
        out, rstd = torch.full_like(total, 7.0), torch.empty(rows, device=DEV)
        mx = B.make_mx(rows, cols, FORMS[form], DEV)
        B.normtest_rms_norm(x, w, out[:, :cols], residual=r, eps=EPS, sum_out=total[:, :cols], out_mx=mx, rstd=rstd, fit=fit)
        assert (total[:, cols:] == 7.0).all() and (out[:, cols:] == 7.0).all()
        h = total[:, :cols]
        # the sum in fp32, rounded to the type
        want = (x.float() + r.float()).to(t) if residual else x
        assert torch.equal(h, want)
        wide = R.wide(h)
        exact = 1 / np.sqrt((wide ** 2).mean(1) + EPS)
        # the squares' sum is off by a half step for each addition, of which the root halves the effect; quotient, root, reciprocal, eps
        far = (adds(cols) / 2 + 4) * STEP
        assert (np.abs(R.wide(rstd) - exact) <= far * exact).all()
        y = wide * exact[:, None] * (R.wide(w) if weighted else 1.0)
        off = (far + 3 * STEP) * np.abs(y)
        assert (np.abs(R.wide(out[:, :cols]) - y) <= off + half * (np.abs(y) + off) + (6e-8 if dtype == "f16" else 0)).all()
        # in codes: those of y, or of what y may be off by
        got = R.numbers(mx)
        allowed = [R.quantized(y * (1 + d), FORMS[form], fit) for d in (0.0, far + 3 * STEP, -far - 3 * STEP)]
        assert np.logical_or.reduce([got == a for a in allowed]).all()
        behind = R.decode(mx.codes.cpu().numpy(), mx.format).reshape(rows, -1)[:, cols:]
        assert not behind.any()


def test_forward_in_place_and_alone():
    x, r, w = matrix(6, 777, torch.bfloat16, 1), matrix(6, 777, torch.bfloat16, 2), torch.rand(777, device=DEV)
    want, out = torch.empty_like(x), torch.empty_like(x)
    B.normtest_rms_norm(x, w, out, residual=r, sum_out=want)
    for to in (x.clone(), r.clone()):
        a, b = (to, r) if torch.equal(to, x) else (x, to)
        again = torch.empty_like(out)
        B.normtest_rms_norm(a, w, again, residual=b, sum_out=to)
        assert torch.equal(to, want) and torch.equal(again, out)
    total = torch.empty_like(x)
    B.normtest_rms_norm(x, None, residual=r, sum_out=total)         # the sum alone
    assert torch.equal(total, want)
    rstd = torch.empty(6, device=DEV)
    B.normtest_rms_norm(x, None, rstd=rstd)
    assert torch.isfinite(rstd).all()
    B.normtest_rms_norm(torch.empty(0, 64, device=DEV), None, torch.empty(0, 64, device=DEV))


def test_forward_of_zeros_nan_and_infinity():
    x = torch.ones(4, 100, device=DEV)
    x[0] = 0
    x[1, 70] = float("nan")
    x[2, 3] = float("inf")
    out, rstd, mx = torch.empty_like(x), torch.empty(4, device=DEV), B.make_mx(4, 100, B.NT_MX_E4M3, DEV)
    B.normtest_rms_norm(x, None, out, out_mx=mx, rstd=rstd, eps=1e-6)
    assert (out[0] == 0).all() and abs(rstd[0].item() - 1000.0) <= 1000.0 * 8 * STEP
    assert torch.isnan(out[1]).all() and torch.isnan(rstd[1])
    assert rstd[2] == 0 and torch.isnan(out[2, 3]) and (out[2, :3] == 0).all()      # 1 / inf; inf 0 is NaN
    got = R.numbers(mx)
    assert not got[0].any() and np.isnan(got[1]).all() and np.isnan(got[2, :32]).all() and not got[2, 32:].any()
    assert R.decode(mx.codes.cpu().numpy(), mx.format)[:, 3, 4:].any() == False       # noqa: E712  behind the last column


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("cols", [5, 700, 5003, 20000])
def test_forward_at_the_ends_of_the_range(cols, dtype):
    """Rows whose squares no fp32 holds."""
    t = TYPES[dtype]
    half = torch.finfo(t).eps / 2
    size = torch.tensor([1e30, 3e19, 5e-20, 1e-21, 2.0 ** 124], device=DEV)[:, None]
    x = ((torch.rand(5, cols, device=DEV) + 0.5) * size).to(t)
    out, rstd, eps = torch.empty_like(x), torch.empty(5, device=DEV), float(np.float32(1e-41))
    B.normtest_rms_norm(x, None, out, rstd=rstd, eps=eps)
    wide = R.wide(x)
    exact = 1 / np.sqrt((wide ** 2).mean(1) + eps)
    # the sum's rounding to fp32 (halved by the root), root, reciprocal (each correct to a step); the smallest rstd is 2^-125
    far = (0.5 + 2 + 2) * STEP
    assert (np.abs(R.wide(rstd) - exact) <= far * exact).all()
    y = wide * exact[:, None]
    off = (far + 2 * STEP) * y
    assert (np.abs(R.wide(out) - y) <= off + half * (y + off)).all()


@pytest.mark.parametrize("cols", [3, 768, 4096, 20000])
def test_forward_rounds_once(cols):
    gen = torch.Generator().manual_seed(cols)
    x, w = torch.randn(64, cols, generator=gen).to(DEV), (1 + 0.1 * torch.randn(cols, generator=gen)).to(DEV)
    for weight in (w, None):
        out, rstd = torch.empty_like(x), torch.empty(64, device=DEV)
        B.normtest_rms_norm(x, weight, out, rstd=rstd, eps=EPS)
        wide = R.wide(x)
        exact = 1 / np.sqrt((wide ** 2).mean(1) + np.float32(EPS))
        # half a step each, and 2^-40 for what the second words leave
        assert (np.abs(R.wide(rstd) - exact) <= STEP * exact * (1 + 2.0 ** -16)).all()
        y = wide * exact[:, None] * (R.wide(w) if weight is not None else 1.0)
        assert (np.abs(R.wide(out) - y) <= STEP * np.abs(y) * (1 + 2.0 ** -16)).all()
    w[1] = float("inf")
    w[2] = 0
    out = torch.empty_like(x)
    B.normtest_rms_norm(x, w, out)
    assert torch.equal(out[:, 1], torch.sign(x[:, 1]) * float("inf")) and (out[:, 2] == 0).all()


def reference_backward(dy, h, w, rstd, dsum):
    hat = h * rstd[:, None]
    g = dy * w
    inner = (g * hat).mean(1, keepdims=True)
    dx = rstd[:, None] * (g - hat * inner) + dsum
    size = rstd[:, None] * (np.abs(g) + np.abs(hat) * np.abs(g * hat).mean(1, keepdims=True)) + np.abs(dsum)
    return dx, size, (dy * hat).sum(0), np.abs(dy * hat).sum(0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols", SHAPES + [(700, 96), (600, 800), (2500, 130), (550, 2500)], ids=str)
def test_backward(rows, cols, dtype):
    t = TYPES[dtype]
    half = torch.finfo(t).eps / 2
    for k, (with_sum, weighted, beta, scale) in enumerate([(True, True, 1.0, 0.5), (False, True, 0.0, 1.0), (True, False, -0.5, 2.0)]):
        h, dy = matrix(rows, cols, t, 3 * cols + k, pad=(0, 3, 8)[k]), matrix(rows, cols, t, 5 * cols + k, pad=(1, 0, 8)[k])
        dsum = matrix(rows, cols, t, 7 * cols + k) if with_sum else None
        w = 1 + 0.1 * torch.randn(cols, device=DEV) if weighted else None
        rstd = (R.wide(h) ** 2).mean(1)
        rstd = torch.from_numpy(1 / np.sqrt(rstd + EPS)).float().to(DEV)
        dx = torch.full((rows, cols + 4), 7.0, dtype=t, device=DEV)
        dw = torch.randn(cols, device=DEV)
        before = R.wide(dw)
        if beta == 0.0:
            dw.fill_(float("nan"))
        B.normtest_rms_norm_backward(dy, h, w, rstd, dx[:, :cols], dsum=dsum, dweight=dw, scale=scale, beta=beta)
        assert (dx[:, cols:] == 7.0).all()
        want, size, want_w, size_w = reference_backward(R.wide(dy), R.wide(h), R.wide(w) if weighted else 1.0, R.wide(rstd), R.wide(dsum) if with_sum else 0.0)
        off = (adds(cols) + 8) * STEP * size
        assert (np.abs(R.wide(dx[:, :cols]) - want) <= off + half * (np.abs(want) + off) + (6e-8 if dtype == "f16" else 0)).all()
        # a column's sum: rows one after the other in a block, of which there are 256 or 512 (with up to 8 rows at a time), then those
        serial = -(-rows // 256) + 8 + 32 + 16
        off = serial * STEP * (scale * size_w + np.abs(beta * before))
        assert (np.abs(R.wide(dw) - (scale * want_w + beta * before)) <= off).all()
        # either alone gives the same bits, dx in place of dy or dsum too
        alone = torch.empty_like(h)
        B.normtest_rms_norm_backward(dy, h, w, rstd, alone, dsum=dsum)
        assert torch.equal(alone, dx[:, :cols])
        again = torch.from_numpy(before).float().to(DEV)
        B.normtest_rms_norm_backward(dy, h, w, rstd, dweight=again, scale=scale, beta=beta)
        assert torch.equal(again, dw)
        over = dy.clone()
        B.normtest_rms_norm_backward(over, h, w, rstd, over, dsum=dsum)
        assert torch.equal(over, alone)
        if with_sum:
            over = dsum.clone()
            B.normtest_rms_norm_backward(dy, h, w, rstd, over, dsum=over)
            assert torch.equal(over, alone)


def test_backward_against_differences():
    """The derivative along a direction of sum(dy y) + sum(dsum h), from differences of the 64-bit forward pass."""
    rows, cols = 5, 300
    rng = np.random.default_rng(0)
    x, dy, dsum, v = (rng.standard_normal((rows, cols)) for _ in range(4))
    w, vw = 1 + 0.1 * rng.standard_normal(cols), rng.standard_normal(cols)

    def loss(x, w):
        return (dy * (x / np.sqrt((x ** 2).mean(1, keepdims=True) + EPS) * w)).sum() + (dsum * x).sum()
    step = 1e-5
    along_x = (loss(x + step * v, w) - loss(x - step * v, w)) / (2 * step)
    along_w = (loss(x, w + step * vw) - loss(x, w - step * vw)) / (2 * step)
    to = lambda a: torch.from_numpy(a).float().to(DEV)   # noqa: E731
    rstd, dx, dw = torch.empty(rows, device=DEV), torch.empty(rows, cols, device=DEV), torch.empty(cols, device=DEV)
    B.normtest_rms_norm(to(x), to(w), rstd=rstd, eps=EPS)
    B.normtest_rms_norm_backward(to(dy), to(x), to(w), rstd, dx, dsum=to(dsum), dweight=dw)
    # inputs rounded to fp32 and sums of 1500 terms of size about 1: 1e-6 relative to the sum of magnitudes; differences: step^2 and 1e-16 / step
    assert abs((R.wide(dx) * v).sum() - along_x) <= 1e-6 * np.abs(R.wide(dx) * v).sum() + 1e-6
    assert abs((R.wide(dw) * vw).sum() - along_w) <= 1e-6 * np.abs(R.wide(dw) * vw).sum() + 1e-6


def test_backward_without_rows():
    dw = torch.ones(50, device=DEV)
    e = torch.empty(0, 50, device=DEV)
    B.normtest_rms_norm_backward(e, e, None, torch.empty(0, device=DEV), e, dweight=dw, beta=0.5)
    assert (dw == 0.5).all()
