"""CPU checks of the calls on microscaled matrices and of the RMS norm: arguments are refused before the GPU is touched, and the 64-bit
reference that the GPU tests use agrees with torch's own 8-bit type."""
import ctypes

import mx_reference as R
import numpy as np
import pytest
import torch

from paper_2412_21124_amd import binding as B

OK, BAD, UNSUPPORTED, SMALL, LARGE = B.NT_OK, B.NT_ERR_BAD_ARG, B.NT_ERR_UNSUPPORTED, B.NT_ERR_WORKSPACE_TOO_SMALL, B.NT_ERR_TOO_LARGE


def mx(rows, cols, format=B.NT_MX_E2M1, /, **over):
    """A record with fabricated addresses: only for calls that are refused, or have nothing to do."""
    blocks = -(-cols // 32)
    fields = dict(codes=0x10000, scales=0x20000, rows=rows, cols=cols, ld=blocks * (16 if format == B.NT_MX_E2M1 else 32), scale_ld=blocks,
                  format=format, reserved=0)
    fields.update(over)
    return B.nt_mx(*[fields[k] for k, _ in B.nt_mx._fields_])


BAD_MX = [dict(codes=0), dict(scales=0), dict(codes=0x10008), dict(ld=8), dict(ld=40), dict(scale_ld=1), dict(rows=-1), dict(cols=-1), dict(reserved=1)]


def quantize(rows=4, cols=100, *, src=0x1000, dtype=B.NT_F32, ld=100, noise=None, noise_ld=0, out=(), out_t=None, flags=0):
    out = mx(rows, cols) if out == () else out
    return B.lib().normtest_mx_quantize(src, dtype, rows, cols, ld, noise, noise_ld, out, out_t, flags, None)


@pytest.mark.parametrize("over", BAD_MX, ids=str)
def test_bad_matrices(over):
    bad = mx(4, 100, **over)
    assert quantize(out=bad) == BAD
    assert B.lib().normtest_mx_dequantize(bad, 0x1000, B.NT_F32, 100, None) == BAD
    assert product(a=bad) == BAD and product(b=bad, ld=4) == BAD
    assert norm(out_mx=bad, rows=4, cols=100) == BAD


def test_formats_and_types():
    for code in (-1, 2, 7):
        assert quantize(out=mx(4, 100, B.NT_MX_E2M1, format=code, ld=64)) == UNSUPPORTED
        assert product(a=mx(4, 100, B.NT_MX_E2M1, format=code, ld=64)) == UNSUPPORTED
    for dtype in (-1, 3):
        assert quantize(dtype=dtype) == UNSUPPORTED and product(dtype=dtype) == UNSUPPORTED and norm(dtype=dtype) == UNSUPPORTED
        assert backward(dtype=dtype) == UNSUPPORTED
        assert B.lib().normtest_mx_dequantize(mx(4, 100), 0x1000, dtype, 100, None) == UNSUPPORTED


def test_quantize():
    assert quantize(src=None) == BAD and quantize(src=0x1002) == BAD and quantize(ld=99) == BAD
    assert quantize(out=None) == BAD and quantize(flags=2) == BAD
    assert quantize(out=mx(4, 96)) == BAD and quantize(out=mx(5, 100)) == BAD and quantize(out_t=mx(4, 100)) == BAD
    assert quantize(noise=0x3000, noise_ld=99) == BAD
    assert quantize(rows=-1) == BAD and quantize(cols=-1) == BAD
    assert quantize(rows=1 << 40, ld=1 << 40, out=mx(1 << 40, 100)) == LARGE
    # nothing to do: no launch, whatever the addresses
    assert quantize(rows=0, src=None, out=mx(0, 100, codes=0, scales=0)) == OK
    assert quantize(cols=0, src=None, out=mx(4, 0, codes=0, scales=0)) == OK
    assert B.lib().normtest_mx_dequantize(None, 0x1000, B.NT_F32, 100, None) == BAD
    assert B.lib().normtest_mx_dequantize(mx(4, 100), 0x1000, B.NT_F32, 99, None) == BAD
    assert B.lib().normtest_mx_dequantize(mx(0, 100), None, B.NT_F32, 0, None) == OK


def product(M=4, N=8, K=100, *, a=None, b=None, scale=1.0, beta=0.0, out=0x1000, dtype=B.NT_F32, ld=8, workspace=None, size=0):
    a = mx(M, K) if a is None else a
    b = mx(N, K) if b is None else b
    return B.lib().normtest_mx_matmul(a, b, scale, beta, out, dtype, ld, workspace, size, None)


def test_product():
    L = B.lib()
    assert L.normtest_mx_matmul(None, mx(8, 100), 1.0, 0.0, 0x1000, 0, 8, None, 0, None) == BAD
    assert product(out=None) == BAD and product(out=0x1001) == BAD and product(ld=7) == BAD and product(b=mx(8, 101)) == BAD
    for x in (float("nan"), float("inf"), 1e300):
        assert product(scale=x) == BAD and product(beta=x) == BAD
    assert product(K=(1 << 22) + 1) == LARGE and product(M=1 << 31) == LARGE
    assert product(M=0, a=mx(0, 100, codes=0, scales=0), out=None) == OK and product(N=0, b=mx(0, 100), out=None) == OK
    # a product that needs a workspace asks for it
    need = L.normtest_mx_matmul_workspace_bytes(64, 64, 1 << 20, B.NT_MX_E2M1, B.NT_MX_E2M1, B.NT_BF16)
    assert need > 0 and need % (64 * 64 * 4) == 0
    long = dict(M=64, N=64, K=1 << 20, dtype=B.NT_BF16, ld=64)
    assert product(**long) == SMALL and product(**long, workspace=0x8000, size=need - 1) == SMALL and product(**long, workspace=0x8008, size=need) == BAD
    for sizes in ((0, 5, 5), (5, 0, 5), (5, 5, 0), (-1, 5, 5)):
        assert L.normtest_mx_matmul_workspace_bytes(*sizes, 0, 0, 0) == 0


def norm(rows=4, cols=100, *, x=0x1000, x_ld=100, residual=None, residual_ld=0, weight=0x2000, eps=1e-5, dtype=B.NT_F32, sum_out=None, sum_ld=0,
         out=0x3000, out_ld=100, out_mx=None, rstd=0x4000, flags=0):
    return B.lib().normtest_rms_norm(x, x_ld, residual, residual_ld, weight, eps, dtype, rows, cols, sum_out, sum_ld, out, out_ld, out_mx, rstd, flags, None)


def test_norm():
    assert norm(x=None) == BAD and norm(x=0x1002) == BAD and norm(x_ld=99) == BAD and norm(weight=0x2002) == BAD and norm(rstd=0x4001) == BAD
    assert norm(residual=0x5000, residual_ld=99) == BAD and norm(sum_out=0x5000, sum_ld=99) == BAD and norm(out_ld=99) == BAD
    for eps in (0.0, -1.0, float("nan"), float("inf"), 1e-60, 1e60):
        assert norm(eps=eps) == BAD
    assert norm(flags=2) == BAD and norm(out_mx=mx(4, 96)) == BAD and norm(out_mx=mx(3, 100)) == BAD
    assert norm(cols=32769, x_ld=40000, out_ld=40000) == LARGE
    assert norm(rows=0, x=None, out=None) == OK and norm(cols=0, x=None, out=None) == OK


def backward(rows=4, cols=100, *, dy=0x1000, h=0x2000, weight=0x3000, rstd=0x4000, dsum=None, dtype=B.NT_F32, dx=0x5000, ld=100, dweight=None,
             scale=1.0, beta=0.0, workspace=None, size=0):
    return B.lib().normtest_rms_norm_backward(dy, ld, h, ld, weight, rstd, dsum, ld, dtype, rows, cols, dx, ld, dweight, scale, beta, workspace, size, None)


def test_backward():
    assert backward(dy=None) == BAD and backward(h=None) == BAD and backward(rstd=None) == BAD and backward(ld=99) == BAD and backward(dx=None) == BAD
    assert backward(dx=0x5002) == BAD and backward(dweight=0x6002) == BAD and backward(rstd=0x4002) == BAD
    for x in (float("nan"), float("inf"), 1e300):
        assert backward(scale=x) == BAD and backward(beta=x) == BAD
    need = B.normtest_rms_norm_workspace_bytes(4, 100)
    assert need > 0
    assert backward(dweight=0x6000) == SMALL and backward(dweight=0x6000, workspace=0x8000, size=need - 1) == SMALL
    assert backward(dweight=0x6000, workspace=0x8008, size=need) == BAD
    assert backward(cols=32769, ld=40000) == LARGE
    assert backward(rows=0, dy=None, h=None, rstd=None, dx=0x5000) == OK and backward(cols=0, dy=None, h=None, dweight=0x6000) == OK
    assert B.normtest_rms_norm_workspace_bytes(0, 100) == 0 and B.normtest_rms_norm_workspace_bytes(4, 1 << 20) == 0


def test_binding_refuses():
    x, bytes_ = torch.zeros(4, 64), torch.zeros(4, 64, dtype=torch.uint8)
    with pytest.raises(ValueError, match="no CPU path"):
        B.normtest_mx_quantize(x, None, None)
    with pytest.raises(ValueError, match="no CPU path"):
        B.MxTensor(bytes_, bytes_, 64)
    with pytest.raises(ValueError, match="format"):
        B.MxTensor(bytes_, bytes_, 64, 5)
    with pytest.raises(ValueError, match="bytes in a row"):
        B.MxTensor(bytes_, bytes_, 4 * 64 + 1, B.NT_MX_E2M1)
    with pytest.raises(ValueError, match="uint8"):
        B.MxTensor(x, bytes_, 64)
    with pytest.raises(ValueError, match="overlap"):
        B.MxTensor(bytes_.as_strided((4, 32), (16, 1)), bytes_, 64)
    with pytest.raises(ValueError, match="negative"):
        B.make_mx(-1, 4)
    with pytest.raises(TypeError, match="MxTensor"):
        B.normtest_mx_matmul(x, x)
    with pytest.raises(TypeError, match="MxTensor"):
        B.normtest_mx_dequantize(x)
    with pytest.raises(ValueError, match="no CPU path"):
        B.normtest_rms_norm(x, None, x)
    with pytest.raises(ValueError, match="contiguous last axis"):
        B.normtest_rms_norm_backward(x.t()[:2], x, None, x[:, 0], x)
    with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
        B.normtest_mx_quantize(x.double(), None)


def test_record_is_the_headers():
    assert ctypes.sizeof(B.nt_mx) == 56 and B.nt_mx.format.offset == 48


# ---- the reference -------------------------------------------------------------------------

def test_reference_rounds_as_torch_does():
    x = torch.cat([torch.linspace(-500, 500, 4001), torch.linspace(-0.05, 0.05, 4001), torch.tensor([0.0, 2.0 ** -10, 2.0 ** -9, 3 * 2.0 ** -10])])
    got, _ = R.quantize(np.concatenate([x.numpy().astype(float)[:, None], np.full((len(x), 1), 256.0)], 1), R.E4M3)   # 256: the scale is 1
    assert np.array_equal(got[:, 0, 0], x.clamp(-448, 448).to(torch.float8_e4m3fn).double().numpy())
    codes = torch.arange(256, dtype=torch.uint8)
    assert np.array_equal(R.decode(codes.numpy().reshape(1, -1), R.E4M3).ravel(), codes.view(torch.float8_e4m3fn).double().numpy(), equal_nan=True)


def test_reference_by_hand():
    row = np.array([[6.0, 5.0, 2.5, 3.5, 1.75, 0.25, 0.75, -0.26, 7.0]])
    grid, scales = R.quantize(row, R.E2M1)
    assert scales.tolist() == [[127]] and grid[0, 0, :9].tolist() == [6, 4, 2, 4, 2, 0, 1, -0.5, 6]
    grid, scales = R.quantize(row, R.E2M1, fit=True)
    assert scales.tolist() == [[128]] and grid[0, 0, 0] == 3 and grid[0, 0, 8] == 4
    grid, _ = R.quantize(row, R.E2M1, noise=np.array([[255, 127, 127, 128, 0, 127, 128, 255, 0]]))
    assert grid[0, 0, :9].tolist() == [6, 6, 3, 3, 2, 0.5, 0.5, 0, 6]   # 256 0.52 is 133, not over 255.5
    for bad in (np.nan, np.inf, -np.inf):
        grid, scales = R.quantize(np.array([[1.0] * 32 + [bad, 1.0]]), R.E4M3)
        assert scales.tolist() == [[119, 255]] and not grid[0, 1].any()
    assert R.quantize(np.zeros((1, 5)), R.E4M3)[1].tolist() == [[0]] and R.quantize(np.full((1, 5), 2.0 ** -140), R.E4M3)[1].tolist() == [[0]]
