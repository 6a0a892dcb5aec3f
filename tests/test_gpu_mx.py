"""Microscaled quantisation, its inverse and the product on the GPU against 64-bit references."""
import itertools

import mx_reference as R
import numpy as np
import pytest
import torch

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
FORMS = {"e2m1": B.NT_MX_E2M1, "e4m3": B.NT_MX_E4M3}


def matrix(rows, cols, dtype, seed, pad=0, scale=1.0):
    """Normal values, every row and column with a scale of its own, in rows `pad` elements apart."""
    gen = torch.Generator().manual_seed(seed)
    x = torch.randn(rows, cols, generator=gen) * scale
    x *= torch.exp2(torch.randint(-6, 3, (rows, 1), generator=gen).float()) * torch.exp2(torch.randint(-3, 2, (1, cols), generator=gen).float())
    whole = torch.full((rows, cols + pad), 7.0, dtype=dtype, device=DEV)
    whole[:, :cols] = x.to(DEV)
    return whole[:, :cols]


def same(a, b):
    return np.array_equal(a, b, equal_nan=True)


def checked_mx(mx, want, scales):
    """Codes, scales and the zeros behind the last column."""
    blocks = want.shape[1]
    codes = mx.codes.cpu().numpy()[:, :blocks * R.BYTES[mx.format]]
    got = R.decode(codes, mx.format)
    assert np.array_equal(mx.scales.cpu().numpy()[:, :blocks], scales)
    assert np.array_equal(got, want)
    behind = got.reshape(got.shape[0], -1)[:, mx.cols:]
    assert not behind.any()


SHAPES = [(1, 1), (1, 31), (1, 32), (1, 33), (3, 64), (33, 7), (5, 129), (128, 128), (129, 127), (130, 261), (2, 5000), (300, 40), (257, 1000)]


@pytest.mark.parametrize("form,dtype", itertools.product(FORMS, TYPES))
@pytest.mark.parametrize("rows,cols", SHAPES, ids=lambda v: str(v))
def test_quantize(rows, cols, form, dtype):
    """Every flag, both directions, strides: all bits."""
    for k, (fit, noisy, which) in enumerate(itertools.product((False, True), (False, True), ("rows", "transpose", "both"))):
        x = matrix(rows, cols, TYPES[dtype], 100 * rows + cols + k, pad=(0, 3, 8)[k % 3])
        noise = torch.randint(256, (rows, cols + 5), dtype=torch.uint8, device=DEV)[:, :cols] if noisy else None
        other = "e4m3" if form == "e2m1" and k % 2 else form
        out = B.make_mx(rows, cols, FORMS[form], DEV) if which != "transpose" else None
        out_t = B.make_mx(cols, rows, FORMS[other], DEV) if which != "rows" else None
        for m in (out, out_t):
            if m is not None:
                m.codes.fill_(0x5a)
        B.normtest_mx_quantize(x, out, out_t, fit=fit, noise=noise)
        wide, wide_noise = R.wide(x), None if noise is None else noise.cpu().numpy()
        if out is not None:
            checked_mx(out, *R.quantize(wide, FORMS[form], fit, wide_noise))
        if out_t is not None:
            checked_mx(out_t, *R.quantize(wide.T, FORMS[other], fit, None if noise is None else wide_noise.T))


@pytest.mark.parametrize("form", FORMS)
def test_quantize_borders(form):
    """Every number of the format and its neighbours' middles, at every scale, signs, powers of two, subnormals, zeros, NaN and infinities."""
    grid = R.GRID[FORMS[form]]
    middle = (grid[1:] + grid[:-1]) / 2
    nudged = np.concatenate([grid, middle, middle * (1 + 2.0 ** -22), middle * (1 - 2.0 ** -22)]).astype(np.float32)
    rows = []
    for e in (-140, -127, -126, -120, -60, 0, 60, 100, 118):
        for top in (grid[-1], grid[-1] * 1.001, 2.0 ** R.TOP[FORMS[form]], 2.0 ** R.TOP[FORMS[form]] * 1.9999999):
            for sign in (1, -1):
                x = np.zeros((len(nudged) + 30) // 31 * 32, np.float32).reshape(-1, 32)
                x[:, 0] = np.float32(top)
                x[:, 1:].flat[:len(nudged)] = nudged * sign
                rows.append((x.astype(np.float64) * 2.0 ** e).astype(np.float32).ravel())
    width = rows[0].size
    special = np.ones((6, width), np.float32)
    special[0, 5] = np.nan
    special[1, 5] = np.inf
    special[2, width - 1] = -np.inf
    special[3] = 0
    special[4] = -0.0
    special[5] = np.finfo(np.float32).max
    x = torch.from_numpy(np.concatenate([np.stack(rows), special])).to(DEV)
    for fit in (False, True):
        out, out_t = B.make_mx(*x.shape, FORMS[form], DEV), B.make_mx(*x.t().shape, FORMS[form], DEV)
        B.normtest_mx_quantize(x, out, out_t, fit=fit)
        checked_mx(out, *R.quantize(R.wide(x), FORMS[form], fit))
        checked_mx(out_t, *R.quantize(R.wide(x).T, FORMS[form], fit))


@pytest.mark.parametrize("form", FORMS)
def test_noise_is_unbiased(form):
    """All 256 bytes for the same element: how often it goes up is its fraction, to half a byte."""
    x = torch.tensor([[6.0, 0.3, -1.1, 2.7, 5.9, 0.01, 3.3]], device=DEV).repeat(256, 1) * (1 if form == "e2m1" else 70)
    noise = torch.arange(256, dtype=torch.uint8, device=DEV)[:, None].repeat(1, 7)
    mx = B.make_mx(256, 7, FORMS[form], DEV)
    B.normtest_mx_quantize(x, mx, fit=True, noise=noise)
    mean = R.numbers(mx).mean(0)
    grid, scales = R.quantize(R.wide(x[:1]), FORMS[form], True)
    steps = np.array([np.diff(R.GRID[FORMS[form]])[np.searchsorted(R.GRID[FORMS[form]], abs(v) / 2.0 ** (scales[0, 0] - 127.0), side="right") - 1]
                      if abs(v) / 2.0 ** (scales[0, 0] - 127.0) < R.GRID[FORMS[form]][-1] else 0 for v in R.wide(x[0:1])[0]]) * 2.0 ** (scales[0, 0] - 127.0)
    assert (np.abs(mean - R.wide(x[:1])[0]) <= steps / 512 + 1e-12).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("form", FORMS)
def test_dequantize(form, dtype):
    """Every code under every scale byte, rounded to the type; odd columns and strides."""
    count = 16 if form == "e2m1" else 256
    codes = torch.arange(256, dtype=torch.uint8).repeat(256, count // 16 if form == "e2m1" else 1)
    scales = torch.arange(256, dtype=torch.uint8)[:, None].repeat(1, codes.shape[1] // R.BYTES[FORMS[form]])
    cols = codes.shape[1] * (2 if form == "e2m1" else 1)
    for less in (0, 1, 3, 13):
        mx = B.MxTensor(codes.to(DEV), scales.to(DEV), cols - less, FORMS[form])
        out = torch.full((256, cols + 5), 7.0, dtype=TYPES[dtype], device=DEV)
        B.normtest_mx_dequantize(mx, out[:, :cols - less])
        want = torch.from_numpy(R.numbers(mx)).to(TYPES[dtype])
        assert torch.equal(out[:, :cols - less].cpu().nan_to_num(12345.0, 1e30, -1e30), want.nan_to_num(12345.0, 1e30, -1e30))
        assert (out[:, cols - less:] == 7.0).all()
    assert torch.equal(B.normtest_mx_dequantize(mx, dtype=TYPES[dtype]).nan_to_num(1.0), out[:, :cols - 13].nan_to_num(1.0))


# ---- product -------------------------------------------------------------------------------

def operand(rows, cols, form, seed, pad=0, spread=0, aligned=False):
    """A microscaled matrix of random codes and scales, whose rows are `pad` blocks longer than they need, or begin at multiples of 16 scales."""
    gen = torch.Generator().manual_seed(seed)
    blocks = -(-cols // 32)
    if aligned:
        pad = -blocks % 16 + 16 * pad
    per = R.BYTES[FORMS[form]]
    if form == "e2m1":
        codes = torch.randint(256, (rows, (blocks + pad) * per), dtype=torch.uint8, generator=gen)
    else:
        x = torch.randn(rows, (blocks + pad) * per, generator=gen) * 60
        codes = x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    at = torch.arange((blocks + pad) * 32)[None].expand(rows, -1)
    if form == "e2m1":
        keep = (at < cols).view(rows, -1, 2)
        codes = codes & (keep[..., 0] * 15 + keep[..., 1] * 240).to(torch.uint8)
    else:
        codes = torch.where(at < cols, codes, 0)
    codes[:, blocks * per:] = 0x35          # behind the row's last block: never looked at
    scales = torch.randint(120 - spread, 128 + spread, (rows, blocks + pad), dtype=torch.uint8, generator=gen)
    scales[:, blocks:] = 255
    return B.MxTensor(codes.to(DEV), scales.to(DEV), cols, FORMS[form])


def product_bound(a, b, exact, wide_result):
    """How far sums may be off, from the largest magnitude they can reach.  In fp32, one rounding or cut of 2^-23 for every instruction's
    32 columns and the joins of partial sums (some 16); in 8 bits beside that, products are cut below 2^-13 of the largest of their
    eight neighbours, 7 of 8 at most, and the largest product is at most the neighbours' sum."""
    sums = np.abs(a) @ np.abs(b).T
    bound = (a.shape[1] / 32 + 16) * 2.0 ** -23 * sums
    return bound if exact or wide_result else bound + 7 * 2.0 ** -13 * sums


def check_product(a, b, dtype, scale=1.0, beta=0.0, pad=0, out=None):
    M, N = a.rows, b.rows
    whole = matrix(M, N + pad, TYPES[dtype], 5) if out is None else out
    out = whole[:, :N] if M and N else whole[:, :N]
    before, behind = R.wide(out), whole[:, N:].clone()
    if beta == 0.0:
        out.fill_(float("nan"))             # not read
    B.normtest_mx_matmul(a, b, out, scale=scale, beta=beta)
    na, nb = R.numbers(a), R.numbers(b)
    want = scale * (na @ nb.T) + beta * before
    exact = a.format == b.format == B.NT_MX_E2M1
    eps = torch.finfo(TYPES[dtype]).eps / 2
    bound = abs(scale) * product_bound(na, nb, exact, dtype == "f32")
    bound = bound * (1 + eps) + 3 * 2.0 ** -24 * (np.abs(beta * before) + np.abs(want)) + eps * np.abs(want) + 1e-40
    got = R.wide(out)
    assert (np.abs(got - want) <= bound).all(), float(np.max(np.abs(got - want) / bound))
    # and nearer than the worst that can happen: 2-norms, 4e-5 for sums in 8 bits (products cut at random places) beside the result's rounding
    rel = np.linalg.norm(got - want) / max(np.linalg.norm(want), 1e-300)
    cancel = np.linalg.norm(np.abs(scale) * (np.abs(na) @ np.abs(nb).T)) / max(np.linalg.norm(want), 1e-300)
    assert rel <= eps + (1e-6 if exact or dtype == "f32" else 1.5e-4) * cancel
    assert torch.equal(whole[:, N:], behind)
    return out


KINDS = list(itertools.product(FORMS, FORMS))
PRODUCTS = [(1, 1, 1), (1, 16, 32), (1, 100, 500), (3, 17, 513), (16, 64, 1024), (17, 33, 2000), (32, 129, 96), (33, 70, 640), (65, 250, 1100), (130, 131, 31),
            (200, 300, 4099), (1, 513, 8192), (300, 520, 768)]


@pytest.mark.parametrize("form,form_b", KINDS, ids="-".join)
@pytest.mark.parametrize("M,N,K", PRODUCTS, ids=lambda v: str(v))
def test_product(M, N, K, form, form_b):
    for k, (dtype, (scale, beta)) in enumerate(zip(("bf16", "f32", "f16", "f32"), ((1.0, 0.0), (0.5, 1.0), (0.25, -0.5), (-2.0, 0.0)))):
        a, b = operand(M, K, form, 10 * M + K + k, pad=k % 2), operand(N, K, form_b, 7 * N + K + k, pad=k // 2)
        check_product(a, b, dtype, scale, beta, pad=(0, 3, 1, 0)[k])


@pytest.mark.parametrize("form,form_b", KINDS, ids="-".join)
def test_product_scales(form, form_b):
    """Scales over a wide range, where fp32 results keep every block that counts, the extremes, and blocks that are NaN."""
    a, b = operand(40, 700, form, 1, spread=25), operand(50, 700, form_b, 2, spread=25)
    check_product(a, b, "f32")
    a, b = operand(20, 64, form, 3), operand(24, 64, form_b, 4)
    a.scales[:, :] = 0          # 2^-127 times 2^127
    b.scales[:, :] = 254
    check_product(a, b, "bf16")
    if form == form_b == "e2m1":
        check_product(a, b, "f32")
    else:                       # widened to bf16, elements of 2^128 and more are infinite
        assert not torch.isfinite(B.normtest_mx_matmul(a, b, dtype=torch.float32)).any()
    a.scales[:, :] = 4          # the least code 2^-9 2^-123 and the largest 448 2^118: all of them are bf16 numbers
    b.scales[:, :] = 245
    check_product(a, b, "f32")
    check_product(b, a, "f32")
    a, b = operand(40, 700, form, 5), operand(50, 700, form_b, 6)
    a.scales[3, 2] = 255
    b.scales[7, 21] = 255
    for dtype in (torch.bfloat16, torch.float32):
        out = B.normtest_mx_matmul(a, b, dtype=dtype).float().cpu()
        bad = torch.isnan(out)
        want = torch.zeros(40, 50, dtype=torch.bool)
        want[3], want[:, 7] = True, True
        assert torch.equal(bad, want)


@pytest.mark.parametrize("form,form_b", KINDS, ids="-".join)
def test_product_of_many_tiles(form, form_b):
    """More tiles than the chip takes at once, edges that end inside one, and sums over parts of the columns: against a product in 64 bits on the GPU."""
    for M, N, K, dtype in ((1000, 2100, 300, "bf16"), (700, 900, 5000, "f32"), (64, 128, 40000, "f32"), (2, 40, 70000, "bf16"), (520, 1030, 1500, "f16"),
                           (3700, 3700, 700, "bf16"), (3333, 4000, 2100, "f16"), (4100, 3601, 31, "bf16")):
        a, b = operand(M, K, form, M, aligned=M > 3000), operand(N, K, form_b, N, pad=1, aligned=N > 3000)
        na, nb = torch.from_numpy(R.numbers(a)).to(DEV), torch.from_numpy(R.numbers(b)).to(DEV)
        want = na @ nb.t().contiguous()
        got = B.normtest_mx_matmul(a, b, dtype=TYPES[dtype]).double()
        sums = na.abs() @ nb.abs().t().contiguous()
        exact = form == form_b == "e2m1"
        bound = ((K / 32 + 16) * 2.0 ** -23 + (0 if exact or dtype == "f32" else 7 * 2.0 ** -13)) * sums + torch.finfo(TYPES[dtype]).eps / 2 * 1.001 * want.abs()
        most = torch.finfo(TYPES[dtype]).max
        beyond = want.abs() > most * 1.001       # of fp16: infinite there, either beside it
        assert bool((torch.isinf(got) | ~beyond).all())
        assert bool(((got - want).abs() <= bound)[want.abs() < most * 0.999].all())


def test_empty_products():
    a = B.make_mx(5, 0, B.NT_MX_E2M1, DEV)
    b = B.make_mx(7, 0, B.NT_MX_E4M3, DEV)
    out = torch.ones(5, 7, device=DEV)
    B.normtest_mx_matmul(a, b, out, beta=0.5)
    assert (out == 0.5).all()
    B.normtest_mx_matmul(a, b, out)
    assert (out == 0).all()
    assert B.normtest_mx_matmul(B.make_mx(0, 64, B.NT_MX_E2M1, DEV), B.make_mx(3, 64, B.NT_MX_E2M1, DEV)).shape == (0, 3)
    B.normtest_mx_quantize(torch.zeros(0, 64, device=DEV), B.make_mx(0, 64, B.NT_MX_E2M1, DEV), B.make_mx(64, 0, B.NT_MX_E2M1, DEV))
    assert B.normtest_mx_dequantize(B.make_mx(0, 64, B.NT_MX_E4M3, DEV)).shape == (0, 64)


def test_product_repeats():
    """The same bits every time, with partial sums too."""
    a, b = operand(48, 30000, "e4m3", 1), operand(96, 30000, "e2m1", 2)
    first = B.normtest_mx_matmul(a, b, dtype=torch.float32)
    for _ in range(5):
        assert torch.equal(B.normtest_mx_matmul(a, b, dtype=torch.float32), first)


@pytest.mark.parametrize("form,form_b", KINDS, ids="-".join)
@pytest.mark.parametrize("M,N,K", [(1, 16500, 600), (24, 16450, 1290), (7, 16390, 2100), (30, 33000, 40)], ids=lambda v: str(v))
def test_product_of_few_rows_and_many_columns(M, N, K, form, form_b):
    for k, dtype in enumerate(("bf16", "f32")):
        check_product(operand(M, K, form, M + K + k), operand(N, K, form_b, N + K + k, pad=k), dtype, 0.5, 1.0, pad=1 - k)


@pytest.mark.parametrize("form,form_b", KINDS, ids="-".join)
def test_product_of_rows_far_apart(form, form_b):
    """Over 4 MB from row to row: beyond the offsets that tiles load with.  A single row's distance means nothing."""
    far = (1 << 22) + 16

    def apart(m, rows_apart):
        codes = torch.empty(m.rows, rows_apart, dtype=torch.uint8, device=DEV)[:, : m.codes.shape[1]]
        return B.MxTensor(codes.copy_(m.codes), m.scales, m.cols, m.format)

    for k, (M, N, K, dtype) in enumerate([(130, 70, 1100, "f32"), (33, 300, 5000, "bf16"), (5, 90, 700, "f32")]):
        a, b = operand(M, K, form, k), operand(N, K, form_b, k + 50)
        for x, y in ((apart(a, far), b), (a, apart(b, far)), (apart(a, far), apart(b, far))):
            check_product(x, y, dtype)
    one, many = operand(1, 600, form, 3), operand(300, 600, form_b, 4)
    codes = torch.as_strided(one.codes, one.codes.shape, (1 << 40, 1))
    same = B.MxTensor(codes, one.scales, 600, one.format)
    assert torch.equal(B.normtest_mx_matmul(same, many), B.normtest_mx_matmul(one, many))
    assert torch.equal(B.normtest_mx_matmul(many, same), B.normtest_mx_matmul(many, one))
