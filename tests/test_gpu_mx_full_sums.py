"""The product with sums in full, for 16-bit results of an 8-bit operand, against 64 bits."""
import numpy as np
import mx_reference as R
import pytest
import torch
from test_gpu_mx import DEV, FORMS, TYPES, matrix, operand

from paper_2412_21124_amd import binding as B

pytestmark = pytest.mark.gpu

KINDS = [("e4m3", "e2m1"), ("e2m1", "e4m3"), ("e4m3", "e4m3")]


def check(a, b, dtype, scale=1.0, beta=0.0, pad=0):
    """Within the fp32 sum's bound and one rounding: a rounding or cut of 2^-23 of the sum of magnitudes for every 32 columns and the joins of
    parts (some 16), scaling and adding what was there 3 steps of 2^-24, and half a step of the type."""
    whole = matrix(a.rows, b.rows + pad, TYPES[dtype], 5)
    out = whole[:, :b.rows]
    before, behind = out.double(), whole[:, b.rows:].clone()
    if beta == 0.0:
        out.fill_(float("nan"))             # not read
    assert B.normtest_mx_matmul(a, b, out, scale=scale, beta=beta, full_sums=True) is out
    na, nb = torch.from_numpy(R.numbers(a)).to(DEV), torch.from_numpy(R.numbers(b)).to(DEV)
    want = scale * (na @ nb.t().contiguous()) + (beta * before if beta else 0.0)
    sums = abs(scale) * (na.abs() @ nb.abs().t().contiguous())
    eps = torch.finfo(TYPES[dtype]).eps / 2
    bound = (a.cols / 32 + 16) * 2.0 ** -23 * sums + 3 * 2.0 ** -24 * (want.abs() + (abs(beta) * before.abs() if beta else 0.0))
    bound = bound * (1 + eps) + eps * want.abs() + (2.0 ** -25 if dtype == "f16" else 1e-40)
    most = torch.finfo(TYPES[dtype]).max
    held = want.abs() < most * 0.999         # beyond: infinite in fp16
    off = (out.double() - want).abs()
    assert bool((off <= bound)[held].all()), float((off / bound)[held].max())
    assert torch.equal(whole[:, b.rows:], behind)
    return out


def outliers(rows, cols, form, seed):
    """In every 8 neighbours two large codes of opposite sign and six small ones: what a sum that is cut beside the largest loses."""
    gen = torch.Generator().manual_seed(seed)
    blocks = -(-cols // 32)
    if form == "e2m1":
        codes = torch.full((rows, 16 * blocks), 0x22, dtype=torch.uint8)          # ones
        codes[:, -(-cols // 2):] = 0
        if cols % 2:
            codes[:, cols // 2] &= 15
    else:
        x = (torch.rand(rows, 32 * blocks, generator=gen) + 0.5) * 2.0 ** -5
        x[:, 0::8], x[:, 1::8] = 256.0, -256.0
        x[:, cols:] = 0
        codes = x.to(torch.float8_e4m3fn).view(torch.uint8)
    scales = torch.randint(125, 130, (rows, blocks), dtype=torch.uint8, generator=gen) if form == "e4m3" else torch.full((rows, blocks), 127, dtype=torch.uint8)
    return B.MxTensor(codes.to(DEV), scales.to(DEV), cols, FORMS[form])


@pytest.mark.parametrize("form,form_b", KINDS, ids="-".join)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 100, 512), (3, 17, 513), (24, 200, 1100), (33, 70, 640), (130, 131, 31), (300, 520, 768), (2, 40, 70000),
                                   (64, 128, 40000)], ids=str)
def test_against_64_bits(M, N, K, form, form_b):
    for k, (dtype, scale, beta) in enumerate((("bf16", 1.0, 0.0), ("f16", 0.5, 1.0), ("f32", 0.25, -0.5), ("bf16", -2.0, 1.0))):
        check(operand(M, K, form, M + K + k, pad=k % 2), operand(N, K, form_b, N + K + k, pad=k // 2), dtype, scale, beta, pad=(0, 3, 1, 0)[k])


@pytest.mark.parametrize("form,form_b", KINDS, ids="-".join)
@pytest.mark.parametrize("M,N,K", [(1, 60, 300), (20, 33, 2000), (140, 150, 300), (3700, 3700, 320)], ids=str)
def test_large_products_that_cancel(M, N, K, form, form_b):
    # against ones the large codes cancel and leave sums of some 2^-5; the bound is 2^-23 of 512 and small beside them
    a, b = outliers(M, K, form, 1), outliers(N, K, "e2m1" if form == "e4m3" else "e4m3", 2)
    for dtype in ("bf16", "f16"):
        check(a, b, dtype)
    if form == form_b:
        check(outliers(M, K, "e4m3", 3), operand(N, K, "e4m3", 4), "bf16")


def test_many_tiles():
    """Where the default takes large tiles, and beyond."""
    for form, form_b in KINDS:
        a, b = operand(3333, 2100, form, 1, aligned=True), operand(4000, 2100, form_b, 2, aligned=True)
        check(a, b, "bf16")


def test_same_bits_where_nothing_is_widened():
    a, b = operand(70, 1100, "e2m1", 1), operand(130, 1100, "e2m1", 2)
    for dtype in TYPES.values():
        assert torch.equal(B.normtest_mx_matmul(a, b, dtype=dtype, full_sums=True), B.normtest_mx_matmul(a, b, dtype=dtype))
    a = operand(70, 1100, "e4m3", 3)
    assert torch.equal(B.normtest_mx_matmul(a, b, dtype=torch.float32, full_sums=True), B.normtest_mx_matmul(a, b, dtype=torch.float32))
    # a 16-bit result is the fp32 one, rounded
    for dtype in (torch.bfloat16, torch.float16):
        assert torch.equal(B.normtest_mx_matmul(a, b, dtype=dtype, full_sums=True), B.normtest_mx_matmul(a, b, dtype=torch.float32).to(dtype))


def test_paths_streams_and_graph(monkeypatch):
    """Through either call path, with and without a workspace, on another stream, and captured: the same bits."""
    a, b = operand(48, 30000, "e4m3", 1), operand(96, 30000, "e2m1", 2)
    want = B.normtest_mx_matmul(a, b, full_sums=True)
    need = B.normtest_mx_matmul_workspace_bytes(a, b)
    assert need > 0
    out, workspace = torch.empty_like(want), torch.empty(need, dtype=torch.uint8, device=DEV)
    for fast in (B._fast, None):
        with monkeypatch.context() as m:
            m.setattr(B, "_fast", fast)
            for ws in (workspace, None):
                out.zero_()
                B.normtest_mx_matmul(a, b, out, full_sums=True, workspace=ws)
                assert torch.equal(out, want)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    other = B.normtest_mx_matmul(a, b, full_sums=True, stream=st)
    torch.cuda.current_stream().wait_stream(st)
    assert torch.equal(other, want)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.normtest_mx_matmul(a, b, out, full_sums=True, workspace=workspace)
    for k in range(3):
        b.scales.sub_(1)
        graph.replay()
        assert torch.equal(out, B.normtest_mx_matmul(a, b, full_sums=True))
        torch.cuda.synchronize()
    assert np.isfinite(R.wide(out)).all()
