"""CPU checks of the product with sums in full: which kernels it launches, in the workspace that the sizes ask for, and its refusals."""
from __future__ import annotations

import os
import re
import subprocess
import sys

import pytest
from test_mx_host import BAD, LARGE, OK, SMALL, mx
from test_mx_launches_host import HERE

from paper_2412_21124_amd import binding as B

# sizes, formats, type and scales' offset from stdin, a line each; fabricated pointers, as nothing is ever dereferenced
CLIENT = """
import ctypes, struct, sys
fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
vp, dbl, i64, size = ctypes.c_void_p, ctypes.c_double, ctypes.c_int64, ctypes.c_size_t
lib.normtest_mx_matmul_workspace_bytes.restype = size
def mx(rows, cols, form, odd):
    blocks = -(-cols // 32)
    return struct.pack("PPqqqqii", 0x10000, 0x20000 + odd, rows, cols, blocks * (32 if form else 16), -(-blocks // 16) * 16, form, 0)
for line in sys.stdin:
    M, N, K, fa, fb, t, odd = map(int, line.split())
    need = lib.normtest_mx_matmul_workspace_bytes(i64(M), i64(N), i64(K), fa, fb, t)
    for name in ("normtest_mx_matmul", "normtest_mx_matmul_full"):
        rc = getattr(lib, name)(mx(M, K, fa, odd), mx(N, K, fb, 0), dbl(1), dbl(0), vp(0x30000), t, i64(N), vp(0x40000) if need else None, size(need), None)
        print("rc", rc, need, flush=True)
"""


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """Function from calls to, of each, (workspace bytes, launches of the product, of the one with sums in full): (kernel, template arguments, blocks)."""
    fake = str(tmp_path_factory.mktemp("fake") / "libfakehip.so")
    subprocess.run(["gcc", "-std=gnu99", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", os.path.join(HERE, "fake_hip.c"), "-o", fake], check=True)

    def run(calls):
        out = subprocess.run([sys.executable, "-c", CLIENT, fake, B.lib()._name], check=True, capture_output=True, text=True,
                             input="".join(" ".join(map(str, c)) + "\n" for c in calls)).stdout
        got, now = [], []
        for line in out.splitlines():
            if line.startswith("rc "):
                rc, need = map(int, line.split()[1:])
                assert rc == OK
                got.append((need, now))
                now = []
            elif re.search(r"\dk_", line):
                name, grid = line.split()[:2]
                now.append((re.search(r"\d(k_[a-z_]*[a-z])", name).group(1), [int(x) for x in re.findall(r"L[ib](\d+)E", name)], int(grid)))
        assert len(got) == 2 * len(calls) and not now
        return [(a[0], a[1], b[1]) for a, b in zip(got[::2], got[1::2])]

    return run


BF16, F16, F32 = B.NT_BF16, B.NT_F16, B.NT_F32


def test_widened_where_an_operand_has_8_bits(launches):
    got = launches([(1, 16384, 4096, 1, 0, BF16, 0), (300, 520, 768, 0, 1, F16, 0), (8192, 16384, 4096, 1, 0, BF16, 0), (8192, 8192, 8192, 1, 1, BF16, 1)])
    assert got[0][2] == [("k_mm_thin", [1, 0, 1, 1, 2, 4], 512)]
    assert got[1][2][0] == ("k_mm_tile", [0, 1, 1, 128, 128, 2, 2], 15)
    assert got[2][2] == [("k_mm_tile", [1, 0, 1, 128, 128, 2, 2], 64 * 128)]
    assert got[3][2] == [("k_mm_tile", [1, 1, 1, 128, 128, 2, 2], 64 * 64)]


def test_nothing_to_widen(launches):
    """Products in 4 bits are in full as they are, and those for fp32 results always were."""
    same = [(M, N, K, fa, fb, t, 0) for M, N, K in ((1, 300, 5000), (48, 96, 30000), (300, 520, 768), (8192, 8192, 8192)) for fa in (0, 1) for fb in (0, 1)
            for t in (BF16, F16, F32) if t == F32 or fa == fb == 0]
    for call, (_, default, full) in zip(same, launches(same)):
        assert default == full, call


def test_workspace_serves_both(launches):
    """What joins parts reads as many as the workspace has room for."""
    calls = [(M, N, K, 1, fb, t, odd) for M in (1, 33, 64, 200, 2000, 3400, 5000) for N in (1, 100, 3700, 50257) for K in (40, 2048, 40000) for fb in (0, 1)
             for t in (BF16, F16) for odd in (0, 1)]
    for call, (need, default, full) in zip(calls, launches(calls)):
        assert (need > 0) == (len(default) == 2) == (len(full) == 2), call
        assert default[1:] == full[1:], call


def test_refusals():
    """Those of the product."""
    L = B.lib()

    def full(M=4, N=8, K=100, *, a=None, b=None, scale=1.0, beta=0.0, out=0x1000, dtype=BF16, ld=8, workspace=None, size=0):
        return L.normtest_mx_matmul_full(a or mx(M, K, B.NT_MX_E4M3), b or mx(N, K), scale, beta, out, dtype, ld, workspace, size, None)
    assert L.normtest_mx_matmul_full(None, mx(8, 100), 1.0, 0.0, 0x1000, 0, 8, None, 0, None) == BAD
    assert full(out=None) == BAD and full(out=0x1001) == BAD and full(ld=7) == BAD and full(b=mx(8, 101)) == BAD and full(scale=float("nan")) == BAD
    assert full(K=(1 << 22) + 1) == LARGE and full(M=0, a=mx(0, 100, codes=0, scales=0), out=None) == OK
    need = L.normtest_mx_matmul_workspace_bytes(64, 64, 1 << 20, B.NT_MX_E4M3, B.NT_MX_E2M1, BF16)
    long = dict(M=64, N=64, K=1 << 20, ld=64)
    assert need > 0 and full(**long) == SMALL and full(**long, workspace=0x8000, size=need - 1) == SMALL and full(**long, workspace=0x8008, size=need) == BAD


def test_workspace_of_another_type():
    """A type that no result has is refused like those of the other calls."""
    from test_mx_replaced_host import bytes_
    a = B.MxTensor(bytes_(32, 32), bytes_(32, 16), 32, B.NT_MX_E4M3)
    assert B.normtest_mx_matmul_workspace_bytes(a, a) == 0
    for dtype in (B.torch.float64, B.torch.uint8, None):
        with pytest.raises(TypeError, match="float32, bfloat16 or float16"):
            B.normtest_mx_matmul_workspace_bytes(a, a, dtype)
