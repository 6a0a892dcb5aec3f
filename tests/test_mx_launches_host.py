"""What the calls on microscaled matrices and the norm launch, seen without a GPU: the library runs on a runtime that only prints its launches
(fake_hip.c), in a process of its own."""
from __future__ import annotations

import json
import os
import re
import subprocess
import sys

import pytest

from paper_2412_21124_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))

# calls from stdin, one JSON list per line; fabricated pointers, as nothing is ever dereferenced
CLIENT = """
import ctypes, json, struct, sys
fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
vp, dbl, i64, size = ctypes.c_void_p, ctypes.c_double, ctypes.c_int64, ctypes.c_size_t
lib.normtest_mx_matmul_workspace_bytes.restype = size
lib.normtest_rms_norm_workspace_bytes.restype = size
def mx(rows, cols, form, far=0, odd=0):
    blocks = -(-cols // 32)
    return struct.pack("PPqqqqii", 0x10000, 0x20000 + odd, rows, cols, far or blocks * (32 if form else 16), -(-blocks // 16) * 16, form, 0)
for line in sys.stdin:
    c = json.loads(line)
    M, N, K, t = c["M"], c["N"], c.get("K", 0), c["t"]
    need = 0
    if c["call"] == "matmul":
        a, b = mx(M, K, c["fa"], c["far"], c["odd"]), mx(N, K, c["fb"], c.get("far_b", 0))
        need = lib.normtest_mx_matmul_workspace_bytes(i64(M), i64(N), i64(K), c["fa"], c["fb"], t)
        rc = lib.normtest_mx_matmul(a, b, dbl(1), dbl(0), vp(0x30000), t, i64(N), vp(0x40000) if need else None, size(need), None)
    elif c["call"] == "quantize":
        out, out_t = mx(M, N, c["fa"]) if c["rows"] else None, mx(N, M, c["fb"]) if c["cols"] else None
        rc = lib.normtest_mx_quantize(vp(0x1000), t, i64(M), i64(N), i64(N), None, i64(0), out, out_t, 0, None)
    elif c["call"] == "norm":
        rc = lib.normtest_rms_norm(vp(0x1000), i64(N), None, i64(0), None, dbl(1e-5), t, i64(M), i64(N), None, i64(0), vp(0x2000), i64(N), None, None, 0, None)
    else:
        need = lib.normtest_rms_norm_workspace_bytes(i64(M), i64(N))
        rc = lib.normtest_rms_norm_backward(vp(0x1000), i64(N), vp(0x2000), i64(N), None, vp(0x3000), None, i64(0), t, i64(M), i64(N), vp(0x4000), i64(N),
                                            vp(0x5000), dbl(1), dbl(0), vp(0x40000), size(need), None)
    print("rc", rc, need, flush=True)
"""


def matmul(M, N, K, t=B.NT_BF16, fa=1, fb=0, far=0, odd=0):
    return dict(call="matmul", M=M, N=N, K=K, t=t, fa=fa, fb=fb, far=far, odd=odd)


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """Function from a list of calls to (workspace bytes, launches) of each: (kernel, template arguments, blocks, threads, dynamic LDS)."""
    fake = str(tmp_path_factory.mktemp("fake") / "libfakehip.so")
    subprocess.run(["gcc", "-std=gnu99", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", os.path.join(HERE, "fake_hip.c"), "-o", fake], check=True)

    def run(calls, code=0):
        out = subprocess.run([sys.executable, "-c", CLIENT, fake, B.lib()._name], check=True, capture_output=True, text=True,
                             input="".join(json.dumps(c) + "\n" for c in calls)).stdout
        got, now = [], []
        for line in out.splitlines():
            if line.startswith("rc "):
                rc, need = map(int, line.split()[1:])
                assert rc == code
                got.append((need, now))
                now = []
            elif re.search(r"\dk_", line):
                name, grid, block, lds = line.split()
                now.append((re.search(r"\d(k_[a-z_]*[a-z])", name).group(1), [int(x) for x in re.findall(r"L[ib](\d+)E", name)], int(grid), int(block), int(lds)))
        assert len(got) == len(calls) and not now
        return got

    return run


def test_few_rows(launches):
    got = launches([matmul(1, 16384, 4096), matmul(16, 64, 512), matmul(17, 50257, 768, B.NT_F32), matmul(32, 100, 100), matmul(64, 2048, 2048),
                    matmul(1, 16, 1 << 20, fa=0)])
    assert got[0] == (0, [("k_mm_thin", [1, 0, 0, 1, 2, 4], 512, 256, 0)])
    assert got[1] == (0, [("k_mm_thin", [1, 0, 0, 1, 1, 2], 2, 256, 0)])
    assert got[2] == (0, [("k_mm_thin", [1, 0, 1, 2, 2, 2], 1571, 256, 0)])       # fp32 with an 8-bit operand: widened
    assert got[3] == (0, [("k_mm_thin", [1, 0, 0, 2, 1, 2], 2, 256, 0)])
    assert got[4] == (0, [("k_mm_thin", [1, 0, 0, 4, 1, 4], 128, 256, 0)])
    need, kernels = got[5]
    assert [k[0] for k in kernels] == ["k_mm_thin", "k_mm_join"] and need == 512 * 16 * 4


def test_tiles(launches):
    got = launches([matmul(8192, 8192, 8192, fa=0), matmul(8192, 16384, 4096), matmul(8192, 8192, 8192, B.NT_F32, fa=0), matmul(8192, 8192, 8192, B.NT_F32),
                    matmul(8192, 8192, 8192, odd=1), matmul(768, 2304, 16384, B.NT_F32, fb=1), matmul(100, 200, 300), matmul(8192, 8192, 8192, far=1 << 23)])
    assert got[0] == (0, [("k_mm_large", [0, 0], 1024, 512, 4 * 256 * 128 + 16384)])
    assert got[1] == (0, [("k_mm_large", [1, 0], 2048, 512, 163840)])
    assert got[2] == (0, [("k_mm_large", [0, 0], 1024, 512, 147456)])         # 4 bits are exact
    assert got[3] == (0, [("k_mm_tile", [1, 0, 1, 128, 128, 2, 2], 4096, 256, 2 * 128 * 192 + 8192)])
    assert got[4] == (0, [("k_mm_tile", [1, 0, 0, 128, 128, 2, 2], 4096, 256, 57344)])      # scales at an odd address
    need, kernels = got[5]
    assert kernels[0] == ("k_mm_tile", [1, 1, 1, 128, 128, 2, 2], 108, 256, 73728) and kernels[1][0] == "k_mm_join" and need == 4 * 768 * 2304 * 4
    assert got[6][1][0][0] == "k_mm_tile"
    assert got[7][1][0][0] == "k_mm_thin"                                        # rows too far apart for 32-bit offsets


def test_a_large_tile_is_never_split(launches):
    """What adds parts up reads as many as the workspace has: only a kernel that writes them may be asked for them."""
    calls = [matmul(M, N, K, fa=0) for M in (3000, 3500, 3700, 4096) for N in (3000, 3700, 4096, 5000) for K in (512, 2048, 16384)]
    for c, (need, kernels) in zip(calls, launches(calls)):
        if kernels[0][0] == "k_mm_large":
            assert need == 0 and len(kernels) == 1, c
        assert (need > 0) == (len(kernels) == 2)


def test_rows_far_apart(launches):
    """The workspace that the sizes alone tell serves any distance between rows; a single row has none."""
    got = launches([matmul(128, 128, 1 << 16, far=1 << 23), matmul(200, 300, 1 << 16, B.NT_F32, far=1 << 23, fa=0), matmul(1, 8192, 4096, far=1 << 40),
                    dict(matmul(8192, 1, 64), far_b=1 << 40), dict(matmul(6000000, 1, 64), far_b=1 << 40)])
    for i in (0, 1):
        assert [k[0] for k in got[i][1]] == ["k_mm_thin"]                        # not split
    assert got[2] == launches([matmul(1, 8192, 4096)])[0]
    assert got[3] == launches([matmul(8192, 1, 64)])[0] and got[3][1][0][0] == "k_mm_tile"
    assert got[4] == launches([matmul(6000000, 1, 64)])[0]


def test_more_blocks_than_a_launch_takes(launches):
    many = matmul((1 << 31) - 1, 1, 64)
    assert launches([many], B.NT_ERR_TOO_LARGE)[0][1] == []
    assert launches([dict(matmul(1 << 23, 2, 64), far_b=1 << 23)], B.NT_ERR_TOO_LARGE)[0][1] == []


def test_quantize_and_norm(launches):
    q = lambda M, N, rows, cols, t=B.NT_BF16, fa=0, fb=0: dict(call="quantize", M=M, N=N, rows=rows, cols=cols, t=t, fa=fa, fb=fb)   # noqa: E731
    n = lambda call, M, N, t=B.NT_BF16: dict(call=call, M=M, N=N, t=t)   # noqa: E731
    got = launches([q(1, 768, 1, 0), q(300, 40, 1, 0, B.NT_F32, 1), q(16384, 8192, 1, 1), q(100, 300, 0, 1, B.NT_F16, 0, 1), n("norm", 1, 4096), n("norm", 1000, 768),
                    n("norm", 7, 32768), n("backward", 16384, 4096), n("backward", 1000, 768, B.NT_F32), n("backward", 3, 20000)])
    assert got[0][1] == [("k_mx_rows", [1, 0, 0], 1, 256, 0)] and got[1][1] == [("k_mx_rows", [0, 1, 0], 10, 256, 0)]
    assert got[2][1] == [("k_mx_both", [1, 0, 0, 1, 0], 8192, 256, 0)] and got[3][1] == [("k_mx_both", [2, 1, 1, 0, 0], 3, 256, 0)]
    assert got[4][1] == [("k_rms_norm", [1, 256, 2], 1, 256, 0)] and got[5][1] == [("k_rms_norm", [1, 64, 2], 250, 256, 0)]
    assert got[6][1] == [("k_rms_norm", [1, 1024, 4], 7, 1024, 0)]
    assert got[7] == (256 * 4096 * 4, [("k_rms_backward", [1, 256, 2, 4], 256, 1024, 0), ("k_join_columns", [], 256, 256, 0)])
    assert got[8] == (125 * 768 * 4, [("k_rms_backward", [0, 64, 2, 8], 125, 512, 0), ("k_join_columns", [], 48, 256, 0)])
    assert got[9] == (3 * 20000 * 4, [("k_rms_backward", [1, 1024, 4, 1], 3, 1024, 0), ("k_join_columns", [], 1250, 256, 0)])
