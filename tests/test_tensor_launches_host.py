"""What a call on lists launches, seen without a GPU: the library runs on a runtime that only prints its launches (fake_hip.c), in a
process of its own."""
from __future__ import annotations

import ctypes
import json
import os
import re
import subprocess
import sys

import pytest

from paper_2412_21124_amd import binding as B

HERE = os.path.dirname(os.path.abspath(__file__))

# calls from stdin, one JSON list per line; fabricated pointers, as nothing is ever dereferenced but the plan's host image
CLIENT = """
import ctypes, json, struct, sys
fake = ctypes.CDLL(sys.argv[1], mode=ctypes.RTLD_GLOBAL)
lib = ctypes.CDLL(sys.argv[2])
vp, dbl = ctypes.c_void_p, ctypes.c_double
hyper = struct.pack("6d4qiI", 1e-3, 0.9, 0.95, 1e-8, 0.1, 0.1, 1, 64, 0, 1, 1, 2)
for line in sys.stdin:
    c = json.loads(line)
    records = b"".join(struct.pack("Pqqqii", 0x1000, r, n, n, 0, g) for r, n, g in c["shapes"]) or None
    p = ctypes.create_string_buffer(int(sys.argv[3]))
    rc = lib.normtest_plan_make(records, len(c["shapes"]), c["G"], p, None, ctypes.c_size_t(0))
    struct.pack_into("P", p, 0, 0x100000)
    a, n = vp(0x2000), vp(0x3000)
    if c["call"] == "norm":
        rc = rc or lib.normtest_grad_norm(p, a, c["kind"], dbl(1.0), dbl(1.0), n, None)
    elif c["call"] == "clip":
        rc = rc or lib.normtest_clip_grads(p, a, None, n, None)
    elif c["call"] == "accumulate":
        rc = rc or lib.normtest_accumulate(p, a, a, dbl(c["beta"]), dbl(1.0), None, c["kind"], dbl(0.0), dbl(1.0), n if c["total"] else None, None)
    else:
        rc = rc or lib.normtest_adamw_tensors(p, a, a, a, a, None, hyper, dbl(1.0), None, 0, None)
    print("rc", rc, flush=True)
"""


def _call(call, shapes, G=1, kind=0, beta=1.0, total=False):
    return dict(call=call, shapes=[s if len(s) == 3 else (*s, 0) for s in shapes], G=G, kind=kind, beta=beta, total=total)


@pytest.fixture(scope="module")
def launches(tmp_path_factory):
    """Function from a list of calls to the launches of each: (kernel, template arguments, blocks, threads, dynamic LDS)."""
    fake = str(tmp_path_factory.mktemp("fake") / "libfakehip.so")
    subprocess.run(["gcc", "-std=gnu99", "-Wall", "-Wextra", "-Werror", "-shared", "-fPIC", os.path.join(HERE, "fake_hip.c"), "-o", fake], check=True)

    def run(calls):
        out = subprocess.run([sys.executable, "-c", CLIENT, fake, B.lib()._name, str(ctypes.sizeof(B.nt_plan))], check=True, capture_output=True, text=True,
                             input="".join(json.dumps(c) + "\n" for c in calls)).stdout
        got, now = [], []
        for line in out.splitlines():
            if line.startswith("rc "):
                assert line == "rc 0"
                got.append(now)
                now = []
            elif re.search(r"\dk_", line):
                name, grid, block, lds = line.split()
                kind = "max" if "Largest" in name else "l2" if "Square" in name else ""
                now.append((re.search(r"\d(k_[a-z_]*[a-z])", name).group(1), kind, [int(x) for x in re.findall(r"L[ib](\d+)E", name)], int(grid),
                            int(block), int(lds)))
        assert len(got) == len(calls) and not now
        return got

    return run


def test_norms(launches):
    got = launches([_call("norm", []), _call("norm", [(1, 100_003)]), _call("norm", [(1, (1 << 21) - 1)], kind=1), _call("norm", [(1, 1 << 21)]),
                    _call("norm", [(1, 1 << 24)]), _call("norm", [(1, 1 << 27)]), _call("norm", [(1, 1 << 24, g) for g in range(8)], G=8),
                    _call("norm", [(1, 1 << 20, g) for g in range(8)], G=8), _call("norm", [(1000, 8193)]), _call("norm", [(1, 0, 0), (1, 5, 2)], G=4)])
    one = [("k_norm", "l2", [0], b, 256, 0) for b in (1, 25)]
    assert got[0] == [one[0]] and got[1] == [one[1]]
    assert got[2] == [("k_norm", "max", [0], 512, 256, 0)]           # a block per item of 4096
    assert got[3] == [("k_norm", "l2", [0], 128, 256, 0)]            # two items of 8192 each
    assert got[4] == [("k_norm", "l2", [0], 1024, 256, 0)] and got[5] == [("k_norm", "l2", [1], 1024, 256, 0)]
    assert got[6] == [("k_norm", "l2", [1], 1024, 256, 0)]           # 2048 items in each group: walked
    assert got[7] == [("k_norm", "l2", [0], 512, 256, 0)]            # 128: runs of two
    assert got[8] == [("k_norm", "l2", [0], 1024, 256, 0)]           # rows of two items each
    assert got[9] == [("k_norm", "l2", [0], 4, 256, 0)]              # an item for every group without elements


def test_updates(launches):
    got = launches([_call("clip", [(1, 5000)]), _call("clip", [(1, 3 << 23)]), _call("accumulate", [(1, 1 << 27)], beta=0.0),
                    _call("accumulate", [(1, 1 << 27)], total=True), _call("accumulate", [(1, 5000)], beta=0.0, total=True, kind=1),
                    _call("clip", [(1, (1 << 32) + 1)])])
    assert got[0] == [("k_update", "", [0, 0, 256], 2, 256, 0)]
    assert got[1] == [("k_update", "", [0, 1, 256], 6144, 256, 0)]
    assert got[2] == [("k_update", "", [0, 2, 256], 32768, 256, 0)]
    assert got[3] == [("k_update", "l2", [1, 2, 512], 32768, 512, 0)]
    assert got[4] == [("k_update", "max", [0, 0, 512], 2, 512, 0)]
    assert got[5] == [("k_update", "", [0, 2, 256], 1 << 20, 256, 0), ("k_update", "", [0, 2, 256], 1, 256, 0)]


def test_adamw(launches):
    got = launches([_call("adamw", [(1, (1 << 23) - 1)]), _call("adamw", [(1, 1 << 23)]), _call("adamw", [(1, 5 << 23)]),
                    _call("adamw", [(1, 3 << 26)]), _call("adamw", [(1 << 13, 1 << 13)]), _call("adamw", [(1 << 14, 1 << 13)])])
    assert got[0] == [("k_adamw", "", [0, 512], 2048, 512, 0)] and got[1] == [("k_adamw", "", [1, 512], 2048, 512, 0)]
    assert got[2] == [("k_adamw", "", [1, 1024], 10240, 1024, 82000)]
    assert got[3] == [("k_adamw", "", [2, 1024], 16384, 1024, 82000)] * 3
    assert got[4] == [("k_adamw", "", [1, 512], 16384, 512, 0)]      # mostly rows: not kept in step
    assert got[5] == [("k_adamw", "", [2, 512], 32768, 512, 0)]


def test_norms_of_very_many_groups(launches):
    """A grid ends at 2^32 threads, so the norm's blocks take as many items as make one launch of 2^20 of them."""
    got = launches([_call("norm", [(1, 5, 2)], G=1 << 20), _call("norm", [(1, 5, 2)], G=(1 << 20) + 3), _call("norm", [(1, 5, 2)], G=(1 << 24) + 1),
                    _call("norm", [(1, 1 << 21, 1)], G=(1 << 22) + 1), _call("norm", [(1 << 12, 1 << 10, 1)], G=(1 << 21) + 1)])
    items = [1 << 20, (1 << 20) + 3, (1 << 24) + 1, (1 << 21) // 8192 + (1 << 22), (1 << 12) // 8 + (1 << 21)]
    for g, n, run in zip(got, items, [1, 2, 17, 5, 3]):
        assert g == [("k_norm", "l2", [0], -(-n // run), 256, 0)] and -(-n // run) <= 1 << 20


def test_adamw_of_dense_tensors_and_rows(launches):
    """Fewer than half of the elements in rows: kept in step, also the rows' items."""
    got = launches([_call("adamw", [(1, 45_000_001), (3001, 5003), (2000, 1001), (1, 7)])])
    items = 10_987 + 2 * 3001 + 500 + 1
    assert got[0] == [("k_adamw", "", [1, 1024], n, 1024, 82000) for n in (16_384, items - 16_384)]
