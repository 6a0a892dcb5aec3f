"""The build where a compiler fails: it says so once every compiler that it started has ended, and leaves nothing behind."""
import os
import time

import pytest

from paper_2412_21124_amd import build

# the failing source at once; the other one writes its object some time later
HIPCC = """#!/bin/sh
for a in "$@"; do [ "$a" = fails.hip ] && { echo "fails.hip: no" >&2; exit 1; }; done
while [ "$1" != -o ]; do shift; done
sleep 0.5
echo > "$2"
"""


@pytest.mark.parametrize("order", [("fails.hip", "other.hip"), ("other.hip", "fails.hip")], ids=" ".join)
def test_one_source_fails(tmp_path, monkeypatch, order):
    tool, out = tmp_path / "bin", tmp_path / "out"
    tool.mkdir()
    out.mkdir()
    (tool / "hipcc").write_text(HIPCC)
    (tool / "hipcc").chmod(0o755)
    monkeypatch.setenv("PATH", "%s:%s" % (tool, os.environ["PATH"]))
    monkeypatch.setattr(build, "SRC", order[0])
    monkeypatch.setattr(build, "TENSORS_SRC", order[1])
    with pytest.raises(RuntimeError, match="fails.hip: no"):
        build.build_library(str(out / "lib.so"))
    time.sleep(1)
    assert os.listdir(out) == []
