"""CPU tests of the windowed attention's host-checkable parts: the list of pages that a tile of rows reads (every key
that a row sees is listed, nothing behind the sequence is, every unseen slot of a listed page has a seen stand-in of
that page) and the numbering of row tiles, by enumeration in a small harness (window_harness.cpp) built from the
library's own header."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_20397_amd", "csrc")


def test_lists_and_tiles(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "window_harness")
    subprocess.run([hipcc, "-x", "hip", "--offload-arch=gfx950", "-std=c++17", "-O2", "-Xclang", "-target-feature",
                    "-Xclang", "-packed-fp32-ops", "-I", CSRC, os.path.join(ROOT, "tests", "window_harness.cpp"),
                    "-o", exe], check=True, capture_output=True)
    out = subprocess.run([exe], capture_output=True, text=True, check=True, timeout=300).stdout.split()
    assert out[0] == "ok" and int(out[1]) > 10000 and int(out[2]) == 20000, out
