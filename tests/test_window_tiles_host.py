"""CPU test of the windowed attention's row tiles at the sizes that its kernels and their plan share, those of two fp32
blocks among them: tile numbers increase, suffice for every sequence's rows and stay within the launch."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_20397_amd", "csrc")


def test_tiles(tmp_path):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = str(tmp_path / "window_tiles_harness")
    subprocess.run([hipcc, "-x", "hip", "--offload-arch=gfx950", "-std=c++17", "-O2", "-Xclang", "-target-feature",
                    "-Xclang", "-packed-fp32-ops", "-I", CSRC, os.path.join(ROOT, "tests", "window_tiles_harness.cpp"),
                    "-o", exe], check=True, capture_output=True)
    out = subprocess.run([exe], capture_output=True, text=True, check=True, timeout=300).stdout.split()
    assert out == ["ok"], out
