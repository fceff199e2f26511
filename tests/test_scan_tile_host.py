"""How the selective scan's kernels bound their reads and writes, on the host (tests/scan_tile_driver.cpp)."""
import os
import shutil
import subprocess

import pytest

from paper_2010_15884_amd import build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_buffers_reach_the_rows_that_exist_and_nothing_else(tmp_path):
    if shutil.which("hipcc") is None:
        pytest.skip("hipcc is not installed")
    exe = str(tmp_path / "scan_tile_driver")
    subprocess.run(["hipcc", "-x", "hip", "--offload-arch=gfx950", "--offload-host-only", "-std=c++17", "-O1", "-I", os.path.join(build.ROOT, "include"), "-I", build.CSRC,
                    os.path.join(HERE, "scan_tile_driver.cpp"), "-o", exe], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert res.returncode == 0 and "clean" in res.stdout, res.stdout[-2000:]
