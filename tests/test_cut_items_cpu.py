"""The work items of a product by row whose last round of tiles is cut, on the host
(tests/hip_stub/cut_items.cpp): every quarter of every tile once, none past the grid."""
import os
import shutil
import subprocess

import pytest

from paper_2608_14575_amd import hwr

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(hwr.LIB_PATH), "csrc")


def test_cut_items(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "cut_items")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unknown-pragmas", "-I", CSRC,
                    os.path.join(HERE, "hip_stub", "cut_items.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
