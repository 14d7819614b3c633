"""The host side of the operators on a routed batch on a stand-in HIP runtime (no
device): tests/hip_stub/ops_path.cpp defines the HIP functions that they call, runs
a scenario through the C ABI and checks what was asked of the runtime.
tests/hip_stub/group_walk.cpp runs the kernels' walk over ragged groups lane by lane."""
import os
import shutil
import subprocess

import pytest

from paper_2608_14575_amd import hwr

HERE = os.path.dirname(os.path.abspath(__file__))
ROOT = os.path.dirname(HERE)
PKG = os.path.dirname(hwr.LIB_PATH)
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


CSRC = os.path.join(PKG, "csrc")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    if not os.path.exists(hwr.LIB_PATH):
        from paper_2608_14575_amd import build
        build.build()
    exe = str(tmp_path_factory.mktemp("hip_stub") / "ops_path")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Werror", "-D__HIP_PLATFORM_AMD__",
                    "-isystem", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"),
                    os.path.join(HERE, "hip_stub", "ops_path.cpp"), f"-L{PKG}", "-lhwr", f"-Wl,-rpath,{PKG}",
                    f"-Wl,-rpath-link,{os.path.join(ROCM, 'lib')}", "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("scenario", ["row_limit", "largest_grids", "work_space", "current_device",
                                      "errors_are_reported_once", "alignment", "few_rows_of_many_groups"])
def test_operators_host_side(driver, scenario):
    r = subprocess.run([driver, scenario], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr


@pytest.fixture(scope="module")
def walk(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("hip_stub") / "group_walk")
    subprocess.run(["g++", "-std=c++17", "-O1", "-fwrapv", "-Wall", "-Wno-unknown-pragmas", "-I", CSRC,
                    os.path.join(HERE, "hip_stub", "group_walk.cpp"), "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("scenario", ["tiles_cover_the_places", "anything_in_offsets", "anything_in_order"])
def test_walk_over_groups(walk, scenario):
    r = subprocess.run([walk, scenario], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
