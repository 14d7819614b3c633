"""Calls under stream capture on a stand-in HIP runtime (no device): tests/hip_stub/capture_path.cpp,
beside ops_path.cpp, runs a scenario through the C ABI and checks what was asked of the runtime."""
import os
import shutil
import subprocess

import pytest

from paper_2608_14575_amd import hwr

HERE = os.path.dirname(os.path.abspath(__file__))
PKG = os.path.dirname(hwr.LIB_PATH)
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path_factory.mktemp("hip_stub") / "capture_path")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-Wno-unused-function", "-Werror", "-D__HIP_PLATFORM_AMD__",
                    "-isystem", os.path.join(ROCM, "include"), "-I", os.path.join(os.path.dirname(HERE), "include"),
                    os.path.join(HERE, "hip_stub", "capture_path.cpp"), f"-L{PKG}", "-lhwr", f"-Wl,-rpath,{PKG}",
                    f"-Wl,-rpath-link,{os.path.join(ROCM, 'lib')}", "-o", exe], check=True)
    return exe


@pytest.mark.parametrize("scenario", ["adamw_init", "gradients_one_after_the_other"])
def test_captured_calls(driver, scenario):
    r = subprocess.run([driver, scenario], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0 and r.stdout.strip() == "ok", r.stdout + r.stderr
