"""What calls hand on to the kernels, and what one that fails leaves behind: the host side against a HIP runtime that runs on the host (tests/native/host_calls.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def host_calls(tmp_path_factory):
    cxx = shutil.which("g++")
    if cxx is None or not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"):
        pytest.skip("no g++ or no HIP headers")
    csrc = os.path.join(ROOT, "paper_2401_06761_amd", "csrc")
    exe = str(tmp_path_factory.mktemp("native") / "host_calls")
    built = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-I" + os.path.join(ROOT, "include"),
                            "-I" + csrc, os.path.join(ROOT, "tests", "native", "host_calls.cpp")] +
                           [os.path.join(csrc, f) for f in ("plan.cpp", "apar_pool.cpp", "controller.cpp", "rotary.cpp")] + ["-o", exe], capture_output=True, text=True)
    assert built.returncode == 0, built.stderr[-3000:]
    return exe


@pytest.mark.parametrize("check", ["admission", "failures", "reads", "failed_launches"])
def test_host_side(host_calls, check):
    ran = subprocess.run([host_calls, check], capture_output=True, text=True, timeout=120)
    assert ran.returncode == 0 and ran.stdout == f"ok: {check}\n", ran.stdout + ran.stderr
