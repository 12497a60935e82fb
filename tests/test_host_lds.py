"""Room for LDS of the kernels around the mask, on each device, by a program that stands in for the HIP runtime (host_lds_checks.cpp)."""

import os
import subprocess

import paper_2411_15100_amd as xgm
from paper_2411_15100_amd import build as lib_build

HERE = os.path.dirname(os.path.abspath(__file__))


def test_kernels_have_room_for_their_lds_on_every_device(tmp_path):
    xgm.load_library()  # (built if it is not)
    out, include = str(tmp_path / "checks"), os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-Wall", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-isystem", include,
                    os.path.join(HERE, "host_lds_checks.cpp"), "-o", out, "-ldl"], check=True)
    done = subprocess.run([out, lib_build.LIB], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stdout + done.stderr
