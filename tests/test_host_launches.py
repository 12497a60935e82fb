"""Calls around the mask at the ends of their ranges launch what can be launched, by a program that stands in for the HIP runtime (host_launch_checks.cpp)."""

import os
import subprocess

import pytest

import paper_2411_15100_amd as xgm
from paper_2411_15100_amd import build as lib_build

HERE = os.path.dirname(os.path.abspath(__file__))


@pytest.fixture(scope="module")
def checks(tmp_path_factory):
    xgm.load_library()  # (built if it is not)
    out, include = str(tmp_path_factory.mktemp("launches") / "checks"), os.path.join(os.environ.get("ROCM_PATH", "/opt/rocm"), "include")
    subprocess.run([os.environ.get("CXX", "g++"), "-O1", "-std=c++17", "-Wall", "-rdynamic", "-D__HIP_PLATFORM_AMD__", "-isystem", include,
                    os.path.join(HERE, "host_launch_checks.cpp"), "-o", out, "-ldl"], check=True)
    return out


@pytest.mark.parametrize("what", ["lookups", "rows", "projection", "beams"])
def test_what_calls_accept_can_be_launched(checks, what):
    done = subprocess.run([checks, lib_build.LIB, what], capture_output=True, text=True, timeout=120)
    assert done.returncode == 0, done.stdout + done.stderr
