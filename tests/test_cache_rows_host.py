"""Which strides the paged cache's calls take for the rows they write (host, under sanitizers)."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_32197_amd", "csrc")
CHECK = os.path.join(ROOT, "tests", "hostcheck")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def run_check(tmp_path, name):
    cxx = os.environ.get("CXX") or shutil.which("g++")
    if not cxx or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime_api.h")):
        pytest.skip("needs g++ and the HIP runtime API headers")
    exe = str(tmp_path / name)
    srcs = [os.path.join(CSRC, f) for f in ("api.cpp", "api_cache.cpp", "host_plan.cpp")]
    srcs += [os.path.join(CHECK, f) for f in ("stub_launchers.cpp", "cache_stub_launchers.cpp",
                                              name + ".cpp")]
    r = subprocess.run([cxx, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer",
                        "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-D__HIP_PLATFORM_AMD__", f"-I{os.path.join(ROCM, 'include')}", *srcs, "-o",
                        exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert " 0 failures" in r.stdout


def test_rows_that_overlap(tmp_path):
    run_check(tmp_path, "cache_rows_check")


def test_tensors_given_twice(tmp_path):
    run_check(tmp_path, "cache_alias_check")
