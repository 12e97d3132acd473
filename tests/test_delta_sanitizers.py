"""AddressSanitizer and UndefinedBehaviorSanitizer on the host layer of packmamba_delta.h (delta_api.cpp), built by
gcc with stubs for the launchers, under the CPU tests that call it (as test_sanitizers does for api.cpp)."""
import os
import subprocess
import sys

import pytest

from test_sanitizers import CSRC, ROOT, SAN, _runtime


@pytest.mark.skipif(not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"), reason="HIP headers absent")
def test_delta_host_code_under_sanitizers(tmp_path):
    asan = _runtime("libasan.so")
    if asan is None:
        pytest.skip("gcc's AddressSanitizer runtime is not installed")
    objs = []
    stubs = [os.path.join(ROOT, "tests", "sanitize", s) for s in ("launch_stubs.cpp", "linear_stubs.cpp", "delta_stubs.cpp")]
    for src in ("api.cpp", "pack.cpp", "delta_api.cpp", *stubs):
        obj = str(tmp_path / (os.path.basename(src) + ".o"))
        subprocess.run(["g++", "-std=c++17", "-O1", "-fPIC", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                        "-I", os.path.join(ROOT, "include"), "-I", CSRC, *SAN, "-c", os.path.join(CSRC, src), "-o", obj], check=True)
        objs.append(obj)
    lib = str(tmp_path / "libpackmamba_delta_san.so")
    subprocess.run(["g++", "-shared", "-fPIC", *SAN, *objs, "-o", lib], check=True)
    env = dict(os.environ, LD_PRELOAD=asan, PACKMAMBA_LIB=lib, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1", OMP_NUM_THREADS="4", CUDA_VISIBLE_DEVICES="",
               HIP_VISIBLE_DEVICES="")
    tests = [f"tests/test_delta_abi.py::{t}" for t in ("test_header_and_binding_agree", "test_sizes",
                                                        "test_argument_errors_before_launch")]
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider", "-m", "not gpu", *tests],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    out = r.stdout + r.stderr
    assert "ERROR: AddressSanitizer" not in out and "runtime error:" not in out, out[-6000:]
    assert r.returncode == 0 and " passed" in out and "failed" not in out, out[-6000:]
