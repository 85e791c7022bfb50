"""The host layer of the operators around the cache (csrc/cache_ops.cpp) under AddressSanitizer and
UndefinedBehaviorSanitizer, on the CPU: tests/host/cache_ops_test.cpp drives its entry points with random
batches and checks what the kernels would be told.  Built with g++ (host code only), no GPU needed."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_27128_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def test_cache_ops_host_layer(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime_api.h")):
        pytest.skip("g++ or the HIP headers are missing")
    exe = tmp_path / "cache_ops_test"
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{CSRC}", f"-I{ROOT}/include",
                        os.path.join(CSRC, "cache_ops.cpp"), os.path.join(ROOT, "tests", "host", "cache_ops_test.cpp"),
                        "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:halt_on_error=1:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "cache ops ok" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])
