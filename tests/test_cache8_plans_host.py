"""More of the host layer of the 8-bit cache under AddressSanitizer and UndefinedBehaviorSanitizer, on the CPU, built
with g++ (host code only), no GPU needed: which kernels the attention starts (tests/host/cache8_plans_test.cpp), and the
places of the accumulated weights' items (tests/host/mass_places_test.cpp)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_27128_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def run_host(tmp_path, name, sources, said):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime_api.h")):
        pytest.skip("g++ or the HIP headers are missing")
    exe = tmp_path / name
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{CSRC}", f"-I{ROOT}/include",
                        *(os.path.join(CSRC, s) for s in sources), os.path.join(ROOT, "tests", "host", name + ".cpp"),
                        "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:halt_on_error=1:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and said in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])


def test_attention_starts_a_kernel_that_gives_its_weights(tmp_path):
    run_host(tmp_path, "cache8_plans_test", ["cache8_ops.cpp"], "cache8 plans ok")


def test_every_split_of_the_weights_once(tmp_path):
    run_host(tmp_path, "mass_places_test", ["cache8_ops.cpp"], "mass places ok")
