"""More of the host layer of the operators around the cache (csrc/cache_ops.cpp) under AddressSanitizer and
UndefinedBehaviorSanitizer, on the CPU (tests/host/cache_plans_test.cpp, built with g++), and the binding's own check
of outputs.  No GPU needed."""
import os
import random
import shutil
import subprocess
from types import SimpleNamespace

import pytest

from paper_2608_27128_amd import binding

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2608_27128_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def test_cache_plans(tmp_path):
    gxx = shutil.which("g++")
    if gxx is None or not os.path.exists(os.path.join(ROCM, "include", "hip", "hip_runtime_api.h")):
        pytest.skip("g++ or the HIP headers are missing")
    exe = tmp_path / "cache_plans_test"
    r = subprocess.run([gxx, "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all",
                        "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include", f"-I{CSRC}", f"-I{ROOT}/include",
                        os.path.join(CSRC, "cache_ops.cpp"), os.path.join(ROOT, "tests", "host", "cache_plans_test.cpp"),
                        "-o", str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=0:halt_on_error=1:verify_asan_link_order=0",
               UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "cache plans ok" in r.stdout, (r.stdout[-2000:], r.stderr[-4000:])


def test_binding_refuses_outputs_whose_rows_overlap():
    """Any strides, against the rows' places listed one by one; only torch memory is touched."""
    import torch
    rng = random.Random(5)
    refused = kept = 0
    for _ in range(3000):
        heads, T, d = rng.randint(1, 7), rng.randint(1, 12), rng.choice([64, 128])
        t = d + 8 * rng.randint(0, 8) * rng.randint(0, 20)
        h = rng.choice([8 * rng.randint(0, 400), t * rng.randint(1, 4) + 8 * rng.randint(0, t // 8)])
        like = torch.empty((1, 1, 8), dtype=torch.bfloat16)
        big = torch.empty(heads * h + T * t + d, dtype=torch.bfloat16)
        out = big.as_strided((heads, T, d), (h, t, 1))
        at = sorted(a * h + b * t for a in range(heads) for b in range(T))
        if any(y - x < d for x, y in zip(at, at[1:])):
            refused += 1
            with pytest.raises(ValueError, match="overlap"):
                binding._out_rows(out, (heads, T, d), like, "out")
        else:
            kept += 1
            assert binding._out_rows(out, (heads, T, d), like, "out") is out
    assert refused > 500 and kept > 500


def test_binding_refuses_inputs_that_require_a_gradient():
    """Before anything else, so that CPU tensors show it; under no_grad the next check speaks."""
    import torch
    x = torch.zeros((2, 8, 128), dtype=torch.bfloat16)
    y = x.clone().requires_grad_()
    w = torch.ones(128, requires_grad=True)
    rope, pos = torch.zeros((8, 128), requires_grad=True), torch.zeros(8, dtype=torch.int32)

    class Cache:
        d, n_heads, n_seqs, device = 128, 2, 1, x.device
    calls = [lambda: binding.qk_norm_rope(y, None), lambda: binding.qk_norm_rope(x, y), lambda: binding.qk_norm_rope(x, x, w),
             lambda: binding.qk_norm_rope(x, x, None, w), lambda: binding.qk_norm_rope(x, x, rope=rope, positions=pos),
             lambda: binding.qk_norm_rope(x, None, q_out=y), lambda: binding.sink_attention(y, x, x, 8),
             lambda: binding.sink_attention(x, y, x, 8), lambda: binding.sink_attention(x, x, y, 8),
             lambda: binding.sink_attention(x, x, x, 8, out=y), lambda: binding.cache4_attention(y, Cache, pos),
             lambda: binding.cache4_attention(x, Cache, pos, out=y)]
    for call in calls:
        with pytest.raises(ValueError, match="gradient"):
            call()
        with torch.no_grad(), pytest.raises(ValueError, match="GPU"):
            call()


@pytest.mark.parametrize("raw", [None, lambda index: 100 + index])
def test_stream_handle_with_and_without_torch_private_name(monkeypatch, raw):
    """A torch without the undocumented function for a stream's handle gives it by its stream object."""
    c = SimpleNamespace() if raw is None else SimpleNamespace(_cuda_getCurrentRawStream=raw)
    cuda = SimpleNamespace(current_stream=lambda device: SimpleNamespace(cuda_stream=100 + device.index))
    monkeypatch.setattr(binding, "_torch", lambda: SimpleNamespace(_C=c, cuda=cuda))
    assert binding._stream(SimpleNamespace(index=3)) == 103
