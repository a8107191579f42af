"""Host code of the caches of 8-bit codes and of the log probabilities (pool.cpp, cells.cpp, logprobs.cpp:
checks, what is handed on to the kernels, copies that carry scales), built for the CPU with g++ over
host stand-ins for HIP and the kernels (tests/cpu_runtime/) and run under AddressSanitizer (+ UBSan)
and ThreadSanitizer."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUB = os.path.join(ROOT, "tests", "cpu_runtime")
CSRC = os.path.join(ROOT, "paper_2606_29565_amd", "csrc")
SANITIZERS = {"asan": ["-fsanitize=address,undefined", "-fno-omit-frame-pointer"],
              "tsan": ["-fsanitize=thread"]}

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")


@pytest.mark.parametrize("san", sorted(SANITIZERS))
def test_codes_scenarios_clean_under_sanitizer(tmp_path, san):
    exe = str(tmp_path / f"codes_{san}")
    sources = [os.path.join(CSRC, f) for f in ("runtime.cpp", "pool.cpp", "cells.cpp", "logprobs.cpp")] + [
        os.path.join(STUB, f) for f in ("stub_hip.cpp", "stub_kernels.cpp", "driver_codes.cpp")]
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", *SANITIZERS[san], "-I", STUB,
                        "-DSPP_GATE_WAIT_MS=stub::gate_wait_ms", "-I", os.path.join(ROOT, "include"),
                        "-I", CSRC, *sources, "-o", exe, "-lpthread"],
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1",
               TSAN_OPTIONS="halt_on_error=0:exitcode=66")
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600, env=env)
    assert r.returncode == 0 and r.stdout.strip().endswith("OK"), (r.stdout + r.stderr)[-6000:]
    for marker in ("WARNING: ThreadSanitizer", "ERROR: AddressSanitizer", "runtime error:"):
        assert marker not in r.stderr, r.stderr[-6000:]
