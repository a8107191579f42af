"""The largest launches of spp_paged_write and spp_paged_read (cells.cpp), built for the CPU with g++ over host stand-ins
for HIP and the kernels (tests/cpu_runtime/driver_cells_grid.cpp) and run under AddressSanitizer (+ UBSan)."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUB = os.path.join(ROOT, "tests", "cpu_runtime")
CSRC = os.path.join(ROOT, "paper_2606_29565_amd", "csrc")


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")
def test_accepted_calls_fit_a_launch(tmp_path):
    exe = str(tmp_path / "grid")
    sources = [os.path.join(CSRC, f) for f in ("runtime.cpp", "pool.cpp", "cells.cpp")] + [
        os.path.join(STUB, f) for f in ("stub_hip.cpp", "stub_kernels.cpp", "stub_paged.cpp", "driver_cells_grid.cpp")]
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-I", STUB,
                        "-DSPP_GATE_WAIT_MS=stub::gate_wait_ms", "-I", os.path.join(ROOT, "include"), "-I", CSRC, *sources,
                        "-o", exe, "-lpthread"], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0 and r.stdout.strip().endswith("OK"), (r.stdout + r.stderr)[-4000:]
