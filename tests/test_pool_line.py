"""The order of a pool's device work (pool.cpp: what its calls wait for, what the calls after them
wait for, what a failed launch leaves), built for the CPU with g++ over host stand-ins for HIP and
the kernels (tests/cpu_runtime/) and run under AddressSanitizer (+ UBSan) and ThreadSanitizer."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STUB = os.path.join(ROOT, "tests", "cpu_runtime")
CSRC = os.path.join(ROOT, "paper_2606_29565_amd", "csrc")
SANITIZERS = {"asan": ["-fsanitize=address,undefined", "-fno-omit-frame-pointer"],
              "tsan": ["-fsanitize=thread"]}
SCENARIOS = ["reserve_orders", "failed_page_copy", "failed_session_copy",
             "failed_reserve_changes_nothing", "later_work_holds_no_step",
             "more_models_than_events", "workspace_of_smaller_calls"]

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not available")


@pytest.fixture(scope="module", params=sorted(SANITIZERS))
def driver(request, tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("pool_line") / request.param)
    sources = [os.path.join(CSRC, "runtime.cpp"), os.path.join(CSRC, "pool.cpp")] + [
        os.path.join(STUB, f) for f in ("stub_hip.cpp", "stub_kernels.cpp", "driver_pool_line.cpp")]
    r = subprocess.run(["g++", "-std=c++17", "-O1", "-g", *SANITIZERS[request.param], "-I", STUB,
                        "-DSPP_GATE_WAIT_MS=stub::gate_wait_ms", "-I", os.path.join(ROOT, "include"),
                        "-I", CSRC, *sources, "-o", exe, "-lpthread"],
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-4000:]
    return exe


@pytest.mark.parametrize("scenario", SCENARIOS)
def test_pool_line(driver, scenario):
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:halt_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1",
               TSAN_OPTIONS="halt_on_error=0:exitcode=66")
    r = subprocess.run([driver, scenario], capture_output=True, text=True, timeout=120, env=env)
    assert r.returncode == 0 and r.stdout.strip().endswith("OK"), (r.stdout + r.stderr)[-6000:]
    for marker in ("WARNING: ThreadSanitizer", "ERROR: AddressSanitizer", "runtime error:"):
        assert marker not in r.stderr, r.stderr[-6000:]
