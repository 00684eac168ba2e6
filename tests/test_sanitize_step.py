"""The host side of steps (step_plan.cpp) under AddressSanitizer and
UndefinedBehaviorSanitizer: tests/test_step_abi.py against the sanitized
library of tests/test_sanitize_host.py.  CPU only."""
import os
import subprocess
import sys

import pytest

H = pytest.importorskip("test_sanitize_host")


@pytest.mark.skipif(not os.path.exists("/opt/rocm/include/hip/hip_runtime.h"),
                    reason="ROCm headers are needed to build the host sources")
def test_step_host_code_is_clean_under_asan_and_ubsan():
    env = dict(os.environ)
    env.update({
        "TSR_LIBRARY": H._build_sanitized(),
        "LD_PRELOAD": H._gxx_runtime("libasan.so") + ":" + H._gxx_runtime("libubsan.so"),
        "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=1",
        "UBSAN_OPTIONS": "halt_on_error=1:print_stacktrace=1",
    })
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-m", "not gpu",
                        "-p", "no:cacheprovider", "tests/test_step_abi.py"], cwd=H.ROOT, env=env,
                       capture_output=True, text=True, timeout=600)
    out = r.stdout + r.stderr
    assert "AddressSanitizer" not in out and "runtime error:" not in out, out[-6000:]
    assert r.returncode == 0, out[-6000:]
