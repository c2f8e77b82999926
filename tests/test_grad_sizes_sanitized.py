"""tests/test_grad_sizes_cpu.py against the host-sanitized build of the library, whose plans of the gradient operators
(iso_grad_plan.cpp) are instrumented, in a child process with the sanitizer runtime preloaded."""
import os
import subprocess
import sys

import pytest

from paper_2607_19331_amd import build as B

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_plans_under_host_sanitizers():
    assert "iso_grad_plan.cpp" in B.HOST_SOURCES
    rt = B.asan_runtime()
    if rt is None or not os.path.exists(B.SANITIZED_LIB):
        pytest.skip("no host-sanitized build (the toolchain has no AddressSanitizer runtime)")
    env = dict(os.environ)
    env.update({"LD_PRELOAD": rt, "ISO_LIB_PATH": B.SANITIZED_LIB,
                "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=1",
                "UBSAN_OPTIONS": "halt_on_error=1:print_stacktrace=1"})
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "-m", "not gpu",
                        os.path.join(ROOT, "tests", "test_grad_sizes_cpu.py")], cwd=ROOT, env=env,
                       capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, (r.stdout[-3000:], r.stderr[-3000:])
    assert "passed" in r.stdout
