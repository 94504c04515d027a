"""The argument checks of the paged cache's entry points and the table of angles under AddressSanitizer + UndefinedBehaviorSanitizer
on the host, in a child process, as for the other entry points."""
import os
import subprocess
import sys

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_paged_boundary_tests_pass_under_host_asan_ubsan():
    from paper_2509_09754_amd import build
    if not os.path.exists(build.HIPCC):
        pytest.skip("no hipcc in this environment")
    lib = build.SAN_LIB_PATH
    sources = [os.path.join(build.CSRC, f) for f in os.listdir(build.CSRC)] + [os.path.join(ROOT, "include", "lava.h")]
    if not os.path.exists(lib) or os.path.getmtime(lib) < max(os.path.getmtime(f) for f in sources):
        lib = build.build_library(verbose=False, sanitize=True)
    runtime = build.sanitizer_runtime()
    assert os.path.isabs(runtime) and os.path.exists(runtime), runtime
    env = dict(os.environ, LD_PRELOAD=runtime, LAVA_LIBRARY=lib, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    res = subprocess.run([sys.executable, "-m", "pytest", os.path.join(ROOT, "tests", "test_paged_boundary.py"), "-q", "-x",
                          "-p", "no:cacheprovider"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    tail = (res.stdout + res.stderr)[-3000:]
    assert res.returncode == 0, tail
    assert "passed" in res.stdout and "ERROR: AddressSanitizer" not in tail and "runtime error:" not in tail, tail
