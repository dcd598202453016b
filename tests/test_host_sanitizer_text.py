"""The host code of causal plans and of the paged cache under AddressSanitizer and UBSan (see test_host_sanitizer.py)."""
import os
import subprocess
import sys

import pytest

from paper_2606_13872_amd import build

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.slow
def test_causal_and_cache_tests_pass_under_the_sanitizers():
    if os.environ.get("SRA_HOST_LIB"):
        pytest.skip("already running on the sanitizer build")
    lib = build.build_sanitized()
    asan = subprocess.run(["g++", "-print-file-name=libasan.so"], capture_output=True, text=True).stdout.strip()
    if not os.path.isabs(asan) or not os.path.exists(asan):
        pytest.skip("no libasan for g++ here")
    env = dict(os.environ, SRA_HOST_LIB=lib, LD_PRELOAD=asan, ASAN_OPTIONS="detect_leaks=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-x", "-p", "no:cacheprovider",
                        os.path.join(ROOT, "tests", "test_causal.py"), os.path.join(ROOT, "tests", "test_cache.py")],
                       capture_output=True, text=True, env=env, cwd=ROOT, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
