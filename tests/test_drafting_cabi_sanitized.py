"""The host checks of the 8-bit cache and of drafted decoding again, against the library whose host code is
built with AddressSanitizer and UndefinedBehaviorSanitizer (as test_cabi_sanitized.py does for test_cabi.py)."""

import os
import subprocess
import sys

import pytest

from paper_2607_01308_amd import build
from test_cabi_sanitized import CHILD, ROOT

HEADERS = ("internal.h", "draft.h", "qcache.h")
SOURCES = [os.path.join(build.CSRC, x) for x in ("api.cpp", *HEADERS)] + [os.path.join(ROOT, "include", "cmerge.h")]


@pytest.mark.skipif(bool(os.environ.get("LD_PRELOAD")),
                    reason="this process already preloads a library; the sanitizer runtime "
                           "must come first")
@pytest.mark.parametrize("tests", ["test_drafting_cabi.py", "test_drafting_overlap.py", "test_empty_overlap.py",
                                   "test_qcache_cabi.py", "test_qcache_overlap.py", "test_qcache_strides.py"])
def test_host_checks_under_the_sanitizers(tests):
    lib = build.SAN_LIB
    if not os.path.exists(lib) or os.path.getmtime(lib) < max(os.path.getmtime(s) for s in SOURCES):
        build.build_sanitized()
    env = dict(os.environ, LD_PRELOAD=build.sanitizer_runtime(),
               ASAN_OPTIONS="detect_leaks=0:halt_on_error=1:abort_on_error=0",
               UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-c", CHILD, lib, os.path.join(ROOT, "tests", tests), ROOT], env=env,
                       capture_output=True, text=True, timeout=600, cwd=ROOT)
    out = r.stdout[-4000:] + r.stderr[-4000:]
    assert r.returncode == 0, out
    assert "AddressSanitizer" not in r.stderr and "runtime error" not in r.stderr, out
    assert " passed" in r.stdout, out
