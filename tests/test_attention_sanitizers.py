"""The attention calls' host code under AddressSanitizer and UndefinedBehaviorSanitizer (CPU): the host-only tests of
include/eas_attention.h against the host-sanitized build, as tests/test_host_sanitizers.py runs the others."""
import os
import subprocess
import sys

import pytest

from test_host_sanitizers import ROOT, _asan_runtime


@pytest.mark.skipif(_asan_runtime() is None or not os.path.exists("/opt/rocm/bin/hipcc"),
                    reason="needs hipcc and the clang ASan runtime")
def test_attention_host_code_is_clean_under_asan_and_ubsan():
    sys.path.insert(0, ROOT)
    from paper_2609_31551_amd import build
    lib = build.build(verbose=False, sanitize=True)
    env = dict(os.environ, LD_PRELOAD=_asan_runtime(), EAS_LIBRARY=lib,
               ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="halt_on_error=1:print_stacktrace=1")
    r = subprocess.run([sys.executable, "-m", "pytest", "-q", "-p", "no:cacheprovider", "tests/test_attention_abi.py"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stdout[-4000:] + r.stderr[-4000:]
    assert " passed" in r.stdout and "failed" not in r.stdout
