"""The host side of selections under AddressSanitizer and UndefinedBehaviorSanitizer, CPU only: tests/test_host_select.py against
the sanitized build of layout.cpp (see tests/test_host_sanitizers.py)."""
import os
import subprocess
import sys

import pytest

from test_host_sanitizers import ROOT, _asan_runtime


def test_selections_under_asan_and_ubsan():
    runtime = _asan_runtime()
    if runtime is None:
        pytest.skip("no AddressSanitizer runtime next to g++")
    sys.path.insert(0, ROOT)
    from paper_2602_12029_amd import build
    env = dict(os.environ)
    env.update({"PREFILLSHARE_HOST_ONLY_LIB": build.build_host_sanitized(), "LD_PRELOAD": " ".join(filter(None, [runtime, env.get("LD_PRELOAD", "")])),
                "ASAN_OPTIONS": "detect_leaks=0:abort_on_error=1:halt_on_error=1", "UBSAN_OPTIONS": "halt_on_error=1:print_stacktrace=1"})
    res = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", os.path.join(ROOT, "tests", "test_host_select.py"),
                          "-k", "not wrappers"], cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    tail = (res.stdout + res.stderr)[-4000:]
    assert res.returncode == 0, tail
    assert "passed" in res.stdout and "runtime error" not in res.stderr and "AddressSanitizer" not in res.stderr, tail
