"""The serving operators' C-ABI tests against the library with its host code
under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU)."""
import os
import subprocess
import sys

import pytest

sanitizers = pytest.importorskip("test_sanitizers")
instrumented = sanitizers.instrumented


def test_serving_abi_under_asan_ubsan(instrumented):
    env, _ = instrumented
    tests = ["tests/test_abi_serving.py", "tests/test_abi_serving_limits.py"]
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-p", "no:cacheprovider", *tests],
                       capture_output=True, text=True, env=env, cwd=os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
    assert r.returncode == 0, r.stdout[-3000:] + r.stderr[:2000] + r.stderr[-1000:]
    assert " passed" in r.stdout
