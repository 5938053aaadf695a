"""The pages' entry points with arguments at the ends of their types (``tests/sanitize/pages_check.cpp``), their host code
under AddressSanitizer and UndefinedBehaviorSanitizer (no GPU)."""
import os
import shutil
import subprocess

import pytest

sanitizers = pytest.importorskip("test_sanitizers")
ROOT, CSRC, INCLUDE, SAN = sanitizers.ROOT, sanitizers.CSRC, sanitizers.INCLUDE, sanitizers.SAN


def test_pages_arguments_under_asan_ubsan(tmp_path):
    if shutil.which("g++") is None:
        pytest.skip("g++ not available")
    exe = str(tmp_path / "pages_check")
    subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", *SAN, "-I", INCLUDE, "-I", CSRC, "-I", "/opt/rocm/include",
                    os.path.join(CSRC, "pages.cpp"), os.path.join(CSRC, "host_plan.cpp"),
                    os.path.join(ROOT, "tests", "sanitize", "pages_check.cpp"), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, env=dict(os.environ, ASAN_OPTIONS="abort_on_error=1"))
    assert r.returncode == 0, r.stdout + r.stderr
    assert "pages checks passed" in r.stdout
