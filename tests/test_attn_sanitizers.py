"""The attention calls' host code (attn_api.cpp) under AddressSanitizer and
UndefinedBehaviorSanitizer on the CPU, over random and extreme arguments
(tests/attn_sanitize_driver.cpp)."""
import os
import shutil
import subprocess

import pytest

from test_sanitizers import CSRC, LINK, ROOT, SAN


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_attention_host_code_is_clean(tmp_path):
    if not os.path.exists("/opt/rocm/include/hip/hip_runtime_api.h"):
        pytest.skip("HIP headers not installed")
    exe = str(tmp_path / "driver")
    r = subprocess.run(["g++", "-std=c++17", "-D__HIP_PLATFORM_AMD__", "-I" + os.path.join(ROOT, "include"), "-I" + CSRC,
                        "-I/opt/rocm/include", "-Wno-deprecated-declarations"] + SAN + LINK +
                       [os.path.join(CSRC, "attn_api.cpp"), os.path.join(ROOT, "tests", "attn_sanitize_driver.cpp"),
                        "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    out = r.stdout + r.stderr
    assert r.returncode == 0 and "runtime error" not in out and "AddressSanitizer" not in out, out[-6000:]
    assert "sanitized attention checks passed" in out
