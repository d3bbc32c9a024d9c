"""The split choice with node counts under AddressSanitizer and UndefinedBehaviorSanitizer
(CPU only): random batches, the largest lengths and heads, no nodes at all."""
import os
import shutil
import subprocess

import pytest

from test_speculate_abi_sanitized import CSRC, ROCM, ROOT


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_split_choice_under_sanitizers(tmp_path):
    exe = tmp_path / "tree_split_driver"
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer",
           "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(CSRC, "mla_speculate_abi.cpp"), os.path.join(ROOT, "tests", "tree_split_host_driver.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1"))
    assert r.returncode == 0, r.stderr[-4000:]
    assert "all checks passed" in r.stdout
