"""The host side of the speculative step's C ABI under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU only).

``csrc/mla_speculate_abi.cpp`` is plain C++: it is compiled with g++ and
``-fsanitize=address,undefined`` (no recovery) together with
``speculate_host_driver.cpp``, whose stubs stand in for the kernel launchers.  The
driver chooses split sizes for random batches, lays out workspaces, goes to the
limits of every size, and checks the launch's block order and node ranges.
"""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2609_36760_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_speculative_step_host_abi_under_sanitizers(tmp_path):
    exe = tmp_path / "speculate_driver"
    san = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-fno-omit-frame-pointer"]
    cmd = ["g++", "-std=c++17", "-O1", "-g", *san, "-D__HIP_PLATFORM_AMD__",
           "-I", os.path.join(ROCM, "include"), "-I", os.path.join(ROOT, "include"), "-I", CSRC,
           os.path.join(CSRC, "mla_speculate_abi.cpp"), os.path.join(ROOT, "tests", "speculate_host_driver.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=1:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1")
    r = subprocess.run([str(exe)], capture_output=True, text=True, env=env, timeout=300)
    print(r.stdout, r.stderr[-4000:])
    assert r.returncode == 0, r.stderr[-4000:]
    assert "all checks passed" in r.stdout
