"""The streamed-generation entry points' host side under AddressSanitizer and
UndefinedBehaviorSanitizer (tests/host/stream_harness.cpp): operands that end with their last
element, tables with entries out of range, workspaces of exactly the size asked for, calls
without queries or keys, a launch that fails."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/llvm/bin/clang++"


@pytest.mark.skipif(not os.path.exists(CLANG), reason="ROCm clang++ not installed")
def test_stream_entry_points_under_asan_and_ubsan(tmp_path):
    exe = tmp_path / "harness"
    cmd = [CLANG, "-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", "-fsanitize=address,undefined",
           "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
           os.path.join(ROOT, "paper_2607_06631_amd", "csrc", "stream.cpp"),
           os.path.join(ROOT, "tests", "host", "stream_harness.cpp"), "-o", str(exe)]
    r = subprocess.run(cmd, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=300,
                       env=dict(os.environ, ASAN_OPTIONS="detect_leaks=1"))
    assert r.returncode == 0, (r.stdout[-2000:], r.stderr[-6000:])
    assert "all cases passed" in r.stdout
    shutil.rmtree(tmp_path, ignore_errors=True)
