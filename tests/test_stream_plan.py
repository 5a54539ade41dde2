"""The index arithmetic of streamed attention (csrc/stream.h) on the CPU, case by case against
its definition (tests/host/stream_plan.hip): the key tiles of rows under every kind of mask, and
that no key is read which no row sees; that every piece has its workgroup."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def harness(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    exe = tmp_path_factory.mktemp("plan") / "harness"
    src = os.path.join(ROOT, "tests", "host", "stream_plan.hip")
    r = subprocess.run([hipcc, "-O2", "-std=c++17", "--offload-arch=gfx950", "--cuda-host-only", src, "-o", str(exe)],
                       capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-4000:]
    return str(exe)


@pytest.mark.parametrize("what", ("tiles", "turns"))
def test_against_the_definition(harness, what):
    r = subprocess.run([harness, what], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert "cases passed" in r.stdout
