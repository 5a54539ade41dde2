"""The kernels that each type's unit of streamed attention holds: those that it launches."""
import os
import re
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.parametrize("unit,wide", (("f32", 0), ("bf16", 4)))
def test_wide_kernels_where_they_are_launched(tmp_path, unit, wide):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    from paper_2607_06631_amd import build
    out = tmp_path / "stream.ll"
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    src = os.path.join(ROOT, "paper_2607_06631_amd", "csrc", f"attn_stream_{unit}.hip")
    r = subprocess.run([hipcc, *flags, "--cuda-device-only", "-emit-llvm", "-S", "-Xclang", "-disable-llvm-passes", src,
                        "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    kernels = re.findall(r"^define .*amdgpu_kernel void @_ZN3dif\d+(attn_[a-z]+_kernel)I", out.read_text(), re.M)
    assert "attn_tokens_kernel" in kernels and "attn_rows_kernel" in kernels
    assert kernels.count("attn_wide_kernel") == wide
