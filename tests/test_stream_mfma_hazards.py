"""attn_wide_kernel issues its MFMAs as inline assembly and keeps the matrix cores'
dependency distances itself: its compiled code is scanned for the three hazard patterns
of ``tests/mfma_hazards.py``, and for spills into the key loop's registers."""
import os
import re
import shutil
import subprocess

import pytest

from tests import mfma_hazards as mh

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SRC = os.path.join(ROOT, "paper_2607_06631_amd", "csrc", "attn_stream_bf16.hip")
KERNELS = [f"_ZN3dif16attn_wide_kernelILb{sc}ELb{paged}EEEvNS_10RowsParamsIDF16bEE" for sc in (0, 1) for paged in (0, 1)]


@pytest.fixture(scope="module")
def asm(tmp_path_factory):
    hipcc = shutil.which("hipcc") or "/opt/rocm/bin/hipcc"
    if not os.path.exists(hipcc):
        pytest.skip("hipcc not available")
    from paper_2607_06631_amd import build
    out = tmp_path_factory.mktemp("asm") / "stream.s"
    flags = [f for f in build.FLAGS if f != "-fPIC"]
    r = subprocess.run([hipcc, *flags, "--cuda-device-only", "-S", SRC, "-o", str(out)], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr[-2000:]
    return out.read_text()


@pytest.mark.parametrize("kernel", KERNELS)
def test_wide_kernel_keeps_mfma_distances(asm, kernel):
    hz = mh.scan(asm, kernel)
    assert not hz, "\n".join(f"{h.kind} ({h.wait_states} wait states): {h.first} -> {h.second}" for h in hz)


@pytest.mark.parametrize("kernel", KERNELS)
def test_wide_kernel_does_not_spill(asm, kernel):
    body = asm[asm.index(f"\n{kernel}:"):]
    body = body[:body.index(".Lfunc_end")]
    assert body.count("v_mfma_f32_32x32x16_bf16") > 200
    assert not re.findall(r"scratch_(?:load|store)", body)
