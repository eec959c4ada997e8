"""The serving kernels as compiled (CPU only: hipcc cross-compiles the device code): no
packed fp32 instruction, no spilled VGPR, no scratch, and the registers that the planned
number of workgroups on a CU needs."""
from __future__ import annotations

import re
import subprocess

import pytest

from paper_2506_12355_amd import build as qbuild

# kernels of each source, and most VGPRs: two wavefronts on each of a CU's SIMDs (decoding:
# two workgroups of four, or one of eight)
SOURCES = {"serving/decode.hip": 256, "serving/norm_rope.hip": 128}


@pytest.mark.parametrize("source", sorted(SOURCES))
def test_compiled_kernels(tmp_path, source):
    try:
        qbuild.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    assert source in qbuild.SERVING_SOURCES
    out = str(tmp_path / "k.s")
    cmd = qbuild.compile_command(source, out)
    assert "-fno-honor-nans" not in cmd   # these kernels tell NaNs apart
    cmd[cmd.index("-c")] = "-S"
    res = subprocess.run(cmd + ["--cuda-device-only"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    text = open(out).read()
    kernels = re.findall(r"^\s+\.name:\s+(_Z\w*kernel\w*)$", text, flags=re.M)
    assert kernels
    assert not re.search(r"v_pk_(add|mul|fma|mov)_f32", text)
    for key, most in (("vgpr_spill_count", 0), ("private_segment_fixed_size", 0), ("vgpr_count", SOURCES[source])):
        values = [int(x) for x in re.findall(rf"\.{key}:\s+(\d+)", text)]
        assert len(values) == len(kernels) and max(values) <= most, (key, values)
    if "decode" in source:
        assert "v_mfma_f32_16x16x32_bf16" in text and "v_mfma_f32_16x16x32_f16" in text
