"""The kernels of row norms and of decoding behind a shared prefix as compiled (CPU only):
no packed fp32 instruction, no spilled VGPR, no scratch, registers for two wavefronts on each
SIMD, and no SGPR hazard at the loads that go straight into LDS, which are inline assembly."""
from __future__ import annotations

import re
import subprocess

import pytest

from paper_2506_12355_amd import build as qbuild
from tests import asm_hazards

SOURCES = {"serving/rms_norm.hip": 128, "serving/shared.hip": 256}


def _is_load_to_lds(inst):
    return inst.startswith("global_load_lds")


@pytest.mark.parametrize("debug", [False, True])
@pytest.mark.parametrize("source", sorted(SOURCES))
def test_compiled_kernels(tmp_path, source, debug, monkeypatch):
    try:
        qbuild.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    assert source in qbuild.SERVING_SOURCES
    out = str(tmp_path / "k.s")
    cmd = qbuild.compile_command(source, out, debug_sync=debug)
    assert "-fno-honor-nans" not in cmd   # these kernels tell NaNs apart
    cmd[cmd.index("-c")] = "-S"
    res = subprocess.run(cmd + ["--cuda-device-only"], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    text = open(out).read()
    kernels = list(re.finditer(r"^(_Z\w*kernel\w*):\s*(?:;.*)?$", text, flags=re.M))
    assert kernels
    assert not re.search(r"v_pk_(add|mul|fma|mov)_f32", text)
    for key, most in (("vgpr_spill_count", 0), ("private_segment_fixed_size", 0), ("vgpr_count", SOURCES[source])):
        values = [int(x) for x in re.findall(rf"\.{key}:\s+(\d+)", text)]
        assert len(values) == len(kernels) and max(values) <= most, (key, values)
    if "shared" not in source:
        return
    monkeypatch.setattr(asm_hazards, "is_direct_load", _is_load_to_lds)
    loads = 0
    for m in kernels:
        body = text[m.end():text.index(".Lfunc_end", m.end())]
        insts = asm_hazards.instructions(body)
        bad = asm_hazards.dma_sgpr_hazards_cfg(body)
        assert not bad, f"{m.group(1)}: {bad[:3]}"
        for i, inst in enumerate(insts):
            if _is_load_to_lds(inst):
                loads += 1
                assert insts[i - 1].startswith("s_nop"), (m.group(1), inst)   # M0's wait state
        # every such load has landed when the workgroup ends: a wait for all of them after the last
        last = max((i for i, inst in enumerate(insts) if _is_load_to_lds(inst)), default=None)
        if last is not None:
            assert any(re.match(r"s_waitcnt vmcnt\(0\)", x) for x in insts[last:]), m.group(1)
    assert loads
