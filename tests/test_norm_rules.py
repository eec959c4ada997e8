"""How a call of row norms is divided into launches (csrc/serving/norm_rules.h), compiled for
the host."""
from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

from paper_2506_12355_amd import build as qbuild


@pytest.fixture(scope="module")
def rows_of_launch(tmp_path_factory):
    try:
        cc = qbuild.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("rules")
    src, so = os.path.join(d, "r.hip"), os.path.join(d, "r.so")
    with open(src, "w") as f:
        f.write('#include "serving/norm_rules.h"\nextern "C" int rows(int threads) { return qm::rows_of_launch(threads); }\n')
    subprocess.run([cc, "-x", "hip", "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC",
                    "-shared", "-I", qbuild.CSRC, "-o", so, src], check=True, capture_output=True)
    return ctypes.CDLL(so).rows


@pytest.mark.parametrize("threads", [8, 16, 32, 64, 256, 512, 1024])
def test_a_launch_has_fewer_threads_than_hip_refuses(rows_of_launch, threads):
    rows = rows_of_launch(threads)
    assert rows * threads < 2 ** 32 and rows >= 2 ** 21
    # whole workgroups, whose row numbers fit an int
    assert rows % max(1, 256 // threads) == 0 and rows + 256 // threads < 2 ** 31
