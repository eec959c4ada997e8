"""How a decode call is divided (csrc/serving/decode_rules.h), compiled for the host."""
from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

from paper_2506_12355_amd import build as qbuild

WRAPPER = """
#include "serving/decode_rules.h"
extern "C" long long blocks(long long limit, long long window, long long sinks) {
  return qm::decode_blocks(limit, window, sinks);
}
extern "C" int grid(long long rows, long long blocks, int cus) {
  return qm::plan_decode(rows, blocks, cus).grid;
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    try:
        cc = qbuild.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("rules")
    src, so = os.path.join(d, "r.hip"), os.path.join(d, "r.so")
    with open(src, "w") as f:
        f.write(WRAPPER)
    subprocess.run([cc, "-x", "hip", "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC",
                    "-shared", "-I", qbuild.CSRC, "-o", so, src], check=True, capture_output=True)
    lib = ctypes.CDLL(so)
    lib.blocks.argtypes, lib.blocks.restype = [ctypes.c_longlong] * 3, ctypes.c_longlong
    lib.grid.argtypes = [ctypes.c_longlong] * 2 + [ctypes.c_int]
    return lib


def _walked(n, window, sinks):
    """The 32-token blocks that a sequence of n tokens has visible tokens in."""
    if not window:
        return -(-n // 32)
    return len({j // 32 for j in range(n) if j >= n - window or j < sinks})


@pytest.mark.parametrize("window", [0, 1, 2, 31, 32, 33, 64, 65, 100])
@pytest.mark.parametrize("sinks", [0, 1, 32, 33, 70])
def test_blocks_bound_every_length(lib, window, sinks):
    for limit in (1, 31, 32, 33, 64, 65, 130, 250):
        most = max(_walked(n, window, sinks) for n in range(limit + 1))
        bound = lib.blocks(limit, window, sinks)
        assert most <= bound <= most + 3
        assert bound <= -(-limit // 32)


@pytest.mark.parametrize("rows,blocks,whole", [
    (8, 16, True), (8, 17, False), (63, 32, False), (64, 32, True), (64, 33, False), (255, 128, False),
    (256, 128, True), (256, 129, False), (100000, 129, False), (100000, 1, True),
])
def test_plan(lib, rows, blocks, whole):
    assert lib.grid(rows, blocks, 256) == (0 if whole else 512)
