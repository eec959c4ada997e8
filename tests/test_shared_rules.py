"""How a call behind a shared prefix is divided (csrc/serving/shared_rules.h), compiled for
the host."""
from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

from paper_2506_12355_amd import build as qbuild

WRAPPER = """
#include "serving/shared_rules.h"
extern "C" void plan(long long B, long long H, long long Hkv, int d, int es, long long limit, long long prefix, int cus,
                     int* out) {
  const qm::SharedPlan p = qm::plan_shared(B, H, Hkv, d, es, limit, prefix, cus);
  out[0] = p.rt, out[1] = p.tiles, out[2] = p.splits, out[3] = p.prefix_grid, out[4] = p.own_grid, out[5] = p.join_threads;
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
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
    lib.plan.argtypes = [ctypes.c_longlong] * 3 + [ctypes.c_int] * 2 + [ctypes.c_longlong] * 2 + [ctypes.c_int, ctypes.c_void_p]

    def call(B, H, Hkv, limit, prefix, cus=256, d=128, es=2):
        out = (ctypes.c_int * 6)()
        lib.plan(B, H, Hkv, d, es, limit, prefix, cus, out)
        return dict(zip(("rt", "tiles", "splits", "prefix_grid", "own_grid", "join_threads"), out))
    return call


@pytest.mark.parametrize("B,H,Hkv,prefix,rt", [
    (1, 16, 1, 500, 1), (1, 17, 1, 500, 2), (4, 16, 1, 9000, 2), (65, 1, 1, 9000, 8), (64, 1, 1, 9000, 2),
    (128, 1, 1, 2048, 2), (128, 1, 1, 2049, 8), (129, 1, 1, 1, 8), (1 << 20, 2, 1, 1, 8),
])
def test_rows_of_a_workgroup(plan, B, H, Hkv, prefix, rt):
    assert plan(B, H, Hkv, prefix, prefix)["rt"] == rt


def test_every_row_and_block_is_dealt_once(plan):
    """Tiles hold all rows, parts of a tile are never empty, and the launch has a workgroup
    for each (head, part, tile), found as the kernel finds it."""
    for B in (1, 2, 7, 33, 128, 1000):
        for H, Hkv in ((1, 1), (8, 8), (40, 40), (64, 8), (16, 1), (7, 1)):
            for prefix in (1, 31, 32, 33, 257, 2048, 8192, 65500, 1 << 29):
                for cus in (1, 64, 256, 304):
                    p = plan(B, H, Hkv, prefix, prefix, cus)
                    rows, blocks = B * H // Hkv, -(-prefix // 32)
                    assert (p["tiles"] - 1) * 16 * p["rt"] < rows <= p["tiles"] * 16 * p["rt"]
                    assert 1 <= p["splits"] <= max(1, -(-blocks // 8))
                    assert p["own_grid"] == 0
                    if p["prefix_grid"] <= 5000:
                        units = [w // 8 // p["tiles"] * 8 + w % 8 for w in range(p["prefix_grid"])]
                        seen = {(u, w // 8 % p["tiles"]) for w, u in enumerate(units) if u < Hkv * p["splits"]}
                        assert len(seen) == Hkv * p["splits"] * p["tiles"] == sum(u < Hkv * p["splits"] for u in units)
                    edges = {blocks * s // p["splits"] for s in range(p["splits"] + 1)}
                    assert len(edges) == p["splits"] + 1   # no part is empty


def test_own_shares(plan):
    """A workgroup of shares wherever a sequence can have tokens of its own, two a CU at most."""
    assert plan(4, 8, 2, 1000, 1000)["own_grid"] == 0
    for B in (1, 4, 1000):
        for more in (1, 20, 5000):
            p = plan(B, 8, 2, 1000 + more, 1000)
            assert 1 <= p["own_grid"] <= 512
    assert plan(1, 8, 2, 1001, 1000)["own_grid"] == 4   # (1 block + 6) of each of two rows, in fours
    assert plan(64, 64, 8, 9000, 1000)["own_grid"] == 512


def test_threads_of_the_join(plan):
    assert plan(32, 32, 8, 500, 500)["join_threads"] == 64
    assert plan(31, 32, 8, 500, 500)["join_threads"] == 256


@pytest.mark.parametrize("prefix,more,d,es,parts", [
    # 64 sequences of 64/8 heads, 32 tiles: 8 parts are a workgroup a CU, 16 two
    (8192, 0, 128, 2, 16), (8192, 64, 128, 2, 8), (8192, 8000, 128, 2, 8), (32768, 64, 128, 2, 16),
    (32768, 8000, 128, 2, 8), (32768, 2000, 128, 1, 16), (32768, 8000, 128, 1, 8), (8192, 2000, 64, 2, 8),
    (32768, 2000, 64, 2, 16),
])
def test_a_workgroup_of_each_a_cu(plan, prefix, more, d, es, parts):
    """Where own tokens are read beside the prefix's products its parts are one a CU."""
    assert plan(64, 64, 8, prefix + more, prefix, d=d, es=es)["splits"] == parts


@pytest.mark.parametrize("prefix,more,d,parts,own", [
    # 8 sequences of 64/8 heads, 16 tiles of 32 rows
    (16384, 0, 128, 32, 0), (16384, 500, 128, 16, 256), (65536, 500, 128, 32, 256), (65536, 500, 64, 32, 256),
    (1000, 500, 128, 4, 352), (4000, 4000, 128, 16, 256),
])
def test_few_rows(plan, prefix, more, d, parts, own):
    """The same rule; own tokens' workgroups are those for which the prefix's leave room."""
    p = plan(8, 64, 8, prefix + more, prefix, d=d)
    assert (p["splits"], p["own_grid"]) == (parts, own)
