"""The order in which a tile walks its key blocks under a sliding window
(csrc/window_order.h), compiled for the host: every block that a wavefront's rows see is
among the steps it computes, none comes twice, and a wavefront meets them in the same order
whatever its tile's size."""
from __future__ import annotations

import ctypes
import os
import subprocess

import pytest

from paper_2506_12355_amd import build as qbuild

WRAPPER = """
#include "window_order.h"
extern "C" int walk(int row0, int rows, int N, int window, int sinks, int ascending, int* out) {
  qm::WindowOrder o;
  o.set(row0, window, sinks, ascending);
  const int end = row0 + rows < N ? row0 + rows : N, n = o.steps((end + 63) / 64);
  for (int i = 0; i < n; ++i) out[i] = ascending ? o.block_ascending(i) : o.block(i);
  return n;
}
extern "C" int steps(int row0, int n, int window, int sinks) {
  qm::WindowOrder o;
  o.set(row0, window, sinks, false);
  return o.steps(n);
}
"""


@pytest.fixture(scope="module")
def lib(tmp_path_factory):
    try:
        cc = qbuild.hipcc()
    except RuntimeError:
        pytest.skip("hipcc not available")
    d = tmp_path_factory.mktemp("order")
    src, so = os.path.join(d, "o.hip"), os.path.join(d, "o.so")
    with open(src, "w") as f:
        f.write(WRAPPER)
    subprocess.run([cc, "-x", "hip", "--cuda-host-only", "--offload-arch=gfx950", "-O1", "-std=c++17", "-fPIC",
                    "-shared", "-I", qbuild.CSRC, "-o", so, src], check=True, capture_output=True)
    return ctypes.CDLL(so)


def _walk(lib, row0, rows, N, window, sinks, ascending=0):
    out = (ctypes.c_int * 4096)()
    n = lib.walk(row0, rows, N, window, sinks, ascending, out)
    return list(out[:n])


@pytest.mark.parametrize("N", [65, 300, 700, 1500, 2049])
@pytest.mark.parametrize("window", [1, 17, 64, 65, 128, 200, 256, 257, 300, 319, 320, 321, 384, 512, 513, 700, 1500])
def test_walks(lib, N, window):
    for sinks in (0, 3, 64, 70, 300, 600):
        if window + sinks >= N:   # nothing hidden: the causal kernel's
            continue
        for qw in range(0, N, 32):   # a wavefront's first row
            seen = [b for b in range(-(-N // 64)) if 64 * b <= min(qw + 31, N - 1)
                    and (64 * b + 63 > qw - window or 64 * b < sinks)]
            met = []
            for rows in (64, 128, 256):
                row0 = qw // rows * rows
                for ascending in (0, 1):
                    walk = _walk(lib, row0, rows, N, window, sinks, ascending)
                    assert len(set(walk)) == len(walk) and all(0 <= b < -(-N // 64) for b in walk)
                    last = min(-(-min(row0 + rows, N) // 64), (qw + 31) // 64 + 1)
                    computed = walk[:lib.steps(row0, last, window, sinks)]
                    assert set(seen) <= set(computed), (sinks, qw, rows)
                    if ascending:
                        assert walk == sorted(walk)
                    elif rows >= 128:
                        met.append([b for b in computed if b in seen])
            assert met[0] == met[1], (sinks, qw)


def test_whole_blocks_come_first(lib):
    # rows 1024 to 1151 with window 512: keys 513 to 1023 before the diagonal; block 12
    # (768 to 831) is the first that rows up to 1279 see whole
    assert _walk(lib, 1024, 128, 2048, 512, 0) == [12, 13, 14, 15, 8, 9, 10, 11, 16, 17]
    assert _walk(lib, 1024, 128, 2048, 512, 4) == [12, 13, 14, 15, 0, 8, 9, 10, 11, 16, 17]
