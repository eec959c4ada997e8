"""decode_shared keeps what decode keeps of the probabilities (bounds and checks of
test_gpu_decode_weights.py; the sums of a row's parts add at most as many terms as one
wavefront's over all of its blocks would), on each of its ways over a prefix: 16 and 32 rows
a workgroup, and 128 rows over rings in LDS.  The checking build of the library, with a
wait and a barrier more in every step of those rings, gives the same bytes."""
from __future__ import annotations

import math

import pytest

from tests import serving_oracle as so
from tests.test_gpu_decode_weights import _check

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def qa():
    import torch
    import paper_2506_12355_amd as qa
    assert torch.cuda.is_available()
    qa.load_library()
    return qa


def _ints(values):
    import torch
    return torch.tensor(values, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("prefix", [3, 40, 1500])
@pytest.mark.parametrize("B", [1, 3, 20], ids=["16 rows", "32 rows", "rings"])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
def test_weights_keep_their_bits(qa, dtype, d, cache, B, prefix):
    import torch
    dtype = getattr(torch, dtype)
    H, Hkv, page = 16, 2, 16
    g = torch.Generator(device="cuda")
    g.manual_seed(d + B)
    own = [(b * 7) % 40 for b in range(B)]
    low, shared = prefix // page, (prefix + page - 1) // page
    columns = (prefix + 40 + page - 1) // page
    table = torch.full((B, columns), -1, dtype=torch.int32, device="cuda")
    table[:, low:] = shared + torch.arange(B * (columns - low), device="cuda").view(B, -1)
    pages = shared + B * (columns - low)
    first = torch.arange(shared, device="cuda", dtype=torch.int32)
    q = torch.randn(B, H, d, generator=g, device="cuda").to(dtype)
    kind = torch.float8_e4m3fn if cache == "e4m3" else dtype
    kc, vc = ((torch.randn(pages, Hkv, page, d, generator=g, device="cuda") * (30 if cache == "e4m3" else 1)).to(kind)
              for _ in range(2))
    ks, vs = (1 / 32, 1 / 16) if cache == "e4m3" else (1.0, 1.0)
    o, _ = qa.decode_shared(q, kc, vc, table, _ints([prefix + n for n in own]), first, prefix, scale=0.125,
                            k_scale=ks, v_scale=vs)
    for b, n in enumerate(own):
        k, v = (torch.cat((so.tokens_of(c, first, prefix, "bhnd"),
                           so.tokens_of(c, table[b, low:], prefix + n - low * page, "bhnd")[prefix - low * page:])) * f
                for c, f in ((kc, ks), (vc, vs)))
        for h in range(Hkv):
            heads = slice(h * 8, h * 8 + 8)
            _check(q[b, heads], k[:, h].contiguous(), v[:, h].contiguous(), 0.125, o[b, heads], dtype, f"b={b} head {h}")


@pytest.mark.parametrize("B", [1, 4, 20], ids=["16 rows", "32 rows", "rings"])
def test_scores_too_large_for_steps_of_one(qa, B):
    """Scores past 2^24, whose fp32 steps exceed any room above the largest weight: it stays
    1, of either sign of the scale, in the prefix and in the own tokens."""
    import torch
    for dtype in (torch.float16, torch.bfloat16):
        for size in (300.0, 2000.0, 20000.0):
            q = torch.full((B, 8, 128), size, device="cuda", dtype=dtype)
            kc = torch.full((B + 5, 1, 16, 128), size, device="cuda", dtype=dtype)
            vc = torch.zeros(B + 5, 1, 16, 128, device="cuda", dtype=dtype)
            vc[:5] = 3.0
            vc[5:] = 7.0
            table = torch.full((B, 6), -1, device="cuda", dtype=torch.int32)
            table[:, 5] = 5 + torch.arange(B, device="cuda")
            first = torch.arange(5, device="cuda", dtype=torch.int32)
            for scale in (None, -0.05):
                for n, want in ((80, 3.0), (96, (80 * 3.0 + 16 * 7.0) / 96)):
                    o, lse = qa.decode_shared(q, kc, vc, table, _ints([n] * B), first, 80, scale=scale)
                    assert torch.isfinite(lse).all()
                    off = (o.double() - want).abs().max()
                    # equal weights: their sums are exact; the quotient and one rounding
                    assert float(off) <= want * (so.HALF[dtype] + 2.0 ** -20), (dtype, size, n, float(off))


def test_rows_whose_maximum_keeps_rising(qa):
    """Keys in ascending order of their scores: nearly every block raises the maximum."""
    import torch
    B, n, d = 20, 2000, 128
    for dtype in (torch.float16, torch.bfloat16):
        kc, vc = (torch.zeros(125, 1, 16, d, device="cuda", dtype=dtype) for _ in range(2))
        kc[..., 0] = torch.linspace(-8, 8, n, device="cuda").to(dtype).view(125, 1, 16)
        g = torch.Generator(device="cuda")
        g.manual_seed(3)
        vc[:] = torch.randn(125, 1, 16, d, generator=g, device="cuda").to(dtype)
        q = torch.zeros(B, 8, d, device="cuda", dtype=dtype)
        q[..., 0] = torch.linspace(0.1, 8, B * 8, device="cuda").to(dtype).view(B, 8)
        first = torch.arange(125, device="cuda", dtype=torch.int32)
        table = torch.zeros(B, 1, device="cuda", dtype=torch.int32)
        for scale in (1.0, -1.0):
            o, _ = qa.decode_shared(q, kc, vc, table, _ints([n] * B), first, n, scale=scale)
            k, v = (so.tokens_of(c, first, n, "bhnd")[:, 0].contiguous() for c in (kc, vc))
            for b in range(B):
                _check(q[b], k, v, scale, o[b], dtype, f"b={b}")


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("d", [64, 128])
def test_checking_build(qa, d, cache):
    """The rings with and without the further waits and barriers: the same bytes."""
    import torch
    from paper_2506_12355_amd import serving
    debug = qa.open_library(qa.DEBUG_LIB_PATH)
    B, H, Hkv, page, prefix = 24, 32, 4, 64, 9001
    g = torch.Generator(device="cuda")
    g.manual_seed(d)
    kind = torch.float8_e4m3fn if cache == "e4m3" else torch.bfloat16
    kc, vc = ((torch.randn(141 + B, Hkv, page, d, generator=g, device="cuda") * (30 if cache == "e4m3" else 1)).to(kind)
              for _ in range(2))
    q = torch.randn(B, H, d, generator=g, device="cuda").bfloat16()
    table = torch.full((B, 142), -1, dtype=torch.int32, device="cuda")
    table[:, 140] = 141 + torch.arange(B, device="cuda")
    table[:, 141] = 0
    first = torch.randperm(141, generator=g, device="cuda").to(torch.int32)
    args = (q, kc, vc, table, _ints([prefix + b % 5 for b in range(B)]), first, prefix)
    runs = []
    for lib in (None, debug):
        for _ in range(3):
            before = serving.load_library
            if lib is not None:
                serving.load_library = lambda: lib
            try:
                runs.append(qa.decode_shared(*args))
            finally:
                serving.load_library = before
    for o, lse in runs[1:]:
        assert torch.equal(o.view(torch.int16), runs[0][0].view(torch.int16))
        assert torch.equal(lse.view(torch.int32), runs[0][1].view(torch.int32))
