"""decode_shared with more than 64 rows a head, whose blocks go through rings in LDS: what
test_gpu_decode_shared.py checks of fewer rows, on this way over the prefix."""
from __future__ import annotations

import math

import pytest

from tests.test_gpu_decode_shared import State, _bits, _ints

pytestmark = pytest.mark.gpu

OWN = [1, None, 0, 15, 16, 17, 31, 33, 100, 257] + [None, 3, 5, 40] * 4   # 26 sequences


@pytest.fixture(scope="module")
def qa():
    import torch
    import paper_2506_12355_amd as qa
    assert torch.cuda.is_available()
    qa.load_library()
    return qa


SHAPES = [
    # H, Hkv, d, page, layout, cache, dtype
    (8, 1, 128, 16, "bhnd", "same", "bfloat16"),
    (10, 2, 64, 48, "bnhd", "same", "float16"),
    (33, 1, 128, 32, "bhnd", "e4m3", "float16"),
    (3, 1, 64, 256, "bhnd", "e4m3", "bfloat16"),
    (40, 2, 128, 64, "bnhd", "e4m3", "bfloat16"),
    (5, 1, 128, 16, "bnhd", "same", "float16"),
]


@pytest.mark.parametrize("prefix", [1, 16, 31, 32, 33, 64, 95, 100, 257, 1000, 3333])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_against_the_definition(qa, shape, prefix):
    """130 to 858 rows (at 78 and 130 rows a head, short prefixes and long ones), parts of one
    to many blocks, and last blocks that end anywhere."""
    H, Hkv, d, page, layout, cache, dtype = shape
    own = OWN if H // Hkv >= 5 else OWN * 2
    s = State(own, prefix, H, Hkv, d, page, layout, dtype, cache, seed=40)
    s.check(*s.run(qa))


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_scales(qa, scale, cache):
    s = State(OWN, 333, 8, 1, 64, 16, "bhnd", "float16", cache, seed=41, mult=2.0)
    if cache == "e4m3":   # keys and queries of the other case's size
        s.scales = (1 / 15, 1 / 15)
    s.check(*s.run(qa, scale=scale), scale=scale)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("prefix", [103, 1009])
def test_places_that_are_not_visible_do_not_matter(qa, cache, prefix):
    import torch
    s = State(OWN, prefix, 8, 1, 128, 16, "bhnd", "float16", cache, seed=42)
    o, lse = s.run(qa)
    seen = torch.zeros(s.caches[0].shape[0], 16, dtype=torch.bool, device="cuda")
    at = torch.arange(prefix, device="cuda")
    seen[s.prefix_table[at // 16].long(), at % 16] = True
    for b, n in enumerate(s.lengths):
        at = torch.arange(prefix, n, device="cuda") if n else at[:0]
        seen[s.table[b, at // 16].long(), at % 16] = True
    bad = []
    for c, junk in zip(s.caches, (0xFF, 0x7F)):
        if cache == "e4m3":
            bad.append(torch.where(seen[:, None, :, None], c.view(torch.uint8), junk).view(c.dtype).contiguous())
        else:
            bad.append(torch.where(seen[:, None, :, None], c, math.nan if junk == 0xFF else math.inf).contiguous())
    s.caches = bad
    o2, lse2 = s.run(qa)
    assert torch.equal(_bits(o2), _bits(o)) and torch.equal(_bits(lse2), _bits(lse))
    assert torch.isfinite(o2).all()


def test_a_query_that_is_no_number_stays_in_its_row(qa):
    import torch
    s = State(OWN, 700, 8, 1, 128, 16, seed=43)
    o, lse = s.run(qa)
    s.q[1] = math.nan      # a free slot
    s.q[2, 3] = math.inf
    s.q[9, 0] = math.nan
    o2, lse2 = s.run(qa)
    other = torch.ones(len(OWN), 8, dtype=torch.bool, device="cuda")
    other[2, 3] = other[9, 0] = False
    assert torch.equal(_bits(o2[other]), _bits(o[other])) and torch.equal(lse2[other], lse[other])
    assert torch.isnan(o2[9, 0]).all() and torch.isnan(lse2[9, 0])


def test_bad_lengths_and_pages_give_nan_for_their_sequence(qa):
    import torch
    s = State(OWN, 700, 8, 1, 64, 16, seed=44)
    given = list(s.lengths)
    given[3], given[4], given[5] = -1, 2 ** 31 - 1, 699
    s.table[8, 45] = s.caches[0].shape[0]
    o, lse = s.run(qa, lengths=given)
    for b in (3, 4, 5, 8):
        assert torch.isnan(o[b]).all() and torch.isnan(lse[b]).all(), b
    s.check(o, lse, sequences=[b for b in range(len(OWN)) if b not in (3, 4, 5, 8)])
    s.prefix_table[40] = -1
    o, lse = s.run(qa)
    for b, n in enumerate(OWN):
        if n is None:
            assert (o[b] == 0).all() and torch.isneginf(lse[b]).all()
        else:
            assert torch.isnan(o[b]).all() and torch.isnan(lse[b]).all(), b


def test_many_tiles_and_parts(qa):
    """More (head, tile) pairs than run at once, and few with many parts; pages past one look-up
    of 32 blocks; the same bytes from run to run."""
    import torch
    s = State([2] * 90, 2500, 40, 40, 64, 64, "bnhd", "bfloat16", seed=45)   # 90 rows: 40 tiles
    s.check(*s.run(qa), heads_every=13, sequences=(0, 44, 89))
    s = State([1, None] * 150, 1300, 64, 4, 64, 32, "bhnd", "float16", "e4m3", seed=46)   # 4800 rows a head
    runs = [s.run(qa) for _ in range(3)]
    s.check(*runs[0], sequences=(0, 1, 150, 298))
    for o, lse in runs[1:]:
        assert torch.equal(_bits(o), _bits(runs[0][0])) and torch.equal(_bits(lse), _bits(runs[0][1]))
    s = State([3] * 80, 70001, 1, 1, 128, 128, "bhnd", "bfloat16", seed=47)
    s.check(*s.run(qa), sequences=(0, 79))


def test_graphs_and_streams(qa):
    import torch
    s = State(OWN, 900, 8, 1, 128, 16, "bhnd", "bfloat16", "e4m3", seed=48, columns=90)
    other = State(OWN * 2, 400, 8, 1, 128, 16, seed=49)
    lengths = _ints(s.lengths)
    args = (s.q, *s.caches, s.table, lengths, s.prefix_table, s.prefix)
    kw = dict(k_scale=s.scales[0], v_scale=s.scales[1])
    qa.decode_shared(*args, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = qa.decode_shared(*args, **kw)
    for step in range(4):
        now = list(s.lengths)
        now[9], now[8] = now[9] - 60 * step, 0 if step % 2 else 900
        lengths.copy_(_ints(now))
        s.q.mul_(0.75)
        graph.replay()
        torch.cuda.synchronize()
        o2, lse2 = qa.decode_shared(*args, **kw)
        assert torch.equal(_bits(o), _bits(o2)) and torch.equal(_bits(lse), _bits(lse2))
    ref, ref2 = s.run(qa), other.run(qa)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        a = s.run(qa, stream=streams[0])
        b = other.run(qa, stream=streams[1])
    torch.cuda.synchronize()
    for x, y in zip((*a, *b), (*ref, *ref2)):
        assert torch.equal(_bits(x), _bits(y))


@pytest.mark.parametrize("scale", [0.2, -0.2])
@pytest.mark.parametrize("cache,dtype", [("same", "bfloat16"), ("same", "float16"), ("e4m3", "bfloat16")])
@pytest.mark.parametrize("H", [8, 2], ids=["rings", "32 rows"])
def test_rising_scores_of_one_query_do_not_reach_another(qa, H, cache, dtype, scale):
    """Queries, a free slot's among them, whose scores keep rising along the prefix: the rows
    beside them, in the same 16-row tiles, give the bytes that they give beside quiet ones."""
    import torch
    prefix, page = 1000, 16
    s = State(OWN, prefix, H, 1, 128, page, "bhnd", dtype, cache, seed=60)
    at = torch.arange(prefix, device="cuda")
    keys = s.caches[0].float()
    keys[s.prefix_table[at // page].long(), 0, at % page, 0] = torch.linspace(-200, 200, prefix, device="cuda") * (1 if cache == "e4m3" else 1 / 30)
    s.caches[0] = keys.to(s.caches[0].dtype)
    s.q[..., 0] = 0
    o, lse = s.run(qa, scale=scale)
    loud = (1, 2, 14, 17)   # 1 and 14 are free slots
    for b in loud:
        for h in range(H):
            s.q[b, h, 0] = math.copysign(3.0 + h + b / 4, scale)
    o2, lse2 = s.run(qa, scale=scale)
    rest = [b for b in range(len(OWN)) if b not in loud]
    assert torch.equal(_bits(lse2[rest]), _bits(lse[rest]))
    assert torch.equal(_bits(o2[rest]), _bits(o[rest]))
    s.check(o2, lse2, scale=scale, sequences=(2, 17))
