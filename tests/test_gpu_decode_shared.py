"""decode_shared against the definition in 64 bits (bounds of tests/serving_oracle.py: the
parts of a row are joined in fp32, as those of decode are): prefixes that end anywhere in a
block and a page, own tokens from none to long, free slots, head groups, types, and whatever
lies in places that are not visible."""
from __future__ import annotations

import math

import pytest

from tests import serving_oracle as so

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


def _bits(t):
    import torch
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


class State:
    """Caches, the prefix's table and each sequence's own (pages in random order, entries not
    in use far out of range), and queries.  own: tokens after the prefix; None: a free slot."""

    def __init__(self, own, prefix, H, Hkv, d, page, layout="bhnd", dtype="bfloat16", cache="same", seed=1, columns=0,
                 spare=3, mult=1.0):
        import torch
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)
        dtype = getattr(torch, dtype)
        self.prefix, self.layout, self.d = prefix, layout, d
        self.lengths = [0 if n is None else prefix + n for n in own]
        B, low = len(own), prefix // page
        high = [(n + page - 1) // page if n > prefix else low for n in self.lengths]
        shared = (prefix + page - 1) // page
        pages = shared + sum(h - low for h in high) + spare
        order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
        self.prefix_table = torch.cat((order[:shared], _ints([1 << 30, -7])))   # two entries too many
        self.table = torch.full((B, max(columns, max(high), 1)), -(1 << 30), dtype=torch.int32, device="cuda")
        at = shared
        for b, h in enumerate(high):
            self.table[b, low:h] = order[at:at + h - low]
            at += h - low
        self.q = (torch.randn(B, H, d, generator=g, device="cuda") * mult).to(dtype)
        shape = (pages, page, Hkv, d) if layout == "bnhd" else (pages, Hkv, page, d)
        self.caches = []
        for _ in range(2):
            x = torch.randn(shape, generator=g, device="cuda")
            self.caches.append((x * 30).to(torch.float8_e4m3fn) if cache == "e4m3" else (x * mult).to(dtype))
        self.scales = (1 / 30, 1 / 25) if cache == "e4m3" else (1.0, 1.0)

    def run(self, qa, lengths=None, **kw):
        kw = dict(dict(k_scale=self.scales[0], v_scale=self.scales[1], cache_layout=self.layout), **kw)
        return qa.decode_shared(self.q, *self.caches, self.table, _ints(self.lengths if lengths is None else lengths),
                                self.prefix_table, self.prefix, **kw)

    def tokens(self, b):
        """Keys and values of sequence b in 64 bits, [tokens, Hkv, d]."""
        import torch
        n = self.lengths[b]
        page = self.caches[0].shape[1 if self.layout == "bnhd" else 2]
        low = self.prefix // page
        out = []
        for c, f in zip(self.caches, self.scales):
            first = so.tokens_of(c, self.prefix_table, self.prefix, self.layout)
            if n > self.prefix:
                rest = so.tokens_of(c, self.table[b, low:], n - low * page, self.layout)[self.prefix - low * page:]
                first = torch.cat((first, rest))
            out.append(first * f)
        return out

    def check(self, o, lse, scale=None, heads_every=1, sequences=None):
        import torch
        scale = float(torch.tensor(self.d ** -0.5 if scale is None else scale))
        for b, n in enumerate(self.lengths):
            if sequences is not None and b not in sequences:
                continue
            if n == 0:
                assert (o[b] == 0).all() and torch.isneginf(lse[b]).all(), b
                continue
            k, v = self.tokens(b)
            G = self.q.shape[1] // k.shape[1]
            for g in range(0, k.shape[1], heads_every):
                heads = slice(g * G, (g + 1) * G)
                seen = torch.ones(G, n, dtype=torch.bool, device="cuda")
                want = so.attention_row_bounds(self.q[b, heads], k[:, g].contiguous(), v[:, g].contiguous(), scale, seen, self.q.dtype)
                so.check_attention(o[b, heads], lse[b, heads], want, f"b={b} heads={heads}")


SHAPES = [
    # H, Hkv, d, page, layout, cache: groups of one, some, sixteen and more heads
    (8, 2, 128, 16, "bhnd", "same"),
    (4, 4, 64, 16, "bnhd", "same"),
    (16, 1, 128, 64, "bnhd", "same"),
    (32, 2, 64, 48, "bhnd", "same"),
    (33, 1, 128, 32, "bhnd", "same"),
    (40, 2, 64, 16, "bnhd", "e4m3"),
    (8, 8, 128, 256, "bhnd", "e4m3"),
    (6, 2, 128, 16, "bnhd", "e4m3"),
]
OWN = [1, None, 0, 15, 16, 17, 31, 33, 100, 257]
PREFIXES = [1, 15, 16, 31, 32, 33, 100, 257, 1000]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("prefix", PREFIXES)
def test_against_the_definition(qa, shape, dtype, prefix):
    H, Hkv, d, page, layout, cache = shape
    s = State(OWN, prefix, H, Hkv, d, page, layout, dtype, cache)
    s.check(*s.run(qa))


@pytest.mark.parametrize("own", [[0], [3], [None], [None, 5], [0, 0], [None, None, None]], ids=str)
@pytest.mark.parametrize("prefix", [1, 64, 300])
def test_few_sequences(qa, own, prefix):
    """One row a head and more; no own tokens at all, no sequence at all."""
    for H, Hkv in ((2, 2), (8, 1)):
        s = State(own, prefix, H, Hkv, 128, 16)
        s.check(*s.run(qa))
        most = max(s.lengths)
        if most:
            s.check(*s.run(qa, max_length=most))


@pytest.mark.parametrize("B", [2, 3, 5, 64, 131])
def test_rows_of_several_tiles(qa, B):
    """16, 32 and more rows a head, the last tile not full; sequences past a wavefront's 64."""
    own = [None if i % 17 == 16 else (i * 37) % 90 for i in range(B)]
    for H, Hkv, d, cache in ((16, 2, 64, "same"), (7, 1, 128, "e4m3")):
        s = State(own, 333, H, Hkv, d, 32, "bnhd", "float16", cache, seed=2, columns=40)
        s.check(*s.run(qa))


def test_long_prefixes(qa):
    """Parts of one block a wavefront, and of more blocks than one look-up of pages holds."""
    s = State([5, 100, None, 0], 20000, 8, 2, 128, 64, seed=3)
    s.check(*s.run(qa))
    s = State([7] * 16 + [None, 0, 60], 40001, 64, 64, 64, 128, "bnhd", "float16", seed=4)
    s.check(*s.run(qa), heads_every=21, sequences=(0, 16, 17, 18))
    s = State([0, 1], 33000, 16, 1, 64, 16, "bhnd", "bfloat16", "e4m3", seed=5)
    s.check(*s.run(qa))


def test_long_own_tokens(qa):
    """Own tokens cut between workgroups, beside short ones and none."""
    s = State([9000, 3, 130, None, 0, 2000, 1], 70, 8, 4, 128, 16, "bnhd", seed=6)
    s.check(*s.run(qa))


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0])
def test_scales(qa, scale):
    """Negative, zero and large scales (one key then outweighs all others, of either part)."""
    s = State([77, 400, 0], 150, 4, 2, 128, 16, mult=2.0, seed=7)
    s.check(*s.run(qa, scale=scale), scale=scale)


@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_places_that_are_not_visible_do_not_matter(qa, cache):
    """NaN and infinities past the prefix and the lengths, before the own tokens of the page
    that the prefix ends in, and in pages of no one."""
    import torch
    s = State([1, None, 0, 50, 300], 103, 8, 2, 128, 16, "bhnd", "float16", cache, seed=8)
    o, lse = s.run(qa)
    seen = torch.zeros(s.caches[0].shape[0], 16, dtype=torch.bool, device="cuda")
    for j in range(103):
        seen[s.prefix_table[j // 16].long(), j % 16] = True
    for b, n in enumerate(s.lengths):
        for j in range(103, n):
            seen[s.table[b, j // 16].long(), j % 16] = True
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
    """A free slot's queries may hold anything; another row of the same tile is not affected."""
    import torch
    s = State([9, None, 20, 4], 200, 8, 2, 64, 16, seed=9)
    o, lse = s.run(qa)
    s.q[1] = math.nan
    s.q[2, 3] = math.inf
    o2, lse2 = s.run(qa)
    rows = [(b, h) for b in range(4) for h in range(8) if (b, h) != (2, 3)]
    for b, h in rows:
        assert torch.equal(_bits(o2[b, h]), _bits(o[b, h])) and torch.equal(lse2[b, h], lse[b, h]), (b, h)


def test_bad_lengths_and_pages_give_nan_for_their_sequence(qa):
    import torch
    s = State([100, 200, 64, 300, 40, None, 12], 90, 4, 2, 64, 16, seed=10)
    given = list(s.lengths)
    given[2], given[4], given[6] = -1, 2 ** 31 - 1, 89   # below 0, beyond the table, inside the prefix
    s.table[1, 8] = s.caches[0].shape[0]                 # one past the last page
    s.table[3, :5] = 2 ** 31 - 1                         # before the own tokens: not looked at
    o, lse = s.run(qa, lengths=given)
    for b in (1, 2, 4, 6):
        assert torch.isnan(o[b]).all() and torch.isnan(lse[b]).all(), b
    s.check(o, lse, sequences=(0, 3, 5))
    o, lse = s.run(qa, max_length=189)   # a bound below a length
    assert torch.isnan(o[0]).all() and not torch.isnan(o[2]).any()
    # a page of the prefix
    s.prefix_table[2] = -1
    o, lse = s.run(qa)
    for b in (0, 2, 3, 4, 6):
        assert torch.isnan(o[b]).all() and torch.isnan(lse[b]).all(), b
    assert (o[5] == 0).all() and torch.isneginf(lse[5]).all()


def test_own_tables_may_end_before_the_prefix_does(qa):
    """Sequences that hold the prefix alone need no pages of their own."""
    s = State([0, None, 0], 500, 8, 2, 128, 16, seed=11)
    s.table = s.table[:, :1].contiguous()
    s.check(*s.run(qa))
    import torch
    o, _ = s.run(qa, lengths=[500, 0, 501])
    assert torch.isnan(o[2]).all() and not torch.isnan(o[:2]).any()


def test_no_prefix_is_decode(qa):
    import torch
    s = State([100, None, 3, 257], 0, 8, 2, 128, 16, seed=12)
    o, lse = s.run(qa)
    o2, lse2 = qa.decode(s.q, *s.caches, s.table, _ints(s.lengths))
    assert torch.equal(_bits(o), _bits(o2)) and torch.equal(_bits(lse), _bits(lse2))
    o3, _ = qa.decode_shared(s.q, *s.caches, s.table, _ints(s.lengths), None, 0)
    assert torch.equal(_bits(o3), _bits(o))
    assert qa.decode_shared_workspace(s.q, s.caches[0], s.table, 0) == qa.decode_workspace(s.q, s.caches[0], s.table)


def test_pages_beyond_4_gib(qa):
    """Offsets past 32 bits: the same pages at the start and at the end of a cache of 5 GiB."""
    import torch
    pages = (5 << 30) // (16 * 8 * 128 * 2)
    g = torch.Generator(device="cuda")
    g.manual_seed(13)
    q = torch.randn(2, 16, 128, generator=g, device="cuda").bfloat16()
    kc, vc = (torch.zeros(pages, 8, 16, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    for c in (kc, vc):
        c[:9] = torch.randn(9, 8, 16, 128, generator=g, device="cuda").bfloat16()
        c[-9:] = c[:9]
    own = torch.tensor([[-1, -1, 3, 4, 5], [-1, -1, 6, 7, 8]], dtype=torch.int32, device="cuda")
    lengths, prefix = _ints([70, 41]), _ints([0, 1, 2])
    ref = qa.decode_shared(q, kc[:9].contiguous(), vc[:9].contiguous(), own, lengths, prefix, 37)
    got = qa.decode_shared(q, kc, vc, torch.where(own >= 0, own + pages - 9, -1), lengths, prefix + pages - 9, 37)
    for a, b in zip(ref, got):
        assert torch.isfinite(a).all() and torch.equal(_bits(a), _bits(b))


def test_outputs_and_workspace_are_the_callers(qa):
    import torch
    s = State([300, 10, None], 2000, 8, 2, 64, 16, seed=14)
    need = qa.decode_shared_workspace(s.q, s.caches[0], s.table, s.prefix)
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(s.q), torch.empty(3, 8, device="cuda")
    ro, rl = s.run(qa, out=o, lse=lse, workspace=ws)
    assert ro is o and rl is lse and (ws[need:] == 255).all()
    o2, lse2 = s.run(qa)
    assert torch.equal(_bits(o), _bits(o2)) and torch.equal(_bits(lse), _bits(lse2))
    s.check(o, lse)
    with pytest.raises(qa.QmAttnError) as e:
        s.run(qa, workspace=ws[:need - 1])
    assert e.value.status == qa.QM_ERR_WORKSPACE
    close = qa.decode_shared_workspace(s.q, s.caches[0], s.table, s.prefix, max_length=2000)
    assert close < need
    with pytest.raises(qa.QmAttnError) as e:
        s.run(qa, max_length=1999)
    assert e.value.status == qa.QM_ERR_PAGE


def test_graphs_and_streams(qa):
    """Captured, with lengths and tokens that change between the replays; and two calls at
    once on two streams."""
    import torch
    s = State([300, 10, None, 40], 500, 8, 2, 128, 16, seed=15, columns=80)
    lengths = _ints(s.lengths)
    other = State([30, 100, 5, None], 300, 8, 2, 128, 16, seed=16)
    args = (s.q, *s.caches, s.table, lengths, s.prefix_table, s.prefix)
    qa.decode_shared(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, lse = qa.decode_shared(*args)
    for step in range(4):
        lengths.copy_(_ints([s.lengths[0] - 60 * step, s.lengths[1], 0 if step % 2 else 500, s.lengths[3]]))
        s.q.mul_(0.75)
        graph.replay()
        torch.cuda.synchronize()
        o2, lse2 = qa.decode_shared(*args)
        assert torch.equal(_bits(o), _bits(o2)) and torch.equal(_bits(lse), _bits(lse2))
    ref = other.run(qa)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for _ in range(5):
        a = s.run(qa, stream=streams[0])
        b = other.run(qa, stream=streams[1])
    torch.cuda.synchronize()
    s.check(*a)
    for x, y in zip(b, ref):
        assert torch.equal(_bits(x), _bits(y))


def test_refusals(qa):
    import torch
    s = State([30, 40], 50, 4, 2, 64, 16, seed=17)
    kc, vc = s.caches
    good = dict(q=s.q, k_cache=kc, v_cache=vc, page_table=s.table, lengths=_ints(s.lengths), prefix_table=s.prefix_table,
                prefix_length=50)
    qa.decode_shared(**good)
    for error, kw in [
            (ValueError, dict(q=s.q[:, None])), (TypeError, dict(q=s.q.float())), (ValueError, dict(lengths=None)),
            (ValueError, dict(lengths=_ints([80]))), (ValueError, dict(page_table=s.table[:1])), (TypeError, dict(prefix_length=2.5)),
            (ValueError, dict(prefix_length=-1)), (ValueError, dict(prefix_length=2 ** 31)), (ValueError, dict(prefix_table=s.prefix_table[None])),
            (ValueError, dict(prefix_table=s.prefix_table.long())), (ValueError, dict(prefix_table=s.prefix_table.cpu())),
            (ValueError, dict(prefix_table=None)), (ValueError, dict(out=s.q[:1])), (ValueError, dict(cache_layout="hnd")),
            (ValueError, dict(workspace=torch.empty(8, device="cuda")))]:
        with pytest.raises(error):
            qa.decode_shared(**dict(good, **kw))

    def status(code, **kw):
        with pytest.raises(qa.QmAttnError) as e:
            qa.decode_shared(**dict(good, **kw))
        assert e.value.status == code
    status(qa.QM_ERR_PAGE, prefix_length=97)   # six entries of 16 tokens
    status(qa.QM_ERR_PAGE, max_length=49)
    status(qa.QM_ERR_SCALE, scale=math.inf)
    status(qa.QM_ERR_ALIAS, out=s.q)
    status(qa.QM_ERR_SHAPE, q=torch.zeros(2, 3, 64, device="cuda", dtype=s.q.dtype))
