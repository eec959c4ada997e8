"""decode against the definition in 64 bits: lengths from none to long, pages that end
inside a block, head groups, types, windows, and whatever lies in places that are not
visible; both ways of dividing the work (a workgroup a row, or equal shares and a join)."""
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


def _state(B, H, Hkv, d, lengths, page, layout, dtype, cache, seed, columns=0, spare=3, mult=1.0):
    """q, caches, page table (pages in random order, entries not in use far out of range)."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dtype = getattr(torch, dtype)
    need = [(max(0, n) + page - 1) // page for n in lengths]
    columns = max(columns, max(need), 1)
    pages = sum(need) + spare
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, columns), -(1 << 30), dtype=torch.int32, device="cuda")
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    shape = (pages, page, Hkv, d) if layout == "bnhd" else (pages, Hkv, page, d)
    q = (torch.randn(B, H, d, generator=g, device="cuda") * mult).to(dtype)
    caches = []
    for _ in range(2):
        x = torch.randn(shape, generator=g, device="cuda")
        caches.append((x * 30).to(torch.float8_e4m3fn) if cache == "e4m3" else (x * mult).to(dtype))
    return q, caches[0], caches[1], table


def _scales(cache):
    return (1 / 30, 1 / 25) if cache == "e4m3" else (1.0, 1.0)


def _check(q, kc, vc, table, lengths, o, lse, scale, window, sinks, scales, layout, heads_every=1):
    for b, heads, want in so.decode(q, kc, vc, table, lengths, scale, window, sinks, *scales, layout):
        if heads.start // max(1, heads.stop - heads.start) % heads_every:
            continue
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
LENGTHS = [1, 0, 15, 16, 17, 31, 32, 33, 64, 100, 257, 500]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("shares", [False, True], ids=["rows", "shares"])
def test_against_the_definition(qa, shape, dtype, shares):
    H, Hkv, d, page, layout, cache = shape
    B = len(LENGTHS)
    # a wide page table makes the host expect long sequences: equal shares
    state = _state(B, H, Hkv, d, LENGTHS, page, layout, dtype, cache, 1, columns=8192 // page if shares else 0)
    q, kc, vc, table = state
    scales = _scales(cache)
    most = None if shares else max(LENGTHS)
    need = qa.decode_workspace(q, kc, table, max_length=most, cache_layout=layout)
    assert (need > 0) == shares
    o, lse = qa.decode(q, kc, vc, table, _ints(LENGTHS), k_scale=scales[0], v_scale=scales[1], max_length=most, cache_layout=layout)
    assert (o[1] == 0).all() and torch_isneginf(lse[1])
    _check(q, kc, vc, table, LENGTHS, o, lse, 1 / d ** 0.5, 0, 0, scales, layout)


def torch_isneginf(t):
    import torch
    return bool(torch.isneginf(t).all())


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (16, 4), (33, 0), (64, 33), (100, 64), (300, 200), (499, 0), (501, 9), (2 ** 31 - 1, 2 ** 31 - 1)])
@pytest.mark.parametrize("shares", [False, True], ids=["rows", "shares"])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_windows(qa, window, sinks, shares, cache):
    lengths = LENGTHS + [1003]
    q, kc, vc, table = _state(len(lengths), 8, 2, 64, lengths, 16, "bhnd", "bfloat16", cache, 2,
                              columns=2000 if shares else 0)
    scales = _scales(cache)
    kw = dict(window=window, sinks=sinks, k_scale=scales[0], v_scale=scales[1])
    # a window bounds what the host expects, however wide the page table
    if shares and window <= 501:
        kw["max_length"] = 40000
    o, lse = qa.decode(q, kc, vc, table, _ints(lengths), **kw)
    _check(q, kc, vc, table, lengths, o, lse, 0.125, min(window, 10 ** 6), sinks, scales, "bhnd")


def test_windows_in_shares(qa):
    """Windows long enough that the work is dealt in shares."""
    lengths = [5000, 0, 1999, 3600, 4097]
    q, kc, vc, table = _state(5, 4, 2, 128, lengths, 32, "bnhd", "float16", "same", 3)
    for window, sinks in ((1500, 4), (2000, 700), (1531, 33)):
        assert qa.decode_workspace(q, kc, table, window=window, sinks=sinks, cache_layout="bnhd") > 0
        o, lse = qa.decode(q, kc, vc, table, _ints(lengths), window=window, sinks=sinks, cache_layout="bnhd")
        _check(q, kc, vc, table, lengths, o, lse, 128 ** -0.5, window, sinks, (1.0, 1.0), "bnhd")


@pytest.mark.parametrize("scale", [-0.3, 0.0, 1.0])
@pytest.mark.parametrize("shares", [False, True], ids=["rows", "shares"])
def test_scales(qa, scale, shares):
    """Negative, zero and large scales (one key then outweighs all others)."""
    import torch
    lengths = [77, 400]
    q, kc, vc, table = _state(2, 4, 2, 128, lengths, 16, "bhnd", "bfloat16", "same", 4, columns=500 if shares else 0, mult=2.0)
    o, lse = qa.decode(q, kc, vc, table, _ints(lengths), scale=scale)
    _check(q, kc, vc, table, lengths, o, lse, float(torch.tensor(scale)), 0, 0, (1.0, 1.0), "bhnd")


@pytest.mark.parametrize("cache", ["same", "e4m3"])
@pytest.mark.parametrize("shares", [False, True], ids=["rows", "shares"])
def test_places_that_are_not_visible_do_not_matter(qa, cache, shares):
    """NaN and infinities past the lengths, outside the window and in pages of no one."""
    import torch
    lengths = [1, 0, 15, 50, 300, 411]
    window, sinks = 120, 5
    q, kc, vc, table = _state(6, 8, 2, 128, lengths, 16, "bhnd", "float16", cache, 5, columns=1000 if shares else 0)
    scales = _scales(cache)
    kw = dict(k_scale=scales[0], v_scale=scales[1], window=window, sinks=sinks,
              max_length=16000 if shares else None)
    o, lse = qa.decode(q, kc, vc, table, _ints(lengths), **kw)
    seen = torch.zeros(kc.shape[0], 16, dtype=torch.bool, device="cuda")
    for b, n in enumerate(lengths):
        for j in range(n):
            if j >= n - window or j < sinks:
                seen[table[b, j // 16].long(), j % 16] = True
    bad = []
    for c, junk in ((kc, 0xFF), (vc, 0x7F)):
        if cache == "e4m3":
            c = torch.where(seen[:, None, :, None], c.view(torch.uint8), junk).view(c.dtype)
        else:
            c = torch.where(seen[:, None, :, None], c, float("nan") if junk == 0xFF else float("inf"))
        bad.append(c.contiguous())
    o2, lse2 = qa.decode(q, *bad, table, _ints(lengths), **kw)
    assert torch.equal(_bits(o2), _bits(o)) and torch.equal(_bits(lse2), _bits(lse))
    assert torch.isfinite(o2).all()


@pytest.mark.parametrize("shares", [False, True], ids=["rows", "shares"])
def test_bad_lengths_and_pages_give_nan_for_their_sequence(qa, shares):
    import torch
    lengths = [100, 200, 64, 300, 40, 0]
    q, kc, vc, table = _state(6, 4, 2, 64, lengths, 16, "bhnd", "bfloat16", "same", 6, columns=1000 if shares else 0)
    given = _ints([100, 200, -1, 300, 2 ** 31 - 1, 0])
    table[1, 3] = kc.shape[0]          # one past the last page
    table[3, 17] = -1
    o, lse = qa.decode(q, kc, vc, table, given)
    for b in (1, 2, 3, 4):
        # every head whose keys lie there: pages hold all heads
        assert torch.isnan(o[b]).all() and torch.isnan(lse[b]).all(), b
    _check(q[:1], kc, vc, table, lengths[:1], o[:1], lse[:1], 0.125, 0, 0, (1.0, 1.0), "bhnd")
    assert (o[5] == 0).all() and torch_isneginf(lse[5])
    # a bound below a length
    o, lse = qa.decode(q, kc, vc, table, _ints(lengths), max_length=99)
    assert torch.isnan(o[0]).all() and not torch.isnan(o[2]).any()
    # With a window of 20, sequence 3 sees tokens from 280 on, in pages 17 and 18: page 17
    # is out of range still, and page 16, in the same 32 tokens as page 17, is not needed.
    o, lse = qa.decode(q, kc, vc, table, _ints(lengths), window=20)
    assert bool(torch.isfinite(o[1]).all()) and bool(torch.isnan(o[3]).all())
    table[3, 17], table[3, 16], table[3, :9] = 0, -1, 2 ** 31 - 1
    o, lse = qa.decode(q, kc, vc, table, _ints(lengths), window=20)
    assert bool(torch.isfinite(o[3]).all())
    # nor is page 1, beside the first tokens' page 0
    table[3, 0] = 1
    o, lse = qa.decode(q, kc, vc, table, _ints(lengths), window=20, sinks=9)
    assert bool(torch.isfinite(o[3]).all())


def test_more_sequences_than_lanes(qa):
    """Shares found past the first 64 sequences, runs of empty ones among them."""
    lengths = [0] * 70 + [3000] + [0] * 63 + [17, 0, 900] + [(37 * i) % 300 for i in range(130)]
    q, kc, vc, table = _state(len(lengths), 2, 1, 64, lengths, 16, "bhnd", "bfloat16", "same", 7, columns=300)
    assert qa.decode_workspace(q, kc, table) > 0
    o, lse = qa.decode(q, kc, vc, table, _ints(lengths))
    _check(q, kc, vc, table, lengths, o, lse, 0.125, 0, 0, (1.0, 1.0), "bhnd")


def test_all_sequences_empty(qa):
    import torch
    for columns in (1, 300):
        q, kc, vc, table = _state(3, 4, 2, 64, [0, 0, 0], 16, "bhnd", "bfloat16", "same", 8, columns=columns)
        o, lse = torch.full_like(q, 7.0), torch.full((3, 4), 7.0, device="cuda")
        qa.decode(q, kc, vc, table, _ints([0, 0, 0]), out=o, lse=lse)
        assert (o == 0).all() and torch_isneginf(lse)


def test_many_short_rows_among_long_ones(qa):
    """More rows than workgroups, and rows of thousands of tokens cut many times."""
    lengths = [20000] + [130] * 90 + [9000, 1]
    q, kc, vc, table = _state(len(lengths), 16, 8, 64, lengths, 16, "bnhd", "float16", "same", 9)
    assert qa.decode_workspace(q, kc, table, cache_layout="bnhd") > 0
    o, lse = qa.decode(q, kc, vc, table, _ints(lengths), cache_layout="bnhd")
    _check(q, kc, vc, table, lengths, o, lse, 0.125, 0, 0, (1.0, 1.0), "bnhd", heads_every=3)


def test_shares_of_more_blocks_than_one_look_up(qa):
    """A wavefront looks 32 blocks' pages up at once: shares of more than 128 blocks."""
    n = 41000
    q, kc, vc, table = _state(1, 64, 64, 64, [n], 64, "bhnd", "bfloat16", "same", 10)
    o, lse = qa.decode(q, kc, vc, table, _ints([n]))
    for g in (0, 1, 31, 62, 63):
        k, v = (so.tokens_of(c[:, g:g + 1], table[0], n, "bhnd")[:, 0] for c in (kc, vc))
        import torch
        seen = torch.ones(1, n, dtype=torch.bool, device="cuda")
        want = so.attention_row_bounds(q[0, g:g + 1], k, v, 0.125, seen, q.dtype)
        so.check_attention(o[0, g:g + 1], lse[0, g:g + 1], want, f"head {g}")


def test_pages_beyond_4_gib(qa):
    """Offsets past 32 bits: the same pages at the start and at the end of a cache of 5 GiB."""
    import torch
    pages = (5 << 30) // (16 * 8 * 128 * 2)
    lengths = [40, 33]
    kc, vc = (torch.zeros(pages, 8, 16, 128, device="cuda", dtype=torch.bfloat16) for _ in range(2))
    g = torch.Generator(device="cuda")
    g.manual_seed(11)
    q = torch.randn(2, 16, 128, generator=g, device="cuda").bfloat16()
    low = torch.arange(6, device="cuda", dtype=torch.int32).view(2, 3)
    high = pages - 6 + low
    for c in (kc, vc):
        c[:6] = torch.randn(6, 8, 16, 128, generator=g, device="cuda").bfloat16()
        c[-6:] = c[:6]
    ref = qa.decode(q, kc[:6].contiguous(), vc[:6].contiguous(), low, _ints(lengths))
    got = qa.decode(q, kc, vc, high, _ints(lengths))
    for a, b in zip(ref, got):
        assert torch.equal(_bits(a), _bits(b))
    # and written there
    k = torch.randn(2, 1, 8, 128, generator=g, device="cuda").bfloat16()
    qa.qk_norm_rope_append(q[:, None], k, -k, kc, vc, high, _ints(lengths), layout="bnhd")
    for b, n in enumerate(lengths):
        assert torch.equal(kc[high[b, n // 16].long(), :, n % 16], k[b, 0])
        assert torch.equal(vc[high[b, n // 16].long(), :, n % 16], -k[b, 0])
        assert (kc[low[b, n // 16].long(), :, n % 16] != k[b, 0]).any()


def test_outputs_and_workspace_are_the_callers(qa):
    import torch
    lengths = [3000, 10]
    q, kc, vc, table = _state(2, 4, 2, 64, lengths, 16, "bhnd", "bfloat16", "same", 12)
    need = qa.decode_workspace(q, kc, table)
    assert need > 0 and need == qa.decode_workspace(q, kc, table, max_length=3000)
    assert qa.decode_workspace(q, kc, table, max_length=500) == 0
    ws = torch.full((need + 64,), 255, dtype=torch.uint8, device="cuda")
    o, lse = torch.empty_like(q), torch.empty(2, 4, device="cuda")
    ro, rl = qa.decode(q, kc, vc, table, _ints(lengths), out=o, lse=lse, workspace=ws)
    assert ro is o and rl is lse and (ws[need:] == 255).all()
    o2, lse2 = qa.decode(q, kc, vc, table, _ints(lengths))
    assert torch.equal(_bits(o), _bits(o2)) and torch.equal(_bits(lse), _bits(lse2))
    with pytest.raises(qa.QmAttnError) as e:
        qa.decode(q, kc, vc, table, _ints(lengths), workspace=ws[:need - 1])
    assert e.value.status == qa.QM_ERR_WORKSPACE


def test_refusals(qa):
    import torch
    lengths = [30, 40]
    q, kc, vc, table = _state(2, 4, 2, 64, lengths, 16, "bhnd", "bfloat16", "same", 13)
    lens = _ints(lengths)
    good = dict(q=q, k_cache=kc, v_cache=vc, page_table=table, lengths=lens)
    qa.decode(**good)
    for error, kw in [
            (ValueError, dict(q=q[:, None])), (ValueError, dict(q=q.cpu())), (TypeError, dict(q=q.float())),
            (ValueError, dict(q=q.transpose(0, 1))), (TypeError, dict(q=q.half())), (ValueError, dict(lengths=lens[:1])),
            (ValueError, dict(lengths=lens.long())), (ValueError, dict(lengths=None)), (ValueError, dict(lengths=lens.cpu())),
            (ValueError, dict(page_table=table[:1])), (ValueError, dict(page_table=table[0])),
            (ValueError, dict(v_cache=vc[:2])), (TypeError, dict(v_cache=vc.half())), (ValueError, dict(k_cache=kc.transpose(1, 2))),
            (ValueError, dict(cache_layout="hnd")), (ValueError, dict(window=0)), (ValueError, dict(window=-3)),
            (ValueError, dict(window=2 ** 32 + 5)), (ValueError, dict(max_length=2 ** 31)), (TypeError, dict(window=2.5)),
            (ValueError, dict(out=torch.empty_like(q).cpu())), (ValueError, dict(lse=torch.empty(2, 3, device="cuda"))),
            (ValueError, dict(workspace=torch.empty(8, device="cuda"))),
            (ValueError, dict(workspace=torch.empty(10 ** 7, dtype=torch.uint8)))]:
        with pytest.raises(error):
            qa.decode(**dict(good, **kw))

    def status(code, **kw):
        with pytest.raises(qa.QmAttnError) as e:
            qa.decode(**dict(good, **kw))
        assert e.value.status == code
    status(qa.QM_ERR_WINDOW, sinks=-1)
    status(qa.QM_ERR_PAGE, max_length=0)
    status(qa.QM_ERR_SHAPE, q=torch.zeros(2, 3, 64, device="cuda", dtype=q.dtype))   # 3 heads over 2
    status(qa.QM_ERR_SCALE, scale=math.inf)
    status(qa.QM_ERR_SCALE, v_scale=math.nan)
    status(qa.QM_ERR_SCALE, scale=3e38, k_scale=3.0)
    status(qa.QM_ERR_ALIAS, out=q)
    narrow = [torch.zeros(2, 2, 16, 32, device="cuda", dtype=q.dtype) for _ in range(2)]
    status(qa.QM_ERR_HEADDIM, q=torch.zeros(2, 4, 32, device="cuda", dtype=q.dtype), k_cache=narrow[0], v_cache=narrow[1])
    odd = [torch.zeros(2, 2, 24, 64, device="cuda", dtype=q.dtype) for _ in range(2)]
    status(qa.QM_ERR_PAGE, k_cache=odd[0], v_cache=odd[1])
