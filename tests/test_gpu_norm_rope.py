"""qk_norm_rope and qk_norm_rope_append against the definition in 64 bits: types, widths,
rotation kinds, strided inputs, padded batches, positions without an angle or a page, and
every byte of the cache that a call must leave alone."""
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


def _torch():
    import torch
    return torch


def _gen(seed):
    g = _torch().Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _inputs(B, N, H, Hkv, d, dtype, layout, seed, strided=False):
    """q, k, v: tensors of their own, or views into one projection's output."""
    torch = _torch()
    x = torch.randn(B, N, H + 2 * Hkv, d, generator=_gen(seed), device="cuda", dtype=dtype) * 2
    parts = x.split((H, Hkv, Hkv), dim=2)
    if layout == "bhnd":
        parts = [t.transpose(1, 2) for t in parts]
    return parts if strided else [t.contiguous() for t in parts]


def _by_token(t, layout):
    return t if layout == "bnhd" else t.transpose(1, 2)


def _ints(*values):
    return _torch().tensor(values, dtype=_torch().int32, device="cuda")


SHAPES = [
    # B, N, H, Hkv, d, rotary, interleaved, layout, strided
    (1, 1, 32, 8, 128, 128, False, "bnhd", False),
    (1, 1, 1, 1, 64, 64, True, "bhnd", False),
    (3, 67, 5, 3, 128, 64, False, "bhnd", True),
    (2, 33, 7, 1, 64, 32, True, "bnhd", True),
    (2, 130, 4, 4, 128, 128, True, "bhnd", True),
    (5, 9, 16, 2, 64, 16, False, "bnhd", False),
    (2, 17, 3, 3, 128, 0, False, "bhnd", False),
    (1, 501, 9, 2, 128, 112, False, "bnhd", True),
]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("normed", [True, False])
def test_against_the_definition(qa, shape, dtype, normed):
    torch = _torch()
    B, N, H, Hkv, d, rotary, interleaved, layout, strided = shape
    dtype = getattr(torch, dtype)
    q, k, _ = _inputs(B, N, H, Hkv, d, dtype, layout, 1, strided)
    w = [(1 + 0.3 * torch.randn(d, generator=_gen(2 + i), device="cuda")).to(dtype) if normed else None
         for i in range(2)]
    cos, sin = so.rotation_table(N + 50, rotary) if rotary else (None, None)
    starts = _ints(*[(13 * b) % 50 for b in range(B)])
    out = qa.qk_norm_rope(q, k, cos=cos, sin=sin, q_weight=w[0], k_weight=w[1], eps=1e-5,
                          starts=starts, interleaved=interleaved, layout=layout)
    at = starts[:, None] + torch.arange(N, device="cuda")
    for name, x, weight, got in (("q", q, w[0], out[0]), ("k", k, w[1], out[1])):
        assert got.is_contiguous() and got.shape == x.shape and got.dtype == dtype
        want, slack = so.norm_rope(_by_token(x, layout), weight, cos, sin, at, 1e-5, interleaved)
        so.check_rounded(_by_token(got, layout), want, slack, f"{name} {shape}")


def test_small_and_large_values(qa):
    """Rows of zeros (eps alone divides them), of subnormals and of the type's largest."""
    torch = _torch()
    for dtype, values in ((torch.bfloat16, (0.0, 1e-30, 1e18, -2e4)), (torch.float16, (0.0, 6e-8, 6e4, -1.0))):
        q = torch.tensor(values, device="cuda").to(dtype)[None, :, None, None].expand(1, 4, 2, 64).contiguous()
        w = torch.full((64,), 1.5, device="cuda", dtype=dtype)
        got, _ = qa.qk_norm_rope(q, q, q_weight=w, k_weight=w, eps=1e-6, layout="bnhd")
        want, slack = so.norm_rope(q, w, None, None, torch.zeros(1, 4, device="cuda"), 1e-6, False)
        so.check_rounded(got, want, slack)
        assert (got[0, 0] == 0).all()
    x = torch.zeros(1, 2, 2, 64, device="cuda", dtype=torch.bfloat16)   # 0 / 0 without eps
    w = torch.ones(64, device="cuda", dtype=torch.bfloat16)
    assert torch.isnan(qa.qk_norm_rope(x, x, q_weight=w, eps=0.0, layout="bnhd")[0]).all()


@pytest.mark.parametrize("layout", ["bhnd", "bnhd"])
def test_padded_rows_and_positions_outside_the_table(qa, layout):
    """Rows past a sequence's count are zeros whatever they hold; a position outside the
    table gives NaN in its rows and no others."""
    torch = _torch()
    B, N, H, Hkv, d = 6, 20, 4, 2, 128
    q, k, _ = _inputs(B, N, H, Hkv, d, torch.bfloat16, layout, 3)
    counts = _ints(20, 0, 7, -3, 50, 20)
    starts = _ints(0, 5, 3, 0, 20, -4)
    cos, sin = so.rotation_table(30, 128)
    for b, n in enumerate((20, 0, 7, 0, 20, 20)):
        _by_token(q, layout)[b, n:] = math.nan
        _by_token(k, layout)[b, n:] = math.inf
    out = qa.qk_norm_rope(q, k, cos=cos, sin=sin, starts=starts, counts=counts, layout=layout)
    t = torch.arange(N, device="cuda")
    held = t < counts[:, None]
    at = starts[:, None] + t
    for x, got in zip((q, k), out):
        x, got = _by_token(x, layout), _by_token(got, layout)
        x = torch.where(held[:, :, None, None], x, 0.0)
        want, slack = so.norm_rope(x, None, cos, sin, at, 1e-6, False)
        want = torch.where(held[:, :, None, None], want, 0.0)
        so.check_rounded(got, want, slack)
    nan = torch.isnan(_by_token(out[0], layout)).all(-1).all(-1)
    assert torch.equal(nan, held & ((at < 0) | (at >= 30)))
    assert int(nan.sum()) == 4 + 10   # 6th sequence's first four, the 5th's from position 30 on


def test_starts_near_the_largest_int_do_not_wrap(qa):
    torch = _torch()
    q, k, v = _inputs(1, 8, 2, 2, 64, torch.bfloat16, "bnhd", 5)
    cos, sin = so.rotation_table(16, 64)
    big = _ints(2 ** 31 - 4)   # positions past 2^31 would be negative in 32 bits
    assert torch.isnan(qa.qk_norm_rope(q, k, cos=cos, sin=sin, starts=big, layout="bnhd")[0]).all()
    cache = torch.zeros(2, 2, 16, 64, device="cuda", dtype=torch.bfloat16)
    qa.qk_norm_rope_append(q, k, v, cache, cache.clone(), _ints(0, 1)[None], starts=big, layout="bnhd")
    assert (cache == 0).all()


def _cache(pages, Hkv, page, d, dtype, layout, seed):
    torch = _torch()
    shape = (pages, page, Hkv, d) if layout == "bnhd" else (pages, Hkv, page, d)
    if dtype == torch.float8_e4m3fn:
        return torch.randint(0, 255, shape, generator=_gen(seed), device="cuda", dtype=torch.uint8).view(dtype)
    return torch.randn(shape, generator=_gen(seed), device="cuda", dtype=dtype)


def _bits(t):
    torch = _torch()
    return t.view(torch.uint8 if t.element_size() == 1 else torch.int16)


@pytest.mark.parametrize("B,N,H,Hkv,d,rotary,page,layout,cache_layout,fp8,dtype", [
    (4, 1, 8, 2, 128, 128, 16, "bnhd", "bhnd", False, "bfloat16"),
    (3, 50, 6, 3, 64, 32, 48, "bhnd", "bnhd", False, "float16"),
    (2, 77, 4, 1, 128, 64, 16, "bnhd", "bnhd", True, "bfloat16"),
    (3, 40, 5, 5, 64, 64, 32, "bhnd", "bhnd", True, "float16"),
    (1, 300, 2, 2, 128, 0, 256, "bnhd", "bhnd", True, "float16"),
])
def test_append(qa, B, N, H, Hkv, d, rotary, page, layout, cache_layout, fp8, dtype):
    """Stored keys and values, q and the optional keys; every other byte of the cache and
    the pages that no entry in use names stay as they were."""
    torch = _torch()
    dtype = getattr(torch, dtype)
    kind = torch.float8_e4m3fn if fp8 else dtype
    q, k, v = _inputs(B, N, H, Hkv, d, dtype, layout, 7, strided=True)
    kw = (1 + 0.2 * torch.randn(d, generator=_gen(8), device="cuda")).to(dtype)
    cos, sin = so.rotation_table(N + 100, rotary) if rotary else (None, None)
    starts = _ints(*[(37 * b) % 90 for b in range(B)])
    counts = _ints(*[max(0, N - 11 * b) for b in range(B)])
    columns = (N + 100 + page - 1) // page
    table = torch.randperm(B * columns + 3, generator=torch.Generator().manual_seed(9))[:B * columns]
    table = table.to(torch.int32).view(B, columns).cuda()
    ks, vs = (0.03, 0.05) if fp8 else (1.0, 2.0)
    k_cache, v_cache = (_cache(B * columns + 3, Hkv, page, d, kind, cache_layout, 10 + i) for i in range(2))
    before = [_bits(t).clone() for t in (k_cache, v_cache)]
    k_out = torch.empty(k.shape, device="cuda", dtype=dtype)
    q_out = qa.qk_norm_rope_append(q, k, v, k_cache, v_cache, table, starts, cos=cos, sin=sin,
                                   k_weight=kw, counts=counts, k_scale=ks, v_scale=vs, k_out=k_out,
                                   layout=layout, cache_layout=cache_layout)
    plain = qa.qk_norm_rope(q, k, cos=cos, sin=sin, k_weight=kw, starts=starts, counts=counts, layout=layout)
    assert torch.equal(_bits(q_out), _bits(plain[0])) and torch.equal(_bits(k_out), _bits(plain[1]))
    at = starts[:, None] + torch.arange(N, device="cuda")
    want_k, slack_k = so.norm_rope(_by_token(k, layout), kw, cos, sin, at, 1e-6, False)
    want_v = _by_token(v, layout).double()
    limit = 448.0 if fp8 else math.inf
    written = torch.zeros(k_cache.shape[:1] + (page,), dtype=torch.bool, device="cuda")
    for name, cache, want, slack, scale in (("k", k_cache, want_k, slack_k, ks),
                                            ("v", v_cache, want_v, 0 * want_v, vs)):
        rows = cache.float() if cache_layout == "bnhd" else cache.transpose(1, 2).float()
        for b in range(B):
            n = int(counts[b])
            pos = at[b, :n].long()
            pages, inside = table[b][pos // page].long(), pos % page
            written[pages, inside] = True
            got = rows[pages, inside]
            exact = (want[b, :n] / scale).clamp(-limit, limit)
            # the fp32 product with the reciprocal: two more roundings, 2^-23
            so.check_rounded(got.to(kind), exact, slack[b, :n] / scale + 2.0 ** -23 * exact.abs(), name)
    for cache, old in zip((k_cache, v_cache), before):
        new = _bits(cache)
        keep = ~written[:, :, None, None] if cache_layout == "bnhd" else ~written[:, None, :, None]
        assert torch.equal(torch.where(keep, new, 0), torch.where(keep, old, 0))


def test_append_to_e4m3_saturates_and_keeps_nan(qa):
    torch = _torch()
    k = torch.full((1, 1, 1, 64), 1000.0, device="cuda", dtype=torch.bfloat16)
    k[..., 1], k[..., 2], k[..., 3], k[..., 4] = -1e30, math.nan, 2.0 ** -10, math.inf
    cache = torch.zeros(1, 1, 16, 64, device="cuda", dtype=torch.uint8)
    other = cache.clone()
    qa.qk_norm_rope_append(k, k, k, cache, other, _ints(0)[None], layout="bnhd")
    for c in (cache, other):
        row = c.view(torch.float8_e4m3fn).float()[0, 0, 0]
        assert row[0] == 448 and row[1] == -448 and torch.isnan(row[2])
        assert row[3] == 0.0   # 2^-10 lies between 0 and the smallest code 2^-9: to even
        assert row[4] == 448


def test_tokens_without_a_page_are_not_stored(qa):
    """Positions past the page table, pages out of range, positions without an angle."""
    torch = _torch()
    B, N, Hkv, d, page = 5, 20, 2, 64, 16
    q, k, v = _inputs(B, N, 4, Hkv, d, torch.bfloat16, "bnhd", 11)
    table = _ints(0, 1, 2, 7, -1, 3, 4, 2 ** 31 - 1, 5, 6).view(5, 2)
    starts = _ints(0, 0, 0, 20, -4)
    caches = [torch.full((7, Hkv, page, d), 9.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    qa.qk_norm_rope_append(q, k, v, *caches, table, starts, layout="bnhd")
    for cache, x in zip(caches, (k, v)):
        want = torch.full_like(cache, 9.0)
        for b, (p0, p1) in enumerate(table.tolist()):
            for t in range(N):
                at = int(starts[b]) + t
                if 0 <= at < 2 * page and 0 <= (p0, p1)[at // page] < 7:
                    want[(p0, p1)[at // page], :, at % page] = x[b, t]
        assert torch.equal(cache, want)


def test_refusals(qa):
    torch = _torch()
    q, k, v = _inputs(2, 4, 4, 2, 64, torch.bfloat16, "bnhd", 12)
    cos, sin = so.rotation_table(8, 64)
    good = dict(cos=cos, sin=sin, layout="bnhd")
    qa.qk_norm_rope(q, k, **good)
    for error, kw in [
            (ValueError, dict(cos=None)), (ValueError, dict(sin=sin[:4])), (ValueError, dict(cos=cos.cpu(), sin=sin)),
            (ValueError, dict(cos=cos.half(), sin=sin.half())), (ValueError, dict(layout="nhd")),
            (ValueError, dict(q_weight=torch.ones(64, device="cuda"))),           # not q's type
            (ValueError, dict(q_weight=torch.ones(32, device="cuda", dtype=q.dtype))),
            (ValueError, dict(starts=_ints(0))), (ValueError, dict(starts=_ints(0, 0).long())),
            (ValueError, dict(counts=_ints(0, 0).cpu())), (ValueError, dict(q_out=torch.empty_like(k))),
            (ValueError, dict(k_out=torch.empty_like(k).cpu()))]:
        with pytest.raises(error):
            qa.qk_norm_rope(q, k, **dict(good, **kw))
    with pytest.raises(TypeError):
        qa.qk_norm_rope(q.float(), k.float(), **good)
    with pytest.raises(TypeError):
        qa.qk_norm_rope(q, k.half(), **good)
    with pytest.raises(ValueError):
        qa.qk_norm_rope(q, k[:, :3], **good)
    with pytest.raises(ValueError):
        qa.qk_norm_rope(q.cpu(), k, **good)
    with pytest.raises(ValueError):      # columns not contiguous
        qa.qk_norm_rope(q.transpose(2, 3).contiguous().transpose(2, 3), k, **good)

    def status(call, code):
        with pytest.raises(qa.QmAttnError) as e:
            call()
        assert e.value.status == code
    status(lambda: qa.qk_norm_rope(q, k, cos=cos[:, :20].contiguous(), sin=sin[:, :20].contiguous(), layout="bnhd"),
           qa.QM_ERR_ROTARY)                                                   # 40 columns
    status(lambda: qa.qk_norm_rope(q, k, cos=cos[:3], sin=sin[:3], layout="bnhd"), qa.QM_ERR_ROTARY)
    status(lambda: qa.qk_norm_rope(q, k, eps=-1.0, layout="bnhd"), qa.QM_ERR_ROTARY)
    status(lambda: qa.qk_norm_rope(q, k, eps=math.nan, layout="bnhd"), qa.QM_ERR_ROTARY)
    status(lambda: qa.qk_norm_rope(q, k, q_out=q, layout="bnhd"), qa.QM_ERR_ALIAS)
    wide = torch.zeros(2, 4, 4, 68, device="cuda", dtype=torch.bfloat16)[..., :64]
    status(lambda: qa.qk_norm_rope(wide, k, layout="bnhd"), qa.QM_ERR_STRIDE)   # rows 136 bytes apart
    status(lambda: qa.qk_norm_rope(torch.zeros(2, 4, 4, 32, device="cuda", dtype=q.dtype),
                                   torch.zeros(2, 4, 2, 32, device="cuda", dtype=q.dtype), layout="bnhd"),
           qa.QM_ERR_HEADDIM)
    caches = [torch.zeros(4, 2, 16, 64, device="cuda", dtype=q.dtype) for _ in range(2)]
    table = _ints(0, 1, 2, 3).view(2, 2)
    qa.qk_norm_rope_append(q, k, v, *caches, table, **good)
    for error, kw in [(ValueError, dict(page_table=table[:1])), (ValueError, dict(page_table=table.long())),
                      (ValueError, dict(page_table=table.t())), (TypeError, dict(v_cache=caches[1].half())),
                      (TypeError, dict(k_cache=caches[0].half(), v_cache=caches[1].half())),
                      (ValueError, dict(v_cache=caches[1][:3])), (ValueError, dict(v_cache=caches[1].cpu())),
                      (ValueError, dict(cache_layout="bnhd")), (ValueError, dict(v=q)),
                      (ValueError, dict(k_cache=caches[0][..., :32].contiguous(), v_cache=caches[1][..., :32].contiguous()))]:
        args = dict(dict(good, k_cache=caches[0], v_cache=caches[1], page_table=table, v=v), **kw)
        with pytest.raises(error):
            qa.qk_norm_rope_append(q, k, **args)

    def append(**kw):
        args = dict(dict(good, k_cache=caches[0], v_cache=caches[1], page_table=table, v=v), **kw)
        return lambda: qa.qk_norm_rope_append(q, k, **args)
    status(append(k_scale=0.0), qa.QM_ERR_SCALE)
    status(append(v_scale=math.inf), qa.QM_ERR_SCALE)
    status(append(v_scale=1e-42), qa.QM_ERR_SCALE)       # its reciprocal overflows
    status(append(v_cache=caches[0]), qa.QM_ERR_ALIAS)
    odd = [torch.zeros(4, 2, 8, 64, device="cuda", dtype=q.dtype) for _ in range(2)]
    status(append(k_cache=odd[0], v_cache=odd[1]), qa.QM_ERR_PAGE)
