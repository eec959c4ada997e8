"""qk_norm_rope and qk_norm_rope_append with positions of several axes, against the
definition in 64 bits (bounds as for one axis, tests/serving_oracle.py), and against the
calls of one axis, byte for byte, where all axes go together."""
from __future__ import annotations

import math

import pytest

from tests import serving_oracle as so

pytestmark = pytest.mark.gpu

ROWS = 90   # of the angles' table


@pytest.fixture(scope="module")
def qa():
    import torch
    import paper_2506_12355_amd as qa
    assert torch.cuda.is_available()
    qa.load_library()
    return qa


def _gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _bits(t):
    import torch
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def _by_token(t, layout):
    return t if layout == "bnhd" else t.transpose(1, 2)


def _axes_of(kind, pairs, count):
    """The axis of each pair: a run each, in turn, or any."""
    if kind == "runs":
        return [j * count // pairs for j in range(pairs)]
    if kind == "turns":
        return [j % count for j in range(pairs)]
    return [(j * j + j // 5) % count for j in range(pairs)]


def _define(x, weight, cos, sin, positions, axes, eps, interleaved):
    """x [B, N, heads, d] in 64 bits, positions [A, B, N]; (y, bound on fp32 errors)."""
    import torch
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * weight.double()
    half = cos.shape[1]
    out, size = y.clone(), y.abs()
    bad = torch.zeros_like(positions[0], dtype=torch.bool)
    for a in set(axes):
        bad |= (positions[a] < 0) | (positions[a] >= cos.shape[0])
    for j, a in enumerate(axes):
        at = positions[a].clamp(0, cos.shape[0] - 1).long()
        c, s = cos.double()[at, j][:, :, None], sin.double()[at, j][:, :, None]
        c0, c1 = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        p, q = y[..., c0], y[..., c1]
        out[..., c0], out[..., c1] = p * c - q * s, q * c + p * s
        size[..., c0] = size[..., c1] = p.abs() + q.abs()
    out[bad] = math.nan
    return out, 2.0 ** -18 * size


def _inputs(B, N, H, Hkv, d, dtype, layout, seed):
    import torch
    x = torch.randn(B, N, H + 2 * Hkv, d, generator=_gen(seed), device="cuda", dtype=dtype) * 2
    parts = x.split((H, Hkv, Hkv), dim=2)
    return [t.transpose(1, 2) for t in parts] if layout == "bhnd" else list(parts)


def _positions(A, B, N, seed, low=0, high=ROWS):
    import torch
    return torch.randint(low, high, (A, B, N), generator=_gen(seed), device="cuda", dtype=torch.int32)


SHAPES = [
    # B, N, H, Hkv, d, rotary, interleaved, layout, axes, kind
    (1, 1, 32, 8, 128, 128, False, "bnhd", 3, "runs"),
    (3, 67, 5, 3, 128, 64, False, "bhnd", 3, "turns"),
    (2, 33, 7, 1, 64, 32, True, "bnhd", 4, "any"),
    (2, 130, 4, 4, 128, 128, True, "bhnd", 2, "turns"),
    (5, 9, 16, 2, 64, 16, False, "bnhd", 4, "runs"),
    (1, 501, 9, 2, 128, 112, False, "bnhd", 3, "any"),
    (2, 40, 4, 2, 64, 64, False, "bhnd", 1, "runs"),
    (1, 65, 3, 1, 128, 128, False, "bhnd", 4, "any"),
]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=str)
@pytest.mark.parametrize("normed", [True, False])
def test_against_the_definition(qa, shape, dtype, normed):
    import torch
    B, N, H, Hkv, d, rotary, interleaved, layout, count, kind = shape
    dtype = getattr(torch, dtype)
    q, k, _ = _inputs(B, N, H, Hkv, d, dtype, layout, 1)
    w = [(1 + 0.3 * torch.randn(d, generator=_gen(2 + i), device="cuda")).to(dtype) if normed else None for i in range(2)]
    cos, sin = so.rotation_table(ROWS, rotary)
    positions, axes = _positions(count, B, N, 4), _axes_of(kind, rotary // 2, count)
    out = qa.qk_norm_rope(q, k, cos=cos, sin=sin, q_weight=w[0], k_weight=w[1], eps=1e-5, positions=positions,
                          axes=None if count == 1 else axes, interleaved=interleaved, layout=layout)
    for name, x, weight, got in (("q", q, w[0], out[0]), ("k", k, w[1], out[1])):
        assert got.is_contiguous() and got.shape == x.shape and got.dtype == dtype
        want, slack = _define(_by_token(x, layout), weight, cos, sin, positions, axes, 1e-5, interleaved)
        so.check_rounded(_by_token(got, layout), want, slack, f"{name} {shape}")


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("cache", ["same", "e4m3"])
def test_axes_that_go_together_are_one_axis(qa, interleaved, cache):
    """The results of the calls with starts, cached ones among them: each within the bounds
    of the definition (the two kernels are compiled apart, and in a cos - b sin either product
    may be the one that is not rounded before the sum, so that bytes may differ), and with or
    without a cache the same bytes."""
    import torch
    B, N, H, Hkv, d = 3, 50, 8, 2, 128
    q, k, v = _inputs(B, N, H, Hkv, d, torch.bfloat16, "bnhd", 5)
    cos, sin = so.rotation_table(ROWS, d)
    starts = torch.tensor([0, 40, 7], dtype=torch.int32, device="cuda")
    counts = torch.tensor([50, 13, 0], dtype=torch.int32, device="cuda")
    positions = (starts[:, None] + torch.arange(N, device="cuda", dtype=torch.int32)).expand(3, B, N).contiguous()
    kind = torch.float8_e4m3fn if cache == "e4m3" else torch.bfloat16
    table = torch.randperm(18, generator=_gen(6), device="cuda").to(torch.int32).view(3, 6)
    results = []
    for more in (dict(), dict(positions=positions, axes=_axes_of("turns", 64, 3))):
        caches = [torch.zeros(18, Hkv, 16, d, device="cuda", dtype=torch.bfloat16).to(kind) for _ in range(2)]
        k_out = torch.empty(B, N, Hkv, d, device="cuda", dtype=torch.bfloat16)
        q_out = qa.qk_norm_rope_append(q, k, v, *caches, table, starts, cos=cos, sin=sin, counts=counts, k_scale=0.1, v_scale=0.2,
                                       interleaved=interleaved, k_out=k_out, layout="bnhd", **more)
        plain = qa.qk_norm_rope(q, k, cos=cos, sin=sin, counts=counts, interleaved=interleaved, layout="bnhd",
                                **(more or dict(starts=starts)))
        assert torch.equal(_bits(plain[0]), _bits(q_out)) and torch.equal(_bits(plain[1]), _bits(k_out))
        results.append([q_out, k_out, *caches])
    held = (torch.arange(N, device="cuda") < counts[:, None])[:, :, None, None]
    for i, x in enumerate((q, k)):
        want, slack = _define(x, None, cos, sin, positions, [0] * 64, 1e-6, interleaved)
        for got in results:
            so.check_rounded(got[i], torch.where(held, want, 0.0), slack)
    for got in results:
        for cache, rows, f in ((got[2], _define(k, None, cos, sin, positions, [0] * 64, 1e-6, interleaved), 0.1),
                               (got[3], (v.double(), torch.zeros_like(v, dtype=torch.float64)), 0.2)):
            for b, n in enumerate((50, 13, 0)):
                at = (starts[b] + torch.arange(n, device="cuda")).long()
                stored = cache.float()[table[b].long()].transpose(1, 2).flatten(0, 1)[at]
                want, slack = (t[b, :n] / f for t in rows)
                # the quotient's reciprocal and product: two fp32 roundings
                so.check_rounded(stored.to(cache.dtype), want.clamp(-448, 448) if cache.dtype != torch.bfloat16 else want,
                                 slack + 2.0 ** -22 * want.abs())
    # what no token was written to stays zero
    assert torch.equal(results[0][3].view(torch.uint8), results[1][3].view(torch.uint8))
    assert torch.equal(results[0][2].float() == 0, results[1][2].float() == 0)


def test_places_in_the_cache_are_not_the_rotations(qa):
    """Keys turned by their positions, stored at starts + t; rows past the counts and tokens
    whose positions have no angle leave the cache as it was."""
    import torch
    B, N, H, Hkv, d, page = 4, 21, 4, 2, 64, 16
    q, k, v = _inputs(B, N, H, Hkv, d, torch.float16, "bhnd", 7)
    cos, sin = so.rotation_table(ROWS, d)
    axes = _axes_of("runs", 32, 3)
    positions = _positions(3, B, N, 8)
    positions[1, 0, 4] = -1
    positions[2, 3, 20] = ROWS
    positions[0, 2, 10] = 2 ** 31 - 1
    counts = torch.tensor([21, 0, 11, 30], dtype=torch.int32, device="cuda")
    positions[:, 2, 11:] = -5   # not looked at
    starts = torch.tensor([30, 3, 0, 11], dtype=torch.int32, device="cuda")
    table = torch.randperm(20, generator=_gen(9), device="cuda")[:16].to(torch.int32).view(4, 4)
    caches = [torch.randn(20, Hkv, page, d, generator=_gen(10 + i), device="cuda").half() for i in range(2)]
    before = [c.clone() for c in caches]
    k_out = torch.empty(B, Hkv, N, d, device="cuda", dtype=torch.float16)
    q_out = qa.qk_norm_rope_append(q, k, v, *caches, table, starts, cos=cos, sin=sin, counts=counts, positions=positions,
                                   axes=axes, k_out=k_out)
    held = torch.arange(N, device="cuda") < counts[:, None]
    for x, got in ((q, q_out), (k, k_out)):
        want, slack = _define(_by_token(x, "bhnd"), None, cos, sin, positions, axes, 1e-6, False)
        want = torch.where(held[:, :, None, None], want, 0.0)
        so.check_rounded(_by_token(got, "bhnd"), want, slack)
    nan = torch.isnan(k_out).any(1).any(-1)
    assert nan.nonzero().tolist() == [[0, 4], [2, 10], [3, 20]]
    for b in range(B):
        for t in range(N):
            at = int(starts[b]) + t
            if held[b, t] and not nan[b, t] and at < 64:
                p = int(table[b, at // page])
                before[0][p, :, at % page], before[1][p, :, at % page] = k_out[b, :, t], v[b, :, t]
    for a, b in zip(caches, before):
        assert torch.equal(_bits(a), _bits(b))


def test_axes_that_no_pair_has_are_not_looked_at(qa):
    import torch
    q, k, _ = _inputs(2, 17, 4, 2, 128, torch.bfloat16, "bnhd", 12)
    cos, sin = so.rotation_table(ROWS, 128)
    positions = _positions(4, 2, 17, 13)
    axes = [1 if j < 40 else 3 for j in range(64)]
    ref = qa.qk_norm_rope(q, k, cos=cos, sin=sin, positions=positions, axes=axes, layout="bnhd")
    positions[0], positions[2] = -1, 2 ** 31 - 1
    got = qa.qk_norm_rope(q, k, cos=cos, sin=sin, positions=positions, axes=axes, layout="bnhd")
    assert torch.isfinite(ref[0]).all()
    for a, b in zip(ref, got):
        assert torch.equal(_bits(a), _bits(b))


@pytest.mark.parametrize("layout", ["bnhd", "bhnd"])
@pytest.mark.parametrize("H,Hkv,d", [(32, 8, 128), (37, 9, 128), (40, 17, 64), (3, 1, 128)])
def test_large_calls(qa, layout, H, Hkv, d):
    """Calls in which a lane takes several heads of a token (and those of few heads, in which it
    does not), odd counts of heads and tokens, padded rows and positions without an angle
    among them: every element, and every byte of the cache."""
    import torch
    B, N, page = 3, 1203, 16
    q, k, v = _inputs(B, N, H, Hkv, d, torch.bfloat16, layout, 30)
    cos, sin = so.rotation_table(ROWS, d)
    axes = _axes_of("any", d // 2, 3)
    positions = _positions(3, B, N, 31)
    positions[2, 1, 700] = ROWS
    counts = torch.tensor([1203, 1000, 5], dtype=torch.int32, device="cuda")
    starts = torch.tensor([3, 0, 40], dtype=torch.int32, device="cuda")
    table = torch.randperm(3 * 76, generator=_gen(32), device="cuda").to(torch.int32).view(3, 76)
    w = (1 + 0.3 * torch.randn(d, generator=_gen(33), device="cuda")).bfloat16()
    caches = [torch.full((3 * 76, Hkv, page, d), 7.0, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    k_out = torch.empty(k.shape, device="cuda", dtype=torch.bfloat16)
    kw = dict(cos=cos, sin=sin, q_weight=w, k_weight=w, counts=counts, positions=positions, axes=axes, layout=layout)
    q_out = qa.qk_norm_rope_append(q, k, v, *caches, table, starts, k_out=k_out, **kw)
    held = (torch.arange(N, device="cuda") < counts[:, None])[:, :, None, None]
    for x, got in ((q, q_out), (k, k_out)):
        want, slack = _define(_by_token(x, layout), w, cos, sin, positions, axes, 1e-6, False)
        so.check_rounded(_by_token(got, layout), torch.where(held, want, 0.0), slack)
    for a, b in zip(qa.qk_norm_rope(q, k, **kw), (q_out, k_out)):
        assert torch.equal(_bits(a), _bits(b))
    want = [torch.full_like(c, 7.0) for c in caches]
    for b, n in enumerate(counts.tolist()):
        t = torch.tensor([i for i in range(n) if (b, i) != (1, 700)], device="cuda")
        at = t + int(starts[b])
        for c, rows in zip(want, (k_out, v)):
            c.transpose(1, 2)[table[b, at // page].long(), at % page] = _by_token(rows, layout)[b, t]
    for c, e in zip(caches, want):
        assert torch.equal(_bits(c), _bits(e))


def test_captured(qa):
    """The axes of the pairs are read at the call; replays follow the positions."""
    import torch
    q, k, _ = _inputs(2, 30, 4, 2, 128, torch.bfloat16, "bnhd", 14)
    cos, sin = so.rotation_table(ROWS, 128)
    positions, axes = _positions(3, 2, 30, 15), tuple(_axes_of("any", 64, 3))
    kw = dict(cos=cos, sin=sin, positions=positions, axes=axes, layout="bnhd")
    qa.qk_norm_rope(q, k, **kw)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = qa.qk_norm_rope(q, k, **kw)
    for i in range(4):
        positions.copy_(_positions(3, 2, 30, 16 + i))
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, qa.qk_norm_rope(q, k, **kw)):
            assert torch.equal(_bits(a), _bits(b))


def test_refusals(qa):
    import torch
    q, k, v = _inputs(2, 16, 4, 2, 64, torch.bfloat16, "bnhd", 20)
    cos, sin = so.rotation_table(ROWS, 64)
    at = _positions(3, 2, 16, 21)
    axes = _axes_of("runs", 32, 3)
    good = dict(cos=cos, sin=sin, positions=at, axes=axes, layout="bnhd")
    cache = [torch.zeros(4, 2, 16, 64, device="cuda", dtype=torch.bfloat16) for _ in range(2)]
    table = torch.arange(4, device="cuda", dtype=torch.int32).view(2, 2)
    qa.qk_norm_rope(q, k, **good)
    for kw in (dict(positions=at[:, :1]), dict(positions=at[0]), dict(positions=at.long()), dict(positions=at.cpu()),
               dict(positions=at.transpose(1, 2)), dict(positions=at.repeat(2, 1, 1)), dict(axes=None), dict(axes=axes[:31]),
               dict(axes=[3] * 32), dict(axes=[-1] * 32), dict(positions=None)):
        for call in (lambda **a: qa.qk_norm_rope(q, k, **a), lambda **a: qa.qk_norm_rope_append(q, k, v, *cache, table, **a)):
            with pytest.raises(ValueError):
                call(**dict(good, **kw))
    with pytest.raises(TypeError):
        qa.qk_norm_rope(q, k, **dict(good, axes=[0.5] * 32))
    with pytest.raises(ValueError, match="starts"):
        qa.qk_norm_rope(q, k, starts=torch.zeros(2, dtype=torch.int32, device="cuda"), **good)
    with pytest.raises(qa.QmAttnError) as e:
        qa.qk_norm_rope(q, k, positions=at, axes=[], layout="bnhd")   # no rotation
    assert e.value.status == qa.QM_ERR_ROTARY


@pytest.mark.parametrize("interleaved", [False, True])
@pytest.mark.parametrize("layout", ["bnhd", "bhnd"])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("d,N", [(128, 40), (128, 750), (64, 1500), (128, 2000)])
def test_one_rotation_whatever_the_call(qa, d, N, dtype, layout, interleaved):
    """The same keys and queries at the same positions give the same bytes from the call of one
    axis and from that of several, and with or without a cache: in small calls, in large
    ones, and in those that are large for the values that they cache alone."""
    import torch
    H, Hkv, page = 32, 8, 16
    dtype = getattr(torch, dtype)
    q, k, v = _inputs(1, N, H, Hkv, d, dtype, layout, 50)
    cos, sin = so.rotation_table(N + 7, d)
    w = (1 + 0.3 * torch.randn(d, generator=_gen(51), device="cuda")).to(dtype)
    starts = torch.tensor([7], dtype=torch.int32, device="cuda")
    table = torch.randperm((N + 7 + page - 1) // page, generator=_gen(52), device="cuda").to(torch.int32)[None]
    positions = (7 + torch.arange(N, device="cuda", dtype=torch.int32)).expand(3, 1, N).contiguous()
    results = []
    for place in (dict(starts=starts), dict(positions=positions[:1]), dict(positions=positions, axes=_axes_of("turns", d // 2, 3)),
                  dict(positions=positions, axes=_axes_of("runs", d // 2, 3))):
        kw = dict(cos=cos, sin=sin, q_weight=w, k_weight=w, layout=layout, interleaved=interleaved)
        plain = qa.qk_norm_rope(q, k, **kw, **place)
        caches = [torch.zeros(table.shape[1], Hkv, page, d, device="cuda", dtype=dtype) for _ in range(2)]
        k_out = torch.empty(k.shape, device="cuda", dtype=dtype)
        q_out = qa.qk_norm_rope_append(q, k, v, *caches, table, k_out=k_out, **kw, **dict(place, starts=starts))
        results.append([*plain, q_out, k_out, *caches])
    first = results[0]
    assert torch.equal(_bits(first[0]), _bits(first[2])) and torch.equal(_bits(first[1]), _bits(first[3]))
    for got in results[1:]:
        for i, (a, b) in enumerate(zip(got, first)):
            assert torch.equal(_bits(a), _bits(b)), i
