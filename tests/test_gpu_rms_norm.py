"""rms_norm and rms_norm_fp8 against the definition in 64 bits: every way of holding a row,
strided and broadcast inputs, sums in place, scales of rows and groups, rows without a value,
streams and graphs.

Bounds.  s = x + r is one fp32 rounding of an exact sum.  The sum of squares adds at most 32
terms in a thread, over 64 lanes in 6 steps and over 16 wavefronts: below (32 + 6 + 16) 2^-24
of it, halved by the root; the mean's factor, root, quotient, and the products with them and
the weight are 2^-24 each.  Together below 2^-18 of y, then one rounding (so.check_rounded).  A
scale is off by as much again, and the codes are checked against y / the scale that was given.
"""
from __future__ import annotations

import math

import pytest

from tests import serving_oracle as so

pytestmark = pytest.mark.gpu

FP32 = 2.0 ** -18


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


def _normal(*shape, seed, dtype, mult=1.0):
    import torch
    return (torch.randn(*shape, generator=_gen(seed), device="cuda") * mult).to(dtype)


def _bits(t):
    import torch
    return t.contiguous().view({1: torch.uint8, 2: torch.int16, 4: torch.int32}[t.element_size()])


def _define(x, weight, residual, eps):
    """(y, s) in 64 bits."""
    s = x.double() if residual is None else x.double() + residual.double()
    y = s / (s.square().mean(-1, keepdim=True) + eps).sqrt()
    return (y if weight is None else y * weight.double()), s


def _check_sum(got, s):
    if got is not None:
        so.check_rounded(got, s, 2.0 ** -24 * s.abs(), "sum")


def _check_codes(codes, scales, y, group, what=""):
    """Codes of y and their scales (fp32 [..., 1] or [..., groups], or a number)."""
    import torch
    width = y.shape[-1]
    parts = y.reshape(*y.shape[:-1], -1, group or width)
    if torch.is_tensor(scales):
        want = (parts.abs().amax(-1) / 448).clamp(min=2.0 ** -126)
        got = scales.double()
        assert got.shape == want.shape
        assert ((got - want).abs() <= 2 * FP32 * want).all(), f"{what}: scales"
        parts = parts / got[..., None]
    else:
        parts = (parts / scales).clamp(-448, 448)
    codes = codes.view(torch.float8_e4m3fn).reshape(parts.shape)
    # E4M3 has no infinity: beyond 448 by the scale's rounding is 448
    so.check_rounded(codes, parts, 2 * FP32 * parts.abs(), what)


WIDTHS = [8, 24, 64, 72, 128, 200, 256, 264, 512, 776, 1024, 1032, 2048, 2056, 4096, 5120, 8192, 8200, 16384, 16392, 32768]


@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("width", WIDTHS)
def test_against_the_definition(qa, width, dtype):
    import torch
    dtype = getattr(torch, dtype)
    for rows, residual in ((1, True), (67, False), (5, True)):
        x = _normal(rows, width, seed=1, dtype=dtype, mult=2.0)
        r = _normal(rows, width, seed=2, dtype=dtype, mult=5.0) if residual else None
        w = _normal(width, seed=3, dtype=dtype) if rows > 1 else None
        y, s = _define(x, w, r, 1e-5)
        got, total = qa.rms_norm(x, w, residual=r, eps=1e-5)
        assert got.shape == x.shape and got.dtype == dtype and (total is None) == (not residual)
        so.check_rounded(got, y, FP32 * y.abs(), f"{rows} x {width}")
        _check_sum(total, s)


@pytest.mark.parametrize("group", [0, 32, 64, 128, 256, "fixed"])
@pytest.mark.parametrize("width", WIDTHS)
def test_codes_and_scales(qa, width, group):
    import torch
    fixed = group == "fixed"
    if not fixed and group and width % group:
        with pytest.raises(ValueError, match="group"):
            qa.rms_norm_fp8(_normal(3, width, seed=4, dtype=torch.bfloat16), group=group)
        return
    for rows, dtype, residual in ((1, torch.bfloat16, False), (37, torch.float16, True), (6, torch.bfloat16, True)):
        x = _normal(rows, width, seed=5, dtype=dtype)
        # rows and columns of different sizes, so that scales differ
        x *= torch.logspace(-2, 2, rows, device="cuda").to(dtype)[:, None]
        r = _normal(rows, width, seed=6, dtype=dtype) if residual else None
        w = (_normal(width, seed=7, dtype=dtype) * torch.logspace(-3, 1, width, device="cuda").to(dtype)) if rows > 1 else None
        y, s = _define(x, w, r, 1e-6)
        if fixed:
            codes, scales, total = qa.rms_norm_fp8(x, w, residual=r, scale=0.01)   # y beyond 4.48 is cut
            assert scales is None
            _check_codes(codes, float(torch.tensor(0.01)), y, 0, f"{rows} x {width}")
        else:
            codes, scales, total = qa.rms_norm_fp8(x, w, residual=r, group=group or None)
            assert scales.shape == (rows, width // group if group else 1) and scales.dtype == torch.float32
            _check_codes(codes, scales, y, group, f"{rows} x {width}")
        assert codes.dtype == torch.float8_e4m3fn and codes.shape == x.shape
        _check_sum(total, s)


def test_shapes_strides_and_broadcast_residuals(qa):
    """Parts of a wider projection, three dimensions, one row for all; nothing between the
    rows of a strided sum is touched."""
    import torch
    dtype = torch.bfloat16
    wide = _normal(3, 50, 3 * 256 + 8, seed=8, dtype=dtype)
    w = _normal(256, seed=9, dtype=dtype)
    for first in (0, 256, 520):
        x = wide[:, :, first:first + 256]
        r = _normal(1, 1, 256, seed=10, dtype=dtype).expand(3, 50, 256)
        y, s = _define(x, w, r, 1e-6)
        room = torch.full((3, 50, 300 + 4), 7.0, device="cuda", dtype=dtype)
        got, total = qa.rms_norm(x, w, residual=r, sum_out=room[:, :, 8:264])
        assert got.shape == x.shape and got.is_contiguous() and total.data_ptr() == room[:, :, 8:].data_ptr()
        so.check_rounded(got, y, FP32 * y.abs())
        _check_sum(total, s)
        assert (room[:, :, :8] == 7).all() and (room[:, :, 264:] == 7).all()
        codes, scales, total = qa.rms_norm_fp8(x, w, residual=r, group=64)
        assert scales.shape == (3, 50, 4)
        _check_codes(codes, scales, y, 64)
        _check_sum(total, s)
    # a single vector; a dimension of one with any stride
    v = _normal(64, seed=11, dtype=dtype)
    y, _ = _define(v, None, None, 1e-6)
    so.check_rounded(qa.rms_norm(v)[0], y, FP32 * y.abs())
    codes, scales, _ = qa.rms_norm_fp8(v)
    assert scales.shape == (1,)
    _check_codes(codes, scales, y, 0)
    t = _normal(1, 64, 5, seed=12, dtype=dtype).transpose(0, 2)[2:3].transpose(1, 2)   # [1, 1, 64], columns 5 apart
    with pytest.raises(ValueError, match="columns"):
        qa.rms_norm(t)
    with pytest.raises(ValueError, match="equal distances"):
        qa.rms_norm(wide[:, :40, :256])
    with pytest.raises(qa.QmAttnError) as e:
        qa.rms_norm(_normal(4, 68, seed=13, dtype=dtype)[:, :64])   # rows 68 elements apart
    assert e.value.status == qa.QM_ERR_STRIDE


def test_in_place(qa):
    """The sum in the residual's or in x's place gives the bytes of one of its own."""
    import torch
    for width, rows in ((64, 70), (4096, 9), (20000, 3)):
        x, r = (_normal(rows, width, seed=s, dtype=torch.float16) for s in (14, 15))
        w = _normal(width, seed=16, dtype=torch.float16)
        y, total = qa.rms_norm(x, w, residual=r)
        for place in (0, 1):
            a, b = x.clone(), r.clone()
            y2, t2 = qa.rms_norm(a, w, residual=b, sum_out=(a, b)[place])
            assert t2 is (a, b)[place] and torch.equal(_bits(t2), _bits(total)) and torch.equal(_bits(y2), _bits(y))
            assert torch.equal((b, a)[place], (r, x)[place])
        wide = torch.full((rows, width + 16), 3.0, device="cuda", dtype=torch.float16)
        wide[:, :width] = r
        y2, _ = qa.rms_norm(x, w, residual=wide[:, :width], sum_out=wide[:, :width])
        assert torch.equal(_bits(y2), _bits(y)) and torch.equal(wide[:, :width], total) and (wide[:, width:] == 3).all()


@pytest.mark.parametrize("width", [64, 200, 1024, 4096, 16384])
def test_rows_without_a_value(qa, width):
    """Zeros, subnormals, NaN, infinities and overflowing squares stay in their rows."""
    import torch
    x = _normal(9, width, seed=17, dtype=torch.bfloat16)
    clean = x.clone()
    x[1] = 0
    x[2] = 1e-30
    x[3, 5] = math.nan
    x[4, width - 1] = math.inf
    x[5] = 1e30            # squares beyond fp32
    x[6] = -3e18
    w = (1 + 0.1 * _normal(width, seed=18, dtype=torch.float32)).bfloat16()
    y, _ = qa.rms_norm(x, w)
    want, _ = _define(x, w, None, 1e-6)
    for i in (0, 1, 2, 6, 7, 8):
        so.check_rounded(y[i], want[i], FP32 * want[i].abs(), f"row {i}")
    assert (y[1] == 0).all() and torch.isnan(y[3]).all() and torch.isnan(y[4, -1]) and (y[4, :-1] == 0).all() and (y[5] == 0).all()
    good = [0, 7, 8]
    for kw in (dict(), dict(group=32), dict(scale=0.02)):
        if kw.get("group") and width % 32:
            continue
        codes, scales, _ = qa.rms_norm_fp8(x, w, **kw)
        ref, ref_scales, _ = qa.rms_norm_fp8(clean, w, **kw)
        assert torch.equal(_bits(codes[good]), _bits(ref[good]))
        c = codes.float()
        assert (c[1] == 0).all() and torch.isnan(c[3]).all() and torch.isnan(c[4, -1]) and (c[5] == 0).all()
        if scales is None:
            assert (c[4, :-1] == 0).all()
        else:
            flat = scales.view(9, -1)
            assert torch.equal(flat[good], ref_scales.view(9, -1)[good])
            assert (flat[1] == 2.0 ** -126).all() and torch.isnan(flat[3]).all() and torch.isnan(flat[4, -1]) and (flat[5] == 2.0 ** -126).all()
            if kw:   # groups without the infinity are zeros
                assert (flat[4, :-1] == 2.0 ** -126).all() and (c[4, :-32] == 0).all()
    # 0 / 0 without eps; signs of zeros are kept
    z = torch.zeros(1, width, device="cuda", dtype=torch.bfloat16)
    assert torch.isnan(qa.rms_norm(z, eps=0.0)[0]).all()
    assert torch.signbit(qa.rms_norm(-z)[0]).all()


def test_a_weight_that_is_no_number(qa):
    """NaN in the weight: that column, and with a scale a row the whole row."""
    import torch
    x, w = _normal(5, 512, seed=19, dtype=torch.bfloat16), torch.ones(512, device="cuda", dtype=torch.bfloat16)
    w[77] = math.nan
    y, _ = qa.rms_norm(x, w)
    assert torch.isnan(y[:, 77]).all() and int(torch.isnan(y).sum()) == 5
    codes, scales, _ = qa.rms_norm_fp8(x, w)
    assert torch.isnan(scales).all() and torch.isnan(codes.float()).all()
    codes, scales, _ = qa.rms_norm_fp8(x, w, group=64)
    assert int(torch.isnan(scales).sum()) == 5 and int(torch.isnan(codes.float()).sum()) == 5 * 64


def test_the_largest_of_a_scale_is_448(qa):
    import torch
    x = _normal(300, 1024, seed=20, dtype=torch.bfloat16, mult=3.0)
    for group in (None, 64):
        codes, scales, _ = qa.rms_norm_fp8(x, group=group)
        assert (codes.float().abs().view(300, -1, group or 1024).amax(-1) == 448).all()


def test_offsets_past_32_bits(qa):
    """More than 2^31 elements: the last rows as in a call of their own."""
    import torch
    rows, width = 70000, 32768
    x = torch.zeros(rows, width, device="cuda", dtype=torch.bfloat16)
    x[-3:] = _normal(3, width, seed=21, dtype=torch.bfloat16)
    y, total = qa.rms_norm(x, residual=x, sum_out=x)
    tail = _normal(3, width, seed=21, dtype=torch.bfloat16)
    ref, ref_sum = qa.rms_norm(tail, residual=tail)
    assert torch.equal(_bits(y[-3:]), _bits(ref)) and torch.equal(_bits(x[-3:]), _bits(ref_sum))
    assert not y[:-3].any() and not x[:-3].any()
    del y, total
    codes, scales, _ = qa.rms_norm_fp8(x, group=128)
    ref, ref_scales, _ = qa.rms_norm_fp8(ref_sum, group=128)
    assert torch.equal(_bits(codes[-3:]), _bits(ref)) and torch.equal(scales[-3:], ref_scales)
    assert not codes[:-3].view(torch.uint8).any()


def test_streams_and_graphs(qa):
    """On another stream, and captured: every replay as the eager call, with new inputs."""
    import torch
    x, r = (_normal(40, 2048, seed=s, dtype=torch.bfloat16) for s in (22, 23))
    w = _normal(2048, seed=24, dtype=torch.bfloat16)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    side = qa.rms_norm_fp8(x, w, residual=r, stream=s)
    s.synchronize()
    here = qa.rms_norm_fp8(x, w, residual=r)
    for a, b in zip(side, here):
        assert torch.equal(_bits(a), _bits(b))
    with torch.cuda.stream(s):
        qa.rms_norm(x, w, residual=r)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, total = qa.rms_norm(x, w, residual=r)
        codes, scales, _ = qa.rms_norm_fp8(total, w, group=128)
    for i in range(4):
        x.copy_(_normal(40, 2048, seed=30 + i, dtype=torch.bfloat16))
        graph.replay()
        torch.cuda.synchronize()
        y2, t2 = qa.rms_norm(x, w, residual=r)
        c2, s2, _ = qa.rms_norm_fp8(t2, w, group=128)
        for a, b in ((y, y2), (total, t2), (codes, c2), (scales, s2)):
            assert torch.equal(_bits(a), _bits(b))


def test_refusals(qa):
    import torch
    x, w = _normal(4, 64, seed=25, dtype=torch.bfloat16), torch.ones(64, device="cuda", dtype=torch.bfloat16)
    for error, call in [
            (ValueError, lambda: qa.rms_norm(x.cpu())), (TypeError, lambda: qa.rms_norm(x.float())),
            (ValueError, lambda: qa.rms_norm(x, w[:32])), (ValueError, lambda: qa.rms_norm(x, w.half())),
            (ValueError, lambda: qa.rms_norm(x, w.cpu())), (ValueError, lambda: qa.rms_norm(x, w, residual=x[:3])),
            (TypeError, lambda: qa.rms_norm(x, w, residual=x.half())), (ValueError, lambda: qa.rms_norm(x, w, residual=x.cpu())),
            (ValueError, lambda: qa.rms_norm(x, w, sum_out=x)), (ValueError, lambda: qa.rms_norm(x, w, out=x[:2])),
            (ValueError, lambda: qa.rms_norm(x, w, out=x.t())), (ValueError, lambda: qa.rms_norm(x[0, 0])), (ValueError, lambda: qa.rms_norm(x[:0])),
            (ValueError, lambda: qa.rms_norm_fp8(x, w, scale=1.0, group=32)), (ValueError, lambda: qa.rms_norm_fp8(x, w, group=16)),
            (ValueError, lambda: qa.rms_norm_fp8(x, w, group=128)), (ValueError, lambda: qa.rms_norm_fp8(x, w, out=x)),
            (ValueError, lambda: qa.rms_norm_fp8(x, w, scales=torch.ones(4, device="cuda"))),
            (ValueError, lambda: qa.rms_norm_fp8(x, w, scale=2.0, scales=torch.ones(4, device="cuda")))]:
        with pytest.raises(error):
            call()

    def status(code, call):
        with pytest.raises(qa.QmAttnError) as e:
            call()
        assert e.value.status == code
    status(qa.QM_ERR_NORM, lambda: qa.rms_norm(_normal(2, 12, seed=26, dtype=torch.bfloat16)))
    status(qa.QM_ERR_NORM, lambda: qa.rms_norm(_normal(1, 32776, seed=26, dtype=torch.bfloat16)))
    status(qa.QM_ERR_NORM, lambda: qa.rms_norm(x, eps=-1.0))
    status(qa.QM_ERR_SCALE, lambda: qa.rms_norm_fp8(x, scale=0.0))
    status(qa.QM_ERR_SCALE, lambda: qa.rms_norm_fp8(x, scale=-1.0))
    status(qa.QM_ERR_SCALE, lambda: qa.rms_norm_fp8(x, scale=math.nan))
    status(qa.QM_ERR_ALIAS, lambda: qa.rms_norm(x, out=x))
    big = _normal(5, 64, seed=27, dtype=torch.bfloat16)
    status(qa.QM_ERR_ALIAS, lambda: qa.rms_norm(big[:4], residual=x, sum_out=big[1:]))


def test_a_scale_that_is_infinite(qa):
    """A y past fp32 (from an absurd weight): an infinite scale, whose codes are NaN; other
    groups and rows are not affected."""
    import torch
    x = _normal(4, 512, seed=40, dtype=torch.bfloat16)
    w = torch.ones(512, device="cuda", dtype=torch.bfloat16)
    w[200] = 3e38
    x[:, 200] = 1.0
    x[1, 200] = 300.0   # y = 3e38 * 300 / (root of the mean) overflows here
    codes, scales, _ = qa.rms_norm_fp8(x, w, group=64)
    assert torch.isinf(scales[1, 3]) and torch.isnan(codes.float()[1, 192:256]).all()
    rest = torch.ones(4, 8, dtype=torch.bool, device="cuda")
    rest[1, 3] = False
    assert torch.isfinite(scales[rest]).all()
    assert torch.isfinite(codes.float().view(4, 8, 64)[rest]).all()


@pytest.mark.parametrize("width", [64, 128, 256, 512, 1024, 4096, 16384, 32768])
def test_products_beyond_fp32_where_the_result_is_not(qa, width):
    """|s w| past fp32's range, or below it, in rows whose y is neither: a scale a row is that
    of the y that are formed, as a scale a group is, and the rows beside them keep their bytes."""
    import torch
    def inputs(s, w):
        x = _normal(9, width, seed=41, dtype=torch.bfloat16)
        x[2] *= s
        x[7] *= s
        return x, (_normal(width, seed=42, dtype=torch.float32) * w).bfloat16()

    # a mean square past fp32: y is 0, whatever the weight
    x, w = inputs(1.0, 1.0)
    x[2], x[7] = 3e38, -3e38
    w[:] = 1.5
    ref, ref_scales, _ = qa.rms_norm_fp8(x[:2], w)
    for kw in (dict(), dict(group=32), dict(scale=0.02)):
        codes, scales, _ = qa.rms_norm_fp8(x, w, **kw)
        assert (codes.float()[[2, 7]] == 0).all(), kw
        if scales is not None:
            assert (scales[[2, 7]] == 2.0 ** -126).all(), kw
        if not kw:
            assert torch.equal(_bits(codes[:2]), _bits(ref)) and torch.equal(scales[:2], ref_scales)
    # s w overflows (below: is lost), y does not
    for s, w, eps in ((1e12, 1e30, 1e-6), (1e-15, 1e-30, 0.0)):
        x, w = inputs(s, w)
        y, _ = _define(x, w, None, eps)
        assert torch.isfinite(y.float()).all() and (y.abs().amax(-1) > 1e-35).all()
        for group in (None, 32):
            codes, scales, _ = qa.rms_norm_fp8(x, w, eps=eps, group=group)
            _check_codes(codes, scales, y, group or 0, f"{s} {group}")
        quiet = x.clone()
        quiet[2], quiet[7] = 1.0, 1.0
        codes, scales, _ = qa.rms_norm_fp8(x, w, eps=eps)
        ref, ref_scales, _ = qa.rms_norm_fp8(quiet, w, eps=eps)
        rest = [0, 1, 3, 4, 5, 6, 8]
        assert torch.equal(_bits(codes[rest]), _bits(ref[rest])) and torch.equal(scales[rest], ref_scales[rest])


@pytest.mark.parametrize("width,rows,launch", [(1056, (1 << 24) + 70, 1 << 23), (8, (1 << 29) + 3, 1 << 28)])
def test_more_rows_than_one_launch_takes(qa, width, rows, launch):
    """Rows of 2^32 threads and more: those on either side of each launch's end, and some from
    everywhere, as in a call of their own, and every row written."""
    import torch
    # rows that begin 8 elements apart
    x = torch.empty(rows * 8 + width, device="cuda", dtype=torch.bfloat16).normal_(generator=_gen(43)).as_strided((rows, width), (8, 1))
    w = _normal(width, seed=44, dtype=torch.bfloat16)
    at = torch.cat([torch.arange(max(0, e - 40), min(rows, e + 40)) for e in [0, *range(launch, rows, launch), rows]]
                   + [torch.randint(0, rows, (2000,), generator=torch.Generator().manual_seed(45))]).cuda()
    some = x[at].contiguous()
    if width == 8:
        y, _ = qa.rms_norm(x, w, out=torch.full((rows, width), 99.0, device="cuda", dtype=torch.bfloat16))
        assert torch.equal(_bits(y[at]), _bits(qa.rms_norm(some, w)[0]))
        for lo in range(0, rows, 1 << 27):   # (no y of 8 columns reaches 99)
            assert not (y[lo:lo + (1 << 27)] == 99).any()
        return
    r = _normal(1, width, seed=46, dtype=torch.bfloat16)
    scales = torch.full((rows, 1), -1.0, device="cuda")
    codes, _, total = qa.rms_norm_fp8(x, w, residual=r.expand(rows, width), scales=scales)
    ref = qa.rms_norm_fp8(some, w, residual=r.expand(at.numel(), width))
    for a, b in zip((codes.view(torch.uint8), scales, total), ref):
        assert torch.equal(_bits(a[at]), _bits(b))
    assert (scales > 0).all()
    groups = torch.full((rows, 33), -1.0, device="cuda")
    qa.rms_norm_fp8(x, group=32, out=codes, scales=groups)
    ref = qa.rms_norm_fp8(some, group=32)
    assert torch.equal(_bits(codes.view(torch.uint8)[at]), _bits(ref[0])) and torch.equal(groups[at], ref[1])
    assert (groups > 0).all()
