"""fwd_window against the definition in 64 bits, on every row: windows and first keys on
both sides of the 64-key blocks, one token to long sequences, types, widths, layouts and
head groups; exactly the causal kernel where the window hides nothing."""
from __future__ import annotations

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


def _inputs(B, H, Hkv, N, d, dv, dtype, seed, mult=1.0):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [(torch.randn(B, h, N, w, generator=g, device="cuda") * m).to(dtype)
            for h, w, m in ((H, d, mult), (Hkv, d, mult), (Hkv, dv, 1.0))]


def _check(q, k, v, window, sinks, scale, o, lse, what, heads=None):
    B, H, N, _ = q.shape
    seen = so.window_mask(N, window, sinks)
    for b in range(B):
        for h in range(H) if heads is None else heads:
            g = h // (H // k.shape[1])
            want = so.attention_row_bounds(q[b, h], k[b, g], v[b, g], scale, seen, q.dtype)
            so.check_attention(o[b, h], lse[b, h], want, f"{what} b={b} h={h}")


@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("N,window,sinks", [
    (1, 1, 0), (2, 1, 0), (2, 1, 1), (64, 1, 0), (65, 1, 1), (130, 63, 0), (130, 64, 1), (200, 65, 4),
    (300, 1, 0), (300, 2, 64), (300, 17, 65), (513, 128, 63), (513, 129, 128), (777, 500, 4),
    (777, 100, 300), (1000, 256, 4), (1000, 999, 0), (1000, 64, 129),
])
def test_against_the_definition(qa, N, window, sinks, d, dv, dtype):
    import torch
    dtype = getattr(torch, dtype)
    H, Hkv = (2, 2) if d == 192 else (3, 1)
    q, k, v = _inputs(1, H, Hkv, N, d, dv, dtype, N + window)
    o, lse = qa.fwd_window(q, k, v, window, sinks)
    _check(q, k, v, window, sinks, 1 / d ** 0.5, o, lse, f"N={N} window={window} sinks={sinks}")


@pytest.mark.parametrize("B,H,Hkv,N,d,window,sinks,scale,mult", [
    (2, 4, 2, 2049, 128, 300, 70, None, 2.0),     # sharper rows
    (1, 8, 1, 1500, 64, 700, 4, -0.2, 1.0),
    (2, 2, 2, 640, 128, 33, 0, 0.0, 1.0),         # every visible score 0
    (1, 2, 1, 5000, 64, 2500, 1, None, 2.0),
])
def test_batches_groups_and_scales(qa, B, H, Hkv, N, d, window, sinks, scale, mult):
    import torch
    q, k, v = _inputs(B, H, Hkv, N, d, d, torch.bfloat16, 5, mult)
    o, lse = qa.fwd_window(q, k, v, window, sinks, scale=scale)
    scale = 1 / d ** 0.5 if scale is None else float(torch.tensor(scale))
    _check(q, k, v, window, sinks, scale, o, lse, f"{B, H, Hkv, N, d, window, sinks}")


def _bits(t):
    import torch
    return t.contiguous().view(torch.int16 if t.element_size() == 2 else torch.int32)


@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128)])
@pytest.mark.parametrize("H,N,window,sinks", [(6, 700, 200, 3), (40, 300, 65, 0), (2, 3001, 513, 64)])
def test_layouts_and_tile_sizes_give_the_same_bytes(qa, d, dv, H, N, window, sinks):
    import torch
    q, k, v = _inputs(2, H, H // 2, N, d, dv, torch.bfloat16, 6)
    o, lse = qa.fwd_window(q, k, v, window, sinks)
    t = [x.transpose(1, 2).contiguous() for x in (q, k, v)]
    try:
        for rows in (0, 128, 256):
            qa.set_tile_rows(rows)
            o1, lse1 = qa.fwd_window(q, k, v, window, sinks)
            o2, lse2 = qa.fwd_window(*t, window, sinks, layout="bnhd")
            assert torch.equal(_bits(o1), _bits(o)) and torch.equal(_bits(lse1), _bits(lse)), rows
            assert torch.equal(_bits(o2.transpose(1, 2)), _bits(o)) and torch.equal(_bits(lse2), _bits(lse)), rows
    finally:
        qa.set_tile_rows(0)


@pytest.mark.parametrize("d,dv", [(64, 64), (128, 128), (192, 128)])
@pytest.mark.parametrize("window,sinks", [(500, 0), (2 ** 31 - 1, 0), (400, 100), (1, 499), (1, 2 ** 31 - 1), (450, 60)])
def test_a_window_that_hides_nothing_is_the_causal_kernel(qa, window, sinks, d, dv):
    import torch
    q, k, v = _inputs(1, 2, 2, 500, d, dv, torch.float16, 7)
    o, lse = qa.fwd_window(q, k, v, window, sinks)
    ro, rl = qa.fwd(q, k, v, causal=True)
    assert torch.equal(_bits(o), _bits(ro)) and torch.equal(_bits(lse), _bits(rl))


def test_keys_outside_every_window_do_not_matter(qa):
    """The last row's result does not change with keys and values that it does not see,
    infinities and NaN among them (in blocks that its own block of rows skips)."""
    import torch
    N, window, sinks = 2000, 100, 4
    q, k, v = _inputs(1, 2, 1, N, 128, 128, torch.bfloat16, 8)
    o, lse = qa.fwd_window(q, k, v, window, sinks)
    k2, v2 = k.clone(), v.clone()
    k2[:, :, 64:1500], v2[:, :, 64:1500] = float("nan"), float("inf")
    o2, lse2 = qa.fwd_window(q, k2, v2, window, sinks)
    assert torch.equal(_bits(o2[:, :, 1800:]), _bits(o[:, :, 1800:]))
    assert torch.equal(_bits(lse2[:, :, 1800:]), _bits(lse[:, :, 1800:]))
    assert torch.equal(_bits(o2[:, :, :64]), _bits(o[:, :, :64]))


def test_checking_build_gives_the_same_bytes(qa):
    """A barrier after every key block changes nothing: the rings' protocol holds where
    blocks are left out (see test_gpu_debug_sync.py)."""
    import torch
    debug = qa.open_library(qa.DEBUG_LIB_PATH)
    for d, dv, H, N, window, sinks in ((64, 64, 8, 3000, 700, 65), (128, 128, 8, 3000, 700, 65),
                                       (192, 128, 4, 1500, 300, 4), (128, 128, 64, 1500, 200, 0),
                                       (64, 64, 2, 1000, 256, 4), (128, 128, 2, 4000, 2000, 4)):
        q, k, v = _inputs(1, H, H, N, d, dv, torch.bfloat16, 9)
        o, lse = qa.fwd_window(q, k, v, window, sinks)
        o2, lse2 = torch.full_like(o, float("nan")), torch.full_like(lse, float("nan"))
        for rows in (128, 256):
            assert debug.qm_attn_set_tile_rows(rows) == 0
            st = debug.qm_attn_fwd_window(q.data_ptr(), k.data_ptr(), v.data_ptr(), o2.data_ptr(),
                                          lse2.data_ptr(), 1, H, H, N, d, dv, 1 / d ** 0.5, window, sinks,
                                          torch.cuda.current_stream().cuda_stream, qa.QM_BF16, qa.QM_BHND)
            assert st == 0
            torch.cuda.synchronize()
            assert torch.equal(_bits(o2), _bits(o)) and torch.equal(_bits(lse2), _bits(lse)), (d, rows)


def test_refusals(qa):
    import torch
    q, k, v = _inputs(1, 4, 2, 40, 64, 64, torch.bfloat16, 10)
    for window, sinks in ((0, 0), (-1, 0), (4, -1)):
        with pytest.raises(qa.QmAttnError) as e:
            qa.fwd_window(q, k, v, window, sinks)
        assert e.value.status == qa.QM_ERR_WINDOW
    for window, sinks in ((2 ** 31, 0), (2 ** 32 + 1, 0), (4, 2 ** 40)):
        with pytest.raises(ValueError):
            qa.fwd_window(q, k, v, window, sinks)
    with pytest.raises(TypeError):
        qa.fwd_window(q, k, v, 3.5)
    with pytest.raises(ValueError):
        qa.fwd_window(q, k.transpose(2, 3), v, 4)
    with pytest.raises(TypeError):
        qa.fwd_window(q.float(), k.float(), v.float(), 4)
    with pytest.raises(qa.QmAttnError) as e:
        qa.fwd_window(q, k[:, :1].expand(1, 3, 40, 64).contiguous(), v[:, :1].expand(1, 3, 40, 64).contiguous(), 4)
    assert e.value.status == qa.QM_ERR_SHAPE
