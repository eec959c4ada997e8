"""The norm's and the several axes' C entry points without a GPU: every invalid argument
gets its documented status before anything is enqueued.  Every call here carries at least one
invalid argument, and its addresses are never dereferenced."""
from __future__ import annotations

import ctypes
import os

import pytest

import paper_2506_12355_amd as qa
from paper_2506_12355_amd import build as qbuild
from tests import test_serving_boundary as tsb

GIB = 1 << 30
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(qa.LIB_PATH):
        qbuild.build()
    return qa.load_library()


NORM = dict(x=1 * GIB, residual=2 * GIB, weight=3 * GIB, out=4 * GIB, sum=5 * GIB, rows=100, width=512, x_stride=512,
            residual_stride=512, sum_stride=512, eps=1e-6, stream=None, dtype=1)
NORM_REFUSALS = [
    (dict(x=None), qa.QM_ERR_NULL), (dict(out=None), qa.QM_ERR_NULL), (dict(residual=None), qa.QM_ERR_NULL),
    (dict(rows=0), qa.QM_ERR_SHAPE), (dict(rows=-5), qa.QM_ERR_SHAPE),
    (dict(rows=(1 << 31) - 1, x_stride=1 << 58), qa.QM_ERR_SHAPE),
    (dict(dtype=2), qa.QM_ERR_DTYPE), (dict(width=0), qa.QM_ERR_NORM), (dict(width=12), qa.QM_ERR_NORM),
    (dict(width=32776), qa.QM_ERR_NORM), (dict(width=-8), qa.QM_ERR_NORM), (dict(eps=-1e-6), qa.QM_ERR_NORM),
    (dict(eps=NAN), qa.QM_ERR_NORM), (dict(eps=INF), qa.QM_ERR_NORM),
    (dict(x_stride=-512), qa.QM_ERR_STRIDE), (dict(x_stride=516), qa.QM_ERR_STRIDE), (dict(residual_stride=4), qa.QM_ERR_STRIDE),
    (dict(sum_stride=504), qa.QM_ERR_STRIDE), (dict(sum_stride=0), qa.QM_ERR_STRIDE),
    (dict(out=1 * GIB), qa.QM_ERR_ALIAS), (dict(out=2 * GIB + 1024), qa.QM_ERR_ALIAS), (dict(out=3 * GIB), qa.QM_ERR_ALIAS),
    (dict(out=5 * GIB + 99 * 1024), qa.QM_ERR_ALIAS), (dict(sum=3 * GIB), qa.QM_ERR_ALIAS),
    # beside x's and the residual's own place the sum may not touch them
    (dict(sum=1 * GIB + 1024), qa.QM_ERR_ALIAS), (dict(sum=2 * GIB, sum_stride=520), qa.QM_ERR_ALIAS),
    (dict(sum=1 * GIB, residual=1 * GIB + 1024), qa.QM_ERR_ALIAS),
    # a strided x reaches further
    (dict(out=1 * GIB + 99 * 4096, x_stride=2048), qa.QM_ERR_ALIAS),
    (dict(x=1 * GIB + 8), qa.QM_ERR_UNSUPPORTED), (dict(residual=2 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
    (dict(weight=3 * GIB + 4), qa.QM_ERR_UNSUPPORTED), (dict(out=4 * GIB + 8), qa.QM_ERR_UNSUPPORTED),
    (dict(sum=5 * GIB + 8), qa.QM_ERR_UNSUPPORTED),
    # valid but for the alignment: in place, strides of a single row, a broadcast residual
    (dict(sum=2 * GIB, out=4 * GIB + 2), qa.QM_ERR_UNSUPPORTED), (dict(sum=1 * GIB, out=4 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
    (dict(rows=1, x_stride=3, residual_stride=-1, sum_stride=0, out=4 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
    (dict(residual_stride=0, out=4 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
    (dict(weight=None, residual=None, sum=None, residual_stride=-3, sum_stride=-3, out=4 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
]


def _call(entry, defaults, over):
    assert set(over) <= set(defaults)
    return entry(*[(ctypes.c_longlong * 3)(*v) if isinstance(v, tuple) else v for v in dict(defaults, **over).values()])


@pytest.mark.parametrize("over,status", NORM_REFUSALS, ids=str)
def test_rms_norm_refusals(lib, over, status):
    assert _call(lib.qm_rms_norm, NORM, over) == status


NORM_FP8 = dict(x=1 * GIB, residual=2 * GIB, weight=3 * GIB, out=4 * GIB, scales=6 * GIB, sum=5 * GIB, rows=100, width=512,
                x_stride=512, residual_stride=512, sum_stride=512, eps=1e-6, scale=1.0, group=128, stream=None, dtype=1)


@pytest.mark.parametrize("over,status", [c for c in NORM_REFUSALS if "width" not in c[0]] + [
    (dict(width=12, group=0), qa.QM_ERR_NORM), (dict(group=16), qa.QM_ERR_NORM), (dict(group=-32), qa.QM_ERR_NORM),
    (dict(group=256, width=384, sum_stride=512), qa.QM_ERR_NORM), (dict(scales=None), qa.QM_ERR_NORM),
    (dict(scales=None, group=0, scale=0.0), qa.QM_ERR_SCALE), (dict(scales=None, group=0, scale=-2.0), qa.QM_ERR_SCALE),
    (dict(scales=None, group=0, scale=NAN), qa.QM_ERR_SCALE), (dict(scales=None, group=0, scale=INF), qa.QM_ERR_SCALE),
    (dict(scales=None, group=0, scale=1e-40), qa.QM_ERR_SCALE),
    (dict(scales=1 * GIB + 4), qa.QM_ERR_ALIAS), (dict(scales=4 * GIB + 512 * 100 - 4), qa.QM_ERR_ALIAS),
    (dict(scales=5 * GIB), qa.QM_ERR_ALIAS), (dict(scales=6 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
    # codes are half as long as the inputs; a scale a row, which is not looked at beside scales
    (dict(out=5 * GIB - 512 * 100, scales=6 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
    (dict(group=0, scale=NAN, scales=6 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
], ids=str)
def test_rms_norm_fp8_refusals(lib, over, status):
    assert _call(lib.qm_rms_norm_fp8, NORM_FP8, over) == status


def _with_axes(defaults, starts):
    """The arguments of a call of one axis, positions and axes in the place of starts, or
    before it."""
    args = {}
    for name, value in defaults.items():
        if name == "starts":
            args.update(positions=13 * GIB, pair_axis=bytes([0, 1, 2, 2] * 16), axes=3)
            if not starts:
                continue
        args[name] = value
    return args


ROPE, APPEND = _with_axes(tsb.ROPE, False), _with_axes(tsb.APPEND, True)
AXES = [
    (dict(positions=None), qa.QM_ERR_NULL), (dict(pair_axis=None), qa.QM_ERR_NULL), (dict(axes=0), qa.QM_ERR_AXES),
    (dict(axes=5), qa.QM_ERR_AXES), (dict(axes=2), qa.QM_ERR_AXES), (dict(pair_axis=bytes([0] * 63 + [3])), qa.QM_ERR_AXES),
    (dict(rotary=0), qa.QM_ERR_ROTARY), (dict(table_rows=0), qa.QM_ERR_ROTARY), (dict(positions=13 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
    # 3 x 2 x 100 positions
    (dict(q_out=13 * GIB + 2384), qa.QM_ERR_ALIAS), (dict(k_out=13 * GIB), qa.QM_ERR_ALIAS),
    # fewer rows of the table than tokens are no error: positions are anywhere
    (dict(table_rows=5, q_out=3 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
]


def _refusals(cases):
    return [c for c in cases if "starts" not in c[0] and c[0] != dict(q_out=8 * GIB)]


@pytest.mark.parametrize("over,status", AXES + _refusals(tsb.ROPE_REFUSALS), ids=str)
def test_norm_rope_axes_refusals(lib, over, status):
    assert _call(lib.qm_qk_norm_rope_axes, ROPE, over) == status


@pytest.mark.parametrize("over,status", AXES + _refusals(tsb.ROPE_REFUSALS) + [
    (dict(v=None), qa.QM_ERR_NULL), (dict(page_table=None), qa.QM_ERR_NULL), (dict(page_size=24), qa.QM_ERR_PAGE),
    (dict(k_cache=13 * GIB - 16), qa.QM_ERR_ALIAS), (dict(k_scale=0.0), qa.QM_ERR_SCALE), (dict(starts=8 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
], ids=str)
def test_append_axes_refusals(lib, over, status):
    assert _call(lib.qm_qk_norm_rope_append_axes, APPEND, over) == status


def _shared(defaults):
    args = {}
    for name, value in defaults.items():
        if name in ("window", "sinks"):
            continue
        if name == "B":
            args["prefix_table"] = 13 * GIB
        if name == "max_length":
            args.update(prefix_cols=5, prefix_length=70)
        args[name] = value
    return args


SHARED = _shared(tsb.DECODE)


@pytest.mark.parametrize("over,status", [
    (dict(q=None), qa.QM_ERR_NULL), (dict(k_cache=None), qa.QM_ERR_NULL), (dict(v_cache=None), qa.QM_ERR_NULL),
    (dict(o=None), qa.QM_ERR_NULL), (dict(lse=None), qa.QM_ERR_NULL), (dict(page_table=None), qa.QM_ERR_NULL),
    (dict(lengths=None), qa.QM_ERR_NULL), (dict(prefix_table=None), qa.QM_ERR_NULL), (dict(dtype=2), qa.QM_ERR_DTYPE),
    (dict(B=0), qa.QM_ERR_SHAPE), (dict(H=7), qa.QM_ERR_SHAPE), (dict(d=192), qa.QM_ERR_HEADDIM), (dict(page_size=20), qa.QM_ERR_PAGE),
    (dict(prefix_length=-1), qa.QM_ERR_PAGE), (dict(prefix_length=81), qa.QM_ERR_PAGE), (dict(prefix_cols=0), qa.QM_ERR_PAGE),
    (dict(prefix_cols=1 << 30), qa.QM_ERR_PAGE), (dict(prefix_cols=-3), qa.QM_ERR_PAGE),
    (dict(cache_layout=2), qa.QM_ERR_LAYOUT), (dict(scale=INF), qa.QM_ERR_SCALE), (dict(scale=3e38, k_scale=2.0), qa.QM_ERR_SCALE),
    (dict(o=1 * GIB), qa.QM_ERR_ALIAS), (dict(o=13 * GIB - 16), qa.QM_ERR_ALIAS), (dict(lse=13 * GIB), qa.QM_ERR_ALIAS),
    (dict(lengths=7 * GIB + 1), qa.QM_ERR_UNSUPPORTED), (dict(prefix_table=13 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
    # without a prefix its table is not looked at, whatever its address and columns
    (dict(prefix_length=0, prefix_table=4 * GIB + 1, prefix_cols=-1, lengths=7 * GIB + 1), qa.QM_ERR_UNSUPPORTED),
    (dict(prefix_length=0, prefix_table=None, prefix_cols=0, lengths=7 * GIB + 1), qa.QM_ERR_UNSUPPORTED),
], ids=str)
def test_decode_shared_refusals(lib, over, status):
    assert _call(lib.qm_attn_decode_shared, SHARED, over) == status


def test_shared_workspace_refusals(lib):
    need = ctypes.c_size_t(77)
    good = dict(B=2, H=8, Hkv=2, d=128, page_size=16, table_cols=10, prefix_length=70, max_length=100)
    for over, status in [(dict(B=0), qa.QM_ERR_SHAPE), (dict(Hkv=3), qa.QM_ERR_SHAPE), (dict(d=32), qa.QM_ERR_HEADDIM),
                         (dict(page_size=15), qa.QM_ERR_PAGE), (dict(table_cols=0), qa.QM_ERR_PAGE), (dict(max_length=0), qa.QM_ERR_PAGE)]:
        for prefix in (70, 0):
            args = dict(good, prefix_length=prefix, **over)
            assert lib.qm_attn_decode_shared_workspace(*args.values(), ctypes.byref(need)) == status
    assert lib.qm_attn_decode_shared_workspace(*good.values(), None) == qa.QM_ERR_NULL
    assert need.value == 77


def test_status_texts(lib):
    codes = [qa.QM_ERR_NORM, qa.QM_ERR_AXES, qa.QM_ERR_WORKSPACE]
    texts = {qa.strerror(c) for c in codes}
    assert len(texts) == len(codes) and "unknown status" not in texts


def test_host_tensors_are_refused():
    torch = pytest.importorskip("torch")
    x = torch.zeros(3, 64, dtype=torch.bfloat16)
    for call in (lambda: qa.rms_norm(x), lambda: qa.rms_norm_fp8(x)):
        with pytest.raises(ValueError, match="ROCm device"):
            call()


def test_axes_are_read_in_each_call():
    """Whole numbers of any kind, as they stand when a call is made."""
    import numpy as np
    import torch
    from paper_2506_12355_amd.serving import _pair_axes
    held = torch.tensor([0, 1, 2, 2])
    own = tuple(held)
    assert _pair_axes(own, 4, 3) == bytes([0, 1, 2, 2])
    held[0] = 2
    assert _pair_axes(own, 4, 3) == bytes([2, 1, 2, 2])
    assert _pair_axes(np.array([1, 0], dtype=np.int64), 2, 2) == bytes([1, 0])
    assert _pair_axes((1, 0), 2, 2) == bytes([1, 0])
    with pytest.raises(TypeError):
        _pair_axes((1.0, 0.0), 2, 2)
    for axes in ((0, 2), (0, -1), (0, 256), (0, 1, 1), ()):
        with pytest.raises(ValueError, match="axes must"):
            _pair_axes(axes, 2, 2)
