"""The serving entry points of the C ABI without a GPU: every invalid argument gets its
documented status before anything is enqueued.  Every call here carries at least one
invalid argument, and its addresses are never dereferenced."""
from __future__ import annotations

import ctypes
import os

import pytest

import paper_2506_12355_amd as qa
from paper_2506_12355_amd import build as qbuild

GIB = 1 << 30
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(qa.LIB_PATH):
        qbuild.build()
    return qa.load_library()


def _strides(*s):
    return s


def _args(defaults, over):
    assert set(over) <= set(defaults)
    return [(ctypes.c_longlong * 3)(*x) if isinstance(x, tuple) else x for x in dict(defaults, **over).values()]


ROPE = dict(q=1 * GIB, k=2 * GIB, q_out=3 * GIB, k_out=4 * GIB, q_weight=5 * GIB, k_weight=5 * GIB + 4096,
            cos=6 * GIB, sin=7 * GIB, starts=8 * GIB, counts=8 * GIB + 4096, B=2, H=8, Hkv=2, N=100, d=128,
            rotary=128, table_rows=200, eps=1e-6, interleaved=0, q_strides=None, k_strides=None, stream=None,
            dtype=1, layout=0)


def rope(lib, **over):
    return lib.qm_qk_norm_rope(*_args(ROPE, over))


ROPE_REFUSALS = [
    (dict(q=None), qa.QM_ERR_NULL), (dict(k=None), qa.QM_ERR_NULL), (dict(q_out=None), qa.QM_ERR_NULL),
    (dict(cos=None), qa.QM_ERR_NULL), (dict(sin=None), qa.QM_ERR_NULL),
    (dict(B=0), qa.QM_ERR_SHAPE), (dict(H=0), qa.QM_ERR_SHAPE), (dict(Hkv=-1), qa.QM_ERR_SHAPE), (dict(N=0), qa.QM_ERR_SHAPE),
    (dict(B=1 << 14, N=1 << 14), qa.QM_ERR_SHAPE), (dict(B=(1 << 31) - 1, N=(1 << 31) - 1, H=(1 << 31) - 1), qa.QM_ERR_SHAPE),
    (dict(d=96), qa.QM_ERR_HEADDIM), (dict(d=192), qa.QM_ERR_HEADDIM), (dict(d=0), qa.QM_ERR_HEADDIM),
    (dict(dtype=2), qa.QM_ERR_DTYPE), (dict(dtype=-1), qa.QM_ERR_DTYPE), (dict(layout=2), qa.QM_ERR_LAYOUT),
    (dict(rotary=-16), qa.QM_ERR_ROTARY), (dict(rotary=144), qa.QM_ERR_ROTARY), (dict(rotary=24), qa.QM_ERR_ROTARY),
    (dict(rotary=80, d=64), qa.QM_ERR_ROTARY), (dict(table_rows=0), qa.QM_ERR_ROTARY),
    (dict(starts=None, table_rows=99), qa.QM_ERR_ROTARY), (dict(interleaved=2), qa.QM_ERR_ROTARY),
    (dict(eps=-1e-6), qa.QM_ERR_ROTARY), (dict(eps=NAN), qa.QM_ERR_ROTARY), (dict(eps=INF), qa.QM_ERR_ROTARY),
    (dict(q_strides=_strides(0, 12, 0)), qa.QM_ERR_STRIDE), (dict(k_strides=_strides(-8, 0, 0)), qa.QM_ERR_STRIDE),
    (dict(q_strides=_strides(1 << 61, 1 << 61, 0)), qa.QM_ERR_SHAPE),
    (dict(q_out=1 * GIB + 4096), qa.QM_ERR_ALIAS), (dict(k_out=2 * GIB), qa.QM_ERR_ALIAS), (dict(k_out=3 * GIB + 16), qa.QM_ERR_ALIAS),
    (dict(q_out=5 * GIB), qa.QM_ERR_ALIAS), (dict(k_out=6 * GIB + 1024), qa.QM_ERR_ALIAS), (dict(q_out=8 * GIB), qa.QM_ERR_ALIAS),
    # 2 x 100 x 8 x 128 bf16 values: q spans 400 KiB; with a batch stride of 1 MiB of elements, 2 MiB more
    (dict(q_out=1 * GIB + (2 << 20), q_strides=_strides(1 << 20, 1024, 128)), qa.QM_ERR_ALIAS),
    (dict(q=1 * GIB + 8), qa.QM_ERR_UNSUPPORTED), (dict(q_out=3 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
    (dict(q_weight=5 * GIB + 4), qa.QM_ERR_UNSUPPORTED), (dict(sin=7 * GIB + 4), qa.QM_ERR_UNSUPPORTED),
    (dict(starts=8 * GIB + 2), qa.QM_ERR_UNSUPPORTED), (dict(counts=8 * GIB + 4097), qa.QM_ERR_UNSUPPORTED),
]


@pytest.mark.parametrize("over,status", ROPE_REFUSALS + [(dict(k_out=None), qa.QM_ERR_NULL)], ids=str)
def test_norm_rope_refusals(lib, over, status):
    assert rope(lib, **over) == status


def test_strides_of_single_elements_are_not_looked_at(lib):
    """A dimension of size one may have any stride (the call gets as far as the alignment)."""
    odd = dict(k_out=4 * GIB + 2)
    assert rope(lib, B=1, q_strides=_strides(7, 1024, 128), **odd) == qa.QM_ERR_UNSUPPORTED
    assert rope(lib, N=1, k_strides=_strides(1024, -3, 128), **odd) == qa.QM_ERR_UNSUPPORTED
    assert rope(lib, H=1, Hkv=1, q_strides=_strides(1024, 128, 1), k_strides=_strides(0, 0, 1), **odd) == qa.QM_ERR_UNSUPPORTED


APPEND = dict(q=1 * GIB, k=2 * GIB, v=9 * GIB, q_out=3 * GIB, k_out=4 * GIB, k_cache=10 * GIB, v_cache=11 * GIB,
              page_table=12 * GIB, q_weight=5 * GIB, k_weight=5 * GIB + 4096, cos=6 * GIB, sin=7 * GIB,
              starts=8 * GIB, counts=8 * GIB + 4096, B=2, H=8, Hkv=2, N=100, d=128, rotary=128, table_rows=200,
              eps=1e-6, interleaved=0, num_pages=50, page_size=16, table_cols=10, k_scale=1.0, v_scale=1.0,
              q_strides=None, k_strides=None, v_strides=None, stream=None, dtype=1, layout=0, cache_dtype=1,
              cache_layout=0)


def append(lib, **over):
    return lib.qm_qk_norm_rope_append(*_args(APPEND, over))


@pytest.mark.parametrize("over,status", ROPE_REFUSALS + [
    (dict(v=None), qa.QM_ERR_NULL), (dict(k_cache=None), qa.QM_ERR_NULL), (dict(v_cache=None), qa.QM_ERR_NULL),
    (dict(page_table=None), qa.QM_ERR_NULL),
    (dict(num_pages=0), qa.QM_ERR_PAGE), (dict(table_cols=0), qa.QM_ERR_PAGE), (dict(page_size=0), qa.QM_ERR_PAGE),
    (dict(page_size=24), qa.QM_ERR_PAGE), (dict(page_size=8), qa.QM_ERR_PAGE), (dict(page_size=1 << 17), qa.QM_ERR_PAGE),
    (dict(table_cols=1 << 27, page_size=16), qa.QM_ERR_PAGE),
    (dict(cache_dtype=0), qa.QM_ERR_DTYPE), (dict(cache_dtype=3), qa.QM_ERR_DTYPE), (dict(cache_layout=-1), qa.QM_ERR_LAYOUT),
    (dict(k_scale=0.0), qa.QM_ERR_SCALE), (dict(v_scale=NAN), qa.QM_ERR_SCALE), (dict(k_scale=INF), qa.QM_ERR_SCALE),
    (dict(v_scale=1e-40), qa.QM_ERR_SCALE), (dict(v_strides=_strides(0, 4, 0)), qa.QM_ERR_STRIDE),
    (dict(v_cache=10 * GIB), qa.QM_ERR_ALIAS), (dict(k_cache=9 * GIB), qa.QM_ERR_ALIAS), (dict(v_cache=12 * GIB - 16), qa.QM_ERR_ALIAS),
    (dict(q_out=11 * GIB + 256), qa.QM_ERR_ALIAS), (dict(k_cache=10 * GIB + 8), qa.QM_ERR_UNSUPPORTED),
    (dict(page_table=12 * GIB + 2), qa.QM_ERR_UNSUPPORTED), (dict(v=9 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
    # without k_out the call is complete but for another argument
    (dict(k_out=None, v=9 * GIB + 2), qa.QM_ERR_UNSUPPORTED),
], ids=str)
def test_append_refusals(lib, over, status):
    assert append(lib, **over) == status


DECODE = dict(q=1 * GIB, k_cache=2 * GIB, v_cache=3 * GIB, o=4 * GIB, lse=5 * GIB, page_table=6 * GIB, lengths=7 * GIB,
              B=2, H=8, Hkv=2, d=128, num_pages=50, page_size=16, table_cols=10, max_length=100, scale=0.1,
              k_scale=1.0, v_scale=1.0, window=0, sinks=0, workspace=None, workspace_bytes=0, stream=None, dtype=1,
              cache_dtype=1, cache_layout=0)


@pytest.mark.parametrize("over,status", [
    (dict(q=None), qa.QM_ERR_NULL), (dict(k_cache=None), qa.QM_ERR_NULL), (dict(v_cache=None), qa.QM_ERR_NULL),
    (dict(o=None), qa.QM_ERR_NULL), (dict(lse=None), qa.QM_ERR_NULL), (dict(page_table=None), qa.QM_ERR_NULL),
    (dict(lengths=None), qa.QM_ERR_NULL), (dict(dtype=2), qa.QM_ERR_DTYPE), (dict(cache_dtype=0), qa.QM_ERR_DTYPE),
    (dict(B=0), qa.QM_ERR_SHAPE), (dict(H=7), qa.QM_ERR_SHAPE), (dict(Hkv=16), qa.QM_ERR_SHAPE), (dict(Hkv=0), qa.QM_ERR_SHAPE),
    (dict(B=1 << 25), qa.QM_ERR_SHAPE), (dict(d=192), qa.QM_ERR_HEADDIM),
    (dict(page_size=20), qa.QM_ERR_PAGE), (dict(num_pages=0), qa.QM_ERR_PAGE), (dict(table_cols=-1), qa.QM_ERR_PAGE),
    (dict(table_cols=1 << 27), qa.QM_ERR_PAGE), (dict(max_length=0), qa.QM_ERR_PAGE), (dict(cache_layout=2), qa.QM_ERR_LAYOUT),
    (dict(window=-1), qa.QM_ERR_WINDOW), (dict(sinks=-1), qa.QM_ERR_WINDOW),
    (dict(scale=INF), qa.QM_ERR_SCALE), (dict(k_scale=NAN), qa.QM_ERR_SCALE), (dict(v_scale=INF), qa.QM_ERR_SCALE),
    (dict(scale=3e38, k_scale=2.0), qa.QM_ERR_SCALE),
    (dict(o=1 * GIB), qa.QM_ERR_ALIAS), (dict(o=2 * GIB + 16), qa.QM_ERR_ALIAS), (dict(lse=3 * GIB), qa.QM_ERR_ALIAS),
    (dict(lse=4 * GIB), qa.QM_ERR_ALIAS), (dict(o=6 * GIB), qa.QM_ERR_ALIAS), (dict(lse=7 * GIB), qa.QM_ERR_ALIAS),
    (dict(q=1 * GIB + 2), qa.QM_ERR_UNSUPPORTED), (dict(lse=5 * GIB + 4), qa.QM_ERR_UNSUPPORTED),
    (dict(lengths=7 * GIB + 1), qa.QM_ERR_UNSUPPORTED), (dict(v_cache=3 * GIB + 8), qa.QM_ERR_UNSUPPORTED),
], ids=str)
def test_decode_refusals(lib, over, status):
    assert lib.qm_attn_decode(*_args(DECODE, over)) == status


def test_workspace_refusals(lib):
    need = ctypes.c_size_t(77)
    good = dict(B=2, H=8, Hkv=2, d=128, page_size=16, table_cols=10, max_length=100, window=0, sinks=0)
    for over, status in [(dict(B=0), qa.QM_ERR_SHAPE), (dict(Hkv=3), qa.QM_ERR_SHAPE), (dict(d=32), qa.QM_ERR_HEADDIM),
                         (dict(page_size=15), qa.QM_ERR_PAGE), (dict(table_cols=0), qa.QM_ERR_PAGE),
                         (dict(max_length=-5), qa.QM_ERR_PAGE), (dict(table_cols=1 << 28), qa.QM_ERR_PAGE),
                         (dict(window=-2), qa.QM_ERR_WINDOW), (dict(sinks=-1), qa.QM_ERR_WINDOW)]:
        assert lib.qm_attn_decode_workspace(*dict(good, **over).values(), ctypes.byref(need)) == status
    assert lib.qm_attn_decode_workspace(*good.values(), None) == qa.QM_ERR_NULL
    assert need.value == 77


WINDOW = dict(q=1 * GIB, k=2 * GIB, v=3 * GIB, o=4 * GIB, lse=5 * GIB, B=1, H=4, Hkv=2, N=128, d_qk=64, d_v=64,
              scale=0.125, window=10, sinks=2, stream=None, dtype=0, layout=0)


@pytest.mark.parametrize("over,status", [
    (dict(window=0), qa.QM_ERR_WINDOW), (dict(window=-4), qa.QM_ERR_WINDOW), (dict(sinks=-1), qa.QM_ERR_WINDOW),
    (dict(q=None), qa.QM_ERR_NULL), (dict(N=0), qa.QM_ERR_SHAPE), (dict(Hkv=3), qa.QM_ERR_SHAPE), (dict(d_qk=96), qa.QM_ERR_HEADDIM),
    (dict(dtype=2), qa.QM_ERR_DTYPE), (dict(scale=NAN), qa.QM_ERR_SCALE), (dict(layout=5), qa.QM_ERR_LAYOUT),
    (dict(layout=1, d_qk=192, d_v=128), qa.QM_ERR_LAYOUT), (dict(o=1 * GIB), qa.QM_ERR_ALIAS), (dict(k=2 * GIB + 8), qa.QM_ERR_UNSUPPORTED),
], ids=str)
def test_window_refusals(lib, over, status):
    assert qa.qm_attn_fwd_window(**dict(WINDOW, **over)) == status


def test_status_texts(lib):
    codes = [qa.QM_ERR_WINDOW, qa.QM_ERR_PAGE, qa.QM_ERR_ROTARY, qa.QM_ERR_STRIDE, qa.QM_ERR_WORKSPACE, qa.QM_ERR_TILE]
    texts = {qa.strerror(c) for c in codes}
    assert len(texts) == len(codes) and "unknown status" not in texts


def test_host_tensors_are_refused():
    torch = pytest.importorskip("torch")
    x = torch.zeros(1, 2, 4, 64, dtype=torch.bfloat16)
    table = torch.zeros(1, 1, dtype=torch.int32)
    cache = torch.zeros(1, 2, 16, 64, dtype=torch.bfloat16)
    for call in (lambda: qa.qk_norm_rope(x, x), lambda: qa.qk_norm_rope_append(x, x, x, cache, cache, table),
                 lambda: qa.decode(x[:, :, 0], cache, cache, table, table[0]), lambda: qa.fwd_window(x, x, x, 2)):
        with pytest.raises(ValueError, match="ROCm device"):
            call()


def test_a_stream_of_another_device_is_refused():
    torch = pytest.importorskip("torch")
    from paper_2506_12355_amd import binding

    class Stream:
        device = torch.device("cuda", 1)
        cuda_stream = 7

    def entry(*args):
        raise AssertionError("the library was called")

    with pytest.raises(ValueError, match="stream must be"):
        binding._enqueue(entry, torch.device("cuda", 0), Stream(), (), ())
