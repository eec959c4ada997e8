"""The operators around the attention forward that serve a model: head norms with the
position rotation, a paged cache of keys and values, and attention of new tokens over it.

As in ``binding``: argument marshalling only, on torch's memory and streams; every step
runs in the gfx950 kernels of the library (``include/qm_attn.h``).  Outputs and workspaces
that a call makes are tensors of the stream it runs on (see :func:`binding.fwd`).

The cache is two tensors of pages, [num_pages, Hkv, page_size, d] (``cache_layout``
"bhnd") or [num_pages, page_size, Hkv, d] ("bnhd"), of the model's 16-bit type or
``float8_e4m3fn`` (or ``uint8`` E4M3 codes), and a page table [B, columns] of int32: token
t of sequence b is row t % page_size of page ``page_table[b, t // page_size]``.
"""
from __future__ import annotations

import ctypes
import functools

from .binding import (QM_BHND, QM_BNHD, QM_OK, QmAttnError, _dtype_code, _enqueue, _int32,
                      _pool_of, load_library, strerror)

QM_E4M3 = 2   # qm_dtype_t: cached keys and values

_LAYOUTS = {"bhnd": QM_BHND, "bnhd": QM_BNHD}
_Strides = ctypes.c_longlong * 3
_MOST = 2 ** 31 - 1   # no bound on lengths but the page table's


# The checks below read each property of a tensor once and put off what a message needs
# until there is one: a call of one token takes the GPU a few microseconds, less than its
# arguments take the host.

def _layout_code(layout, name="layout"):
    code = _LAYOUTS.get(layout)
    if code is None:
        raise ValueError(f"{name} must be 'bhnd' or 'bnhd', not {layout!r}")
    return code


def _queries(q):
    """The device index of q, which must be a ROCm tensor, and its type and the type's code."""
    if not q.is_cuda:
        raise ValueError("q must be on a ROCm device")
    return q.get_device(), q.dtype, _dtype_code(q)


def _elsewhere(name, t, index):
    """The kernels follow device pointers: every tensor is on the queries' device."""
    return ValueError(f"{name} must be on the queries' device cuda:{index}, not {t.device}")


def _rows(name, t, dtype, index, layout):
    """Sizes (B, N, heads, d) of a [B, heads, N, d] or [B, N, heads, d] tensor whose
    columns are contiguous, and its strides for the library (None: contiguous)."""
    size = t.shape
    if len(size) != 4:
        raise ValueError(f"{name} must have shape {'[B, N, heads, d]' if layout else '[B, heads, N, d]'}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.get_device() != index:
        raise _elsewhere(name, t, index)
    if layout:
        size = tuple(size)
    else:
        B, heads, N, d = size
        size = (B, N, heads, d)
    if t.is_contiguous():
        return size, None
    s = t.stride()
    if s[3] != 1:
        raise ValueError(f"{name}'s columns must be contiguous")
    return size, _Strides(s[0], s[1], s[2]) if layout else _Strides(s[0], s[2], s[1])


def _misfit(name, t, size, index, dtype):
    if t.get_device() != index:
        return _elsewhere(name, t, index)
    return ValueError(f"{name} must be a contiguous {list(size)} tensor of {dtype}")


def _vectors(names, a, b, size, index, dtype):
    """The addresses of two contiguous tensors of `size`, None for None."""
    if a is not None:
        if a.shape != size or a.dtype is not dtype or a.get_device() != index or not a.is_contiguous():
            raise _misfit(names[0], a, size, index, dtype)
        a = a.data_ptr()
    if b is not None:
        if b.shape != size or b.dtype is not dtype or b.get_device() != index or not b.is_contiguous():
            raise _misfit(names[1], b, size, index, dtype)
        b = b.data_ptr()
    return a, b


def _vector(name, t, size, index, dtype):
    """The address of a contiguous tensor of `size`."""
    if t.shape != size or t.dtype is not dtype or t.get_device() != index or not t.is_contiguous():
        raise _misfit(name, t, size, index, dtype)
    return t.data_ptr()


def _new(torch, like):
    """A new contiguous tensor shaped like `like` (empty_like is the shorter call, but
    keeps a subclass and strides)."""
    if type(like) is torch.Tensor and like.is_contiguous():
        return torch.empty_like(like)
    return torch.empty(like.shape, dtype=like.dtype, device=like.device)


def _angles(cos, sin, index):
    """Addresses of the rotation's table, its rows and the columns it rotates."""
    if cos is None and sin is None:
        return None, None, 0, 0
    if cos is None or sin is None:
        raise ValueError("cos and sin are given together")
    size = cos.shape
    if len(size) != 2 or sin.shape != size:
        raise ValueError("cos and sin must have shape [positions, rotary / 2]")
    return (*_vectors(("cos", "sin"), cos, sin, size, index, _torch().float32), 2 * size[1], size[0])


@functools.lru_cache(maxsize=1)
def _torch():
    import torch
    return torch


@functools.lru_cache(maxsize=64)
def _device(index):
    return _torch().device("cuda", index)


def _cache(k_cache, v_cache, page_table, B, d, dtype, code, index, cache_layout):
    """Cache arguments, checked: (num_pages, page_size, heads, columns, the page table's
    address, cache type, layout)."""
    layout = _layout_code(cache_layout, "cache_layout")
    size, kind = k_cache.shape, k_cache.dtype
    if len(size) != 4 or v_cache.shape != size:
        raise ValueError("k_cache and v_cache must have one shape, "
                         + ("[pages, page_size, Hkv, d]" if layout else "[pages, Hkv, page_size, d]"))
    if v_cache.dtype is not kind:
        raise TypeError("k_cache and v_cache must have the same dtype")
    if kind is not dtype:
        if kind not in (_torch().float8_e4m3fn, _torch().uint8):
            raise TypeError(f"the cache must be {dtype}, float8_e4m3fn or uint8, not {kind}")
        code = QM_E4M3
    if not (k_cache.is_contiguous() and v_cache.is_contiguous()):
        raise ValueError("k_cache and v_cache must be contiguous")
    if k_cache.get_device() != index or v_cache.get_device() != index:
        raise _elsewhere("the cache", v_cache if k_cache.get_device() == index else k_cache, index)
    pages, heads, page_size, width = size
    if layout:
        heads, page_size = page_size, heads
    if width != d:
        raise ValueError("the cache must have the queries' width")
    columns = page_table.shape
    if len(columns) != 2 or columns[0] != B:
        raise ValueError("page_table must have shape [B, columns]")
    table = _vector("page_table", page_table, columns, index, _torch().int32)
    return pages, page_size, heads, columns[1], table, code, layout


def _pair_axes(axes, pairs, count):
    """The library's array of each pair's axis."""
    if axes is None:
        if count != 1:
            raise ValueError("axes must name each rotated pair's axis where positions has several")
        return bytes(pairs)
    axes = tuple(axes)
    if len(axes) != pairs:
        raise ValueError(f"axes must name the axis of each of the {pairs} rotated pairs, not of {len(axes)}")
    try:
        own = bytes(axes)
    except ValueError:   # one of them below 0 or above 255
        own = None
    if own is None or (own and max(own) >= count):
        raise ValueError(f"axes must be from 0 to {count - 1}, positions' axes")
    return own


def _positions(positions, axes, rotary, B, N, index):
    """The library's arguments for positions of several axes: addresses, and their number."""
    size = positions.shape
    if len(size) != 3 or not 1 <= size[0] <= 4:
        raise ValueError("positions must have shape [axes, B, N] with 1 to 4 axes")
    at = _vector("positions", positions, (size[0], B, N), index, _torch().int32)
    return at, _pair_axes(axes, rotary // 2, size[0]), size[0]


def qk_norm_rope(q, k, cos=None, sin=None, q_weight=None, k_weight=None, eps: float = 1e-6,
                 starts=None, counts=None, interleaved: bool = False, q_out=None, k_out=None,
                 stream=None, layout: str = "bhnd", positions=None, axes=None):
    """Norm of each query and key head and rotation by its token's position, in one pass.

    q is [B, H, N, d] and k [B, Hkv, N, d] float16 or bfloat16 (``layout="bnhd"``:
    [B, N, heads, d]), d 64 or 128.  Any strides that are multiples of 8 elements are
    taken, so both may be views into one projection's output, or transposed ones, as
    long as the d columns lie together.  Each row is divided by sqrt(mean(x^2) + eps) and
    multiplied by ``q_weight`` or ``k_weight`` [d] (None: that tensor is not normalised),
    then its first columns are rotated by the angles whose ``cos`` and ``sin`` [positions,
    rotary / 2] (float32; None: no rotation) stand in the row of the token's position,
    ``starts[b]`` (int32 [B]; None: 0) + t.  Pair j is columns (j, j + rotary / 2), or
    (2 j, 2 j + 1) with ``interleaved``.  All in float32, rounded once.

    ``counts`` (int32 [B]; None: N): rows of a padded batch past them are written as
    zeros.  A position outside the table gives NaN rows.  Returns (q_out, k_out),
    contiguous in ``layout``, as ``fwd`` and ``fwd_window`` take them
    (``qm_qk_norm_rope``).

    ``positions`` (int32 [A, B, N], A from 1 to 4; instead of ``starts``): positions on
    several axes, such as time, height and width of a picture's parts.  ``axes``, a
    sequence of rotary / 2 whole numbers below A (None where A is 1), names the axis of
    each pair: pair j of token t of sequence b turns by row ``positions[axes[j], b, t]`` of
    the table's column j.  Places past ``counts``, and axes that no pair has, are not looked
    at (``qm_qk_norm_rope_axes``)."""
    index, dtype, code = _queries(q)
    lay = _layout_code(layout)
    (B, N, H, d), qs = _rows("q", q, dtype, index, lay)
    (Bk, Nk, Hkv, dk), ks = _rows("k", k, dtype, index, lay)
    if Bk != B or Nk != N or dk != d:
        raise ValueError("k must match q in B, N and d")
    c, s, rotary, table_rows = _angles(cos, sin, index)
    torch = _torch()
    qw, kw = _vectors(("q_weight", "k_weight"), q_weight, k_weight, (d,), index, dtype)
    first, held = _vectors(("starts", "counts"), starts, counts, (B,), index, torch.int32)
    if positions is not None:
        if starts is not None:
            raise ValueError("starts must be None where positions are given")
        entry, at = load_library().qm_qk_norm_rope_axes, _positions(positions, axes, rotary, B, N, index)
    else:
        if axes is not None:
            raise ValueError("axes are given with positions")
        entry, at = load_library().qm_qk_norm_rope, (first,)
    with _pool_of(stream, q_out is None or k_out is None):
        if q_out is None:
            q_out = _new(torch, q)
        else:
            _vector("q_out", q_out, q.shape, index, dtype)
        if k_out is None:
            k_out = _new(torch, k)
        else:
            _vector("k_out", k_out, k.shape, index, dtype)
    _enqueue(entry, _device(index), stream,
             (q.data_ptr(), k.data_ptr(), q_out.data_ptr(), k_out.data_ptr(), qw, kw, c, s, *at,
              held, B, H, Hkv, N, d, rotary, table_rows, float(eps), 1 if interleaved else 0, qs, ks),
             (code, lay))
    return q_out, k_out


def qk_norm_rope_append(q, k, v, k_cache, v_cache, page_table, starts=None, cos=None, sin=None,
                        q_weight=None, k_weight=None, eps: float = 1e-6, counts=None,
                        interleaved: bool = False, k_scale: float = 1.0, v_scale: float = 1.0,
                        q_out=None, k_out=None, stream=None, layout: str = "bhnd",
                        cache_layout: str = "bhnd", positions=None, axes=None):
    """:func:`qk_norm_rope`, with the keys and the values v written to a paged cache:
    token t of sequence b at position ``starts[b]`` + t, rows past ``counts`` not at all.

    The cache holds key / ``k_scale`` and value / ``v_scale`` (with E4M3 pages, values
    beyond 448 as 448).  Its pages past a sequence's tokens are left as they were, and so
    are the entries of ``page_table`` that name them.  A token whose position has no page
    (or no angle, or a page number out of range) is not stored.  A page that is written
    belongs to one sequence and stands once in its row.  v has k's shape and any
    strides as q and k; ``k_out``, where given, receives the keys as ``qk_norm_rope``
    returns them.  Without cos, sin and weights the keys are stored as they are.  Returns
    q_out (``qm_qk_norm_rope_append``).

    With ``positions`` and ``axes``, as in :func:`qk_norm_rope`, the rotation takes those,
    and ``starts`` says only where in the cache a sequence's tokens go
    (``qm_qk_norm_rope_append_axes``)."""
    index, dtype, code = _queries(q)
    lay = _layout_code(layout)
    (B, N, H, d), qs = _rows("q", q, dtype, index, lay)
    (Bk, Nk, Hkv, dk), ks = _rows("k", k, dtype, index, lay)
    size_v, vs = _rows("v", v, dtype, index, lay)
    if Bk != B or Nk != N or dk != d or size_v != (B, N, Hkv, d):
        raise ValueError("k and v must have one shape and match q in B, N and d")
    c, s, rotary, table_rows = _angles(cos, sin, index)
    pages, page_size, heads, table_columns, table, kind, cache_lay = _cache(
        k_cache, v_cache, page_table, B, d, dtype, code, index, cache_layout)
    if heads != Hkv:
        raise ValueError("the cache must have the keys' heads")
    torch = _torch()
    qw, kw = _vectors(("q_weight", "k_weight"), q_weight, k_weight, (d,), index, dtype)
    first, held = _vectors(("starts", "counts"), starts, counts, (B,), index, torch.int32)
    if positions is not None:
        entry = load_library().qm_qk_norm_rope_append_axes
        at = (*_positions(positions, axes, rotary, B, N, index), first)
    else:
        if axes is not None:
            raise ValueError("axes are given with positions")
        entry, at = load_library().qm_qk_norm_rope_append, (first,)
    if q_out is None:
        with _pool_of(stream, True):
            q_out = _new(torch, q)
    else:
        _vector("q_out", q_out, q.shape, index, dtype)
    if k_out is not None:
        k_out = _vector("k_out", k_out, k.shape, index, dtype)
    _enqueue(entry, _device(index), stream,
             (q.data_ptr(), k.data_ptr(), v.data_ptr(), q_out.data_ptr(), k_out, k_cache.data_ptr(),
              v_cache.data_ptr(), table, qw, kw, c, s, *at, held, B, H, Hkv, N, d, rotary,
              table_rows, float(eps), 1 if interleaved else 0, pages, page_size, table_columns,
              float(k_scale), float(v_scale), qs, ks, vs),
             (code, lay, kind, cache_lay))
    return q_out


def _lines(name, t, size, dtype, index):
    """The elements from row to row of a [..., D] tensor of `size` whose rows lie at equal
    distances, each contiguous."""
    if t.shape != size:
        raise ValueError(f"{name} must have shape {list(size)}, not {list(t.shape)}")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, not {t.dtype}")
    if t.get_device() != index:
        raise _elsewhere(name, t, index)
    if t.is_contiguous():
        return size[-1]
    stride, step, next_ = t.stride(), None, 0
    if size[-1] != 1 and stride[-1] != 1:
        raise ValueError(f"{name}'s columns must be contiguous")
    for n, s in zip(reversed(size[:-1]), reversed(stride[:-1])):
        if n == 1:
            continue
        if step is None:
            step = s
        elif s != next_:
            raise ValueError(f"{name}'s rows must lie at equal distances")
        next_ = s * n
    return size[-1] if step is None else step


def _normed(x, weight, residual, sum_out):
    """The checks that both norms share: device index, type, its code, rows, width, the
    strides of x, residual and sum_out, and the weight's address."""
    if not x.is_cuda:
        raise ValueError("x must be on a ROCm device")
    size = x.shape
    if not size or not x.numel():
        raise ValueError("x must have shape [..., width], with a row at least")
    index, dtype, code = x.get_device(), x.dtype, _dtype_code(x, "x")
    width = size[-1]
    lines = _lines("x", x, size, dtype, index)
    if weight is not None:
        weight = _vector("weight", weight, (width,), index, dtype)
    further = after = width
    if residual is not None:
        further = _lines("residual", residual, size, dtype, index)
        if sum_out is not None:
            after = _lines("sum_out", sum_out, size, dtype, index)
    elif sum_out is not None:
        raise ValueError("sum_out is given with a residual")
    rows = _int32(x.numel() // width, "x's number of rows")
    return index, dtype, code, rows, width, lines, further, after, weight


def rms_norm(x, weight=None, residual=None, eps: float = 1e-6, out=None, sum_out=None, stream=None):
    """Norm of whole rows, of x or of its sum with a residual, in one pass.

    x and ``residual`` (None: none) are [..., width] float16 or bfloat16, width a multiple of
    8 up to 32768, their rows contiguous and at equal distances of a multiple of 8 elements
    (views into a wider projection's output, say, or one row expanded).  With s = x + residual,
    y = s * ``weight`` / sqrt(mean(s^2) + eps) (``weight`` [width], or None), in float32,
    rounded once.

    Returns (y, sum): y contiguous, and s rounded to x's type (None without a residual).
    ``sum_out`` may be ``residual`` (or x) itself, whose place the sum then takes.
    (``qm_rms_norm``)"""
    index, dtype, code, rows, width, lines, further, after, w = _normed(x, weight, residual, sum_out)
    torch = _torch()
    make_sum = residual is not None and sum_out is None
    with _pool_of(stream, out is None or make_sum):
        if out is None:
            out = _new(torch, x)
        else:
            _vector("out", out, x.shape, index, dtype)
        if make_sum:
            sum_out = _new(torch, x)
    _enqueue(load_library().qm_rms_norm, _device(index), stream,
             (x.data_ptr(), None if residual is None else residual.data_ptr(), w, out.data_ptr(),
              None if sum_out is None else sum_out.data_ptr(), rows, width, lines, further, after,
              float(eps)), (code,))
    return out, sum_out


def rms_norm_fp8(x, weight=None, residual=None, eps: float = 1e-6, scale: float | None = None,
                 group: int | None = None, out=None, scales=None, sum_out=None, stream=None):
    """:func:`rms_norm` with a result of E4M3 codes, y = scale * code.

    ``scale``: one factor for all, as ``fwd_fp8`` takes (y beyond 448 of it as 448).  None:
    a factor for each row, or for each ``group`` (32, 64, 128 or 256, dividing width) of a
    row's columns, max |y| / 448 over them, at least 2^-126.

    Returns (codes, scales, sum): ``float8_e4m3fn`` codes shaped like x (``out`` may be
    uint8), float32 scales [..., 1] or [..., width / group] (None with ``scale``), and the sum
    as there.  (``qm_rms_norm_fp8``)"""
    index, dtype, code, rows, width, lines, further, after, w = _normed(x, weight, residual, sum_out)
    torch = _torch()
    make_sum = residual is not None and sum_out is None
    size = x.shape
    if scale is not None:
        if group is not None or scales is not None:
            raise ValueError("scale is one factor for all: group and scales must be None")
        group = 0
    else:
        group = 0 if group is None else _int32(group, "group")
        if group not in (0, 32, 64, 128, 256) or (group and width % group):
            raise ValueError("group must be 32, 64, 128 or 256 and divide x's width")
    with _pool_of(stream, out is None or make_sum or (scale is None and scales is None)):
        if out is None:
            out = torch.empty(size, dtype=torch.float8_e4m3fn, device=_device(index))
        else:
            _vector("out", out, size, index,
                    out.dtype if out.dtype is torch.uint8 else torch.float8_e4m3fn)
        if scale is None:
            shape = (*size[:-1], width // group if group else 1)
            if scales is None:
                scales = torch.empty(shape, dtype=torch.float32, device=_device(index))
            else:
                _vector("scales", scales, shape, index, torch.float32)
        if make_sum:
            sum_out = _new(torch, x)
    _enqueue(load_library().qm_rms_norm_fp8, _device(index), stream,
             (x.data_ptr(), None if residual is None else residual.data_ptr(), w, out.data_ptr(),
              None if scales is None else scales.data_ptr(),
              None if sum_out is None else sum_out.data_ptr(), rows, width, lines, further, after,
              float(eps), 1.0 if scale is None else float(scale), group), (code,))
    return out, scales, sum_out


@functools.lru_cache(maxsize=1024)
def _workspace_bytes(entry, index, *sizes) -> int:
    """Workspace of a decode call of these sizes on device `index` (sizes alone decide), of
    which the library's `entry` tells."""
    import torch
    need = ctypes.c_size_t()
    with torch.cuda.device(index):
        status = getattr(load_library(), entry)(*sizes, ctypes.byref(need))
    if status != QM_OK:
        raise QmAttnError(status, strerror(status))
    return need.value


def decode_workspace(q, k_cache, page_table, max_length: int | None = None,
                     window: int | None = None, sinks: int = 0, cache_layout: str = "bhnd") -> int:
    """Bytes of workspace that :func:`decode` needs for these arguments (0: none)."""
    index, dtype, code = _queries(q)
    if q.dim() != 3:
        raise ValueError("q must have shape [B, H, d]")
    B, H, d = q.shape
    _, page_size, heads, columns, _, _, _ = _cache(k_cache, k_cache, page_table, B, d, dtype, code,
                                                index, cache_layout)
    return _workspace_bytes("qm_attn_decode_workspace", index, B, H, heads, d, page_size, columns,
                            _MOST if max_length is None else _int32(max_length, "max_length"),
                            0 if window is None else _window(window), _int32(sinks, "sinks"))


def _window(window) -> int:
    window = _int32(window, "window")
    if window < 1:
        raise ValueError("window must be at least 1 (None: every cached token is visible)")
    return window


def decode(q, k_cache, v_cache, page_table, lengths, scale: float | None = None,
           window: int | None = None, sinks: int = 0, k_scale: float = 1.0, v_scale: float = 1.0,
           max_length: int | None = None, out=None, lse=None, workspace=None, stream=None,
           cache_layout: str = "bhnd"):
    """Attention of one new token per sequence over a paged cache.

    q is [B, H, d] float16 or bfloat16, d 64 or 128; query head h reads key/value head
    h // (H // Hkv) of the cache, whose real values are ``k_scale`` and ``v_scale`` times
    what it holds.  ``lengths`` (int32 [B]) counts each sequence's cached tokens, the new
    one's among them.  ``window``: only the last ``window`` of them and the first
    ``sinks`` are visible, as for the last row of ``fwd_window``.

    Returns (o [B, H, d], lse float32 [B, H]).  Length 0 gives o = 0 and lse = -inf; a
    length below 0, above ``max_length`` or beyond the page table, or a page number out of
    range, gives NaN for that sequence.  ``max_length`` is a bound that the host knows
    (None: what the page table can hold); the work is split for it, so a close one is
    faster.  ``workspace``: a uint8 tensor of :func:`decode_workspace` bytes (None: one is
    allocated on the call's stream); two calls that may run at once need one each.
    ``scale`` defaults to 1/sqrt(d) rounded to float32.  (``qm_attn_decode``)"""
    return _decode(q, k_cache, v_cache, page_table, lengths, scale, k_scale, v_scale, max_length, out, lse,
                   workspace, stream, cache_layout,
                   window=(0 if window is None else _window(window), _int32(sinks, "sinks")))


def _decode(q, k_cache, v_cache, page_table, lengths, scale, k_scale, v_scale, max_length, out, lse,
            workspace, stream, cache_layout, window=None, prefix=None):
    """Both decoding calls: with a window and first keys, or with a prefix's page table and
    length."""
    index, dtype, code = _queries(q)
    if q.dim() != 3 or not q.is_contiguous():
        raise ValueError("q must be a contiguous [B, H, d] tensor")
    B, H, d = q.shape
    pages, page_size, Hkv, columns, table, kind, cache_lay = _cache(
        k_cache, v_cache, page_table, B, d, dtype, code, index, cache_layout)
    torch = _torch()
    if lengths is None:
        raise ValueError("lengths must be given")
    lens = _vector("lengths", lengths, (B,), index, torch.int32)
    scale = 1.0 / d ** 0.5 if scale is None else float(scale)   # rounded to float32 by the call
    if prefix is not None:
        prefix_table, prefix_length = prefix
        prefix_length = _int32(prefix_length, "prefix_length")
        if prefix_length < 0:
            raise ValueError("prefix_length must be 0 or more")
        if prefix_table is None:
            if prefix_length:
                raise ValueError("prefix_table must be given with a prefix")
            pages_of_prefix, prefix_columns = None, 0
        else:
            prefix_columns = prefix_table.numel()
            pages_of_prefix = _vector("prefix_table", prefix_table, (prefix_columns,), index, torch.int32)
    most = _MOST if max_length is None else _int32(max_length, "max_length")
    with _pool_of(stream, out is None or lse is None or workspace is None):
        if out is None:
            out = _new(torch, q)
        else:
            _vector("out", out, q.shape, index, dtype)
        if lse is None:
            lse = torch.empty(B, H, dtype=torch.float32, device=_device(index))
        else:
            _vector("lse", lse, (B, H), index, torch.float32)
        if prefix is None:
            need = _workspace_bytes("qm_attn_decode_workspace", index, B, H, Hkv, d, page_size, columns,
                                    most, *window)
        else:
            need = _workspace_bytes("qm_attn_decode_shared_workspace", index, B, H, Hkv, d, page_size,
                                    columns, prefix_length, most)
        if workspace is not None:
            if workspace.dtype is not torch.uint8 or workspace.dim() != 1 or not workspace.is_contiguous():
                raise ValueError("workspace must be a contiguous 1-D uint8 tensor")
            if workspace.get_device() != index:
                raise _elsewhere("workspace", workspace, index)
            ws, given = workspace.data_ptr(), workspace.numel()
        elif need:
            workspace = torch.empty(need, dtype=torch.uint8, device=_device(index))
            ws, given = workspace.data_ptr(), need
        else:
            ws, given = None, 0
    tensors = (q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), out.data_ptr(), lse.data_ptr(),
               table, lens)
    if prefix is None:
        _enqueue(load_library().qm_attn_decode, _device(index), stream,
                 (*tensors, B, H, Hkv, d, pages, page_size, columns, most, scale, float(k_scale),
                  float(v_scale), *window, ws, given),
                 (code, kind, cache_lay))
    else:
        _enqueue(load_library().qm_attn_decode_shared, _device(index), stream,
                 (*tensors, pages_of_prefix, B, H, Hkv, d, pages, page_size, columns, prefix_columns,
                  prefix_length, most, scale, float(k_scale), float(v_scale), ws, given),
                 (code, kind, cache_lay))
    return out, lse


def decode_shared_workspace(q, k_cache, page_table, prefix_length: int, max_length: int | None = None,
                            cache_layout: str = "bhnd") -> int:
    """Bytes of workspace that :func:`decode_shared` needs for these arguments."""
    index, dtype, code = _queries(q)
    if q.dim() != 3:
        raise ValueError("q must have shape [B, H, d]")
    B, H, d = q.shape
    _, page_size, heads, columns, _, _, _ = _cache(k_cache, k_cache, page_table, B, d, dtype, code,
                                                index, cache_layout)
    return _workspace_bytes("qm_attn_decode_shared_workspace", index, B, H, heads, d, page_size, columns,
                            _int32(prefix_length, "prefix_length"),
                            _MOST if max_length is None else _int32(max_length, "max_length"))


def decode_shared(q, k_cache, v_cache, page_table, lengths, prefix_table, prefix_length: int,
                  scale: float | None = None, k_scale: float = 1.0, v_scale: float = 1.0,
                  max_length: int | None = None, out=None, lse=None, workspace=None, stream=None,
                  cache_layout: str = "bhnd"):
    """:func:`decode` for sequences that share their first ``prefix_length`` tokens, whose
    pages ``prefix_table`` (int32 [columns]) names for all of them: what is read of the
    prefix is read for many queries at once.

    ``lengths`` counts all of a sequence's tokens, the prefix's among them.  Token t of a
    sequence from ``prefix_length`` on is in page ``page_table[b, t // page_size]``, as for
    ``decode``; entries for earlier tokens are not looked at.  ``prefix_length`` need not be
    a multiple of the page size, and 0 is ``decode`` (``prefix_table`` may then be None).

    Returns (o [B, H, d], lse float32 [B, H]).  Length 0 (a free slot) gives o = 0 and lse
    = -inf; any other length below ``prefix_length`` gives NaN, as do the lengths and page
    numbers out of range that do for ``decode`` (a page of the prefix for every sequence).
    ``max_length``, also where the page table could hold more, tells how the work is best
    divided.  ``workspace``: as for ``decode``, of :func:`decode_shared_workspace` bytes.  For
    layers with a window call ``decode``, with the prefix's pages in each sequence's row.
    (``qm_attn_decode_shared``)"""
    return _decode(q, k_cache, v_cache, page_table, lengths, scale, k_scale, v_scale, max_length, out, lse,
                   workspace, stream, cache_layout, prefix=(prefix_table, prefix_length))
