"""ctypes binding of the C-ABI attention library (include/qm_attn.h).

Argument marshalling only: every step of the attention forward runs in the
gfx950 kernels.  PyTorch supplies device memory and the current HIP stream.
There is no fallback: if ``libqm_attn.so`` is missing, loading fails loudly.
"""
from __future__ import annotations

import contextlib
import ctypes
import operator
import os
import threading

PKG_DIR = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(PKG_DIR, "libqm_attn.so")
DEBUG_LIB_PATH = os.path.join(PKG_DIR, "libqm_attn_debug.so")

# qm_dtype_t
QM_F16 = 0
QM_BF16 = 1

# qm_layout_t
QM_BHND = 0
QM_BNHD = 1

# status codes
QM_OK = 0
QM_ERR_NULL = -1
QM_ERR_SHAPE = -2
QM_ERR_HEADDIM = -3
QM_ERR_DTYPE = -4
QM_ERR_SCALE = -5
QM_ERR_ALIAS = -6
QM_ERR_CAUSAL = -7
QM_ERR_LAUNCH = -8
QM_ERR_UNSUPPORTED = -9
QM_ERR_LAYOUT = -10
QM_ERR_TILE = -11
QM_ERR_WINDOW = -12
QM_ERR_PAGE = -13
QM_ERR_ROTARY = -14
QM_ERR_STRIDE = -15
QM_ERR_WORKSPACE = -16

_lib = None
_lock = threading.Lock()


class QmAttnError(RuntimeError):
    """A non-zero status from the C library."""

    def __init__(self, status: int, message: str):
        super().__init__(f"qm_attn_fwd failed with status {status}: {message}")
        self.status = status


def _declare(lib: ctypes.CDLL) -> ctypes.CDLL:
    """Argument and result types of every entry point of ``include/qm_attn.h``."""
    lib.qm_attn_fwd.argtypes = [
        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
        ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
        ctypes.c_float, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
    ]
    lib.qm_attn_fwd.restype = ctypes.c_int
    lib.qm_attn_fwd_gqa.argtypes = [
        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
        ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
        ctypes.c_float, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
    ]
    lib.qm_attn_fwd_gqa.restype = ctypes.c_int
    lib.qm_attn_fwd_mla.argtypes = [
        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
        ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
        ctypes.c_float, ctypes.c_int, ctypes.c_void_p, ctypes.c_int,
    ]
    lib.qm_attn_fwd_mla.restype = ctypes.c_int
    lib.qm_attn_fwd_fp8.argtypes = [
        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
        ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
        ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_int,
        ctypes.c_void_p,
    ]
    lib.qm_attn_fwd_fp8.restype = ctypes.c_int
    lib.qm_attn_fwd_layout.argtypes = [
        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
        ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
        ctypes.c_float, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
    ]
    lib.qm_attn_fwd_layout.restype = ctypes.c_int
    lib.qm_attn_fwd_fp8_layout.argtypes = [
        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
        ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
        ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_float, ctypes.c_int,
        ctypes.c_void_p, ctypes.c_int,
    ]
    lib.qm_attn_fwd_fp8_layout.restype = ctypes.c_int
    lib.qm_attn_fwd_window.argtypes = [
        ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p,
        ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
        ctypes.c_float, ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_int, ctypes.c_int,
    ]
    lib.qm_attn_fwd_window.restype = ctypes.c_int
    P, I, F = ctypes.c_void_p, ctypes.c_int, ctypes.c_float
    lib.qm_qk_norm_rope.argtypes = [P] * 10 + [I] * 7 + [F, I] + [P] * 3 + [I] * 2
    lib.qm_qk_norm_rope.restype = ctypes.c_int
    lib.qm_qk_norm_rope_append.argtypes = (
        [P] * 14 + [I] * 7 + [F] + [I] * 4 + [F] * 2 + [P] * 4 + [I] * 4)
    lib.qm_qk_norm_rope_append.restype = ctypes.c_int
    lib.qm_attn_decode.argtypes = (
        [P] * 7 + [I] * 8 + [F] * 3 + [I] * 2 + [P, ctypes.c_size_t, P] + [I] * 3)
    lib.qm_attn_decode.restype = ctypes.c_int
    lib.qm_attn_decode_workspace.argtypes = [I] * 9 + [P]
    lib.qm_attn_decode_workspace.restype = ctypes.c_int
    lib.qm_attn_set_tile_rows.argtypes = [ctypes.c_int]
    lib.qm_attn_set_tile_rows.restype = ctypes.c_int
    lib.qm_attn_strerror.argtypes = [ctypes.c_int]
    lib.qm_attn_strerror.restype = ctypes.c_char_p
    return lib


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Load (once) and return the HIP library; raise if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is not None:
            return _lib
        _lib = open_library(path)
        return _lib


def open_library(path: str) -> ctypes.CDLL:
    """A separate handle on a build of the library at ``path`` (the tests use
    it for the checking build, ``libqm_attn_debug.so``); raises if missing."""
    if not os.path.exists(path):
        raise RuntimeError(
            f"{path} is missing: the HIP attention library has not been built "
            "(run `python -m paper_2506_12355_amd.build`)")
    return _declare(ctypes.CDLL(path))


def strerror(status: int) -> str:
    return load_library().qm_attn_strerror(int(status)).decode()


def set_tile_rows(rows: int) -> None:
    """Query rows per workgroup for later calls: 0 (chosen from the shape, the
    default), 128 or 256.  Outputs are byte-identical either way; only speed
    changes (``qm_attn_set_tile_rows``)."""
    status = load_library().qm_attn_set_tile_rows(int(rows))
    if status != QM_OK:
        raise QmAttnError(status, strerror(status))


def qm_attn_fwd(q, k, v, o, lse, B, H, N, d, scale, causal, stream, dtype) -> int:
    """The C entry point with plain integers for pointers; returns the status."""
    return load_library().qm_attn_fwd(q, k, v, o, lse, int(B), int(H), int(N), int(d),
                                      float(scale), int(causal), stream, int(dtype))


def qm_attn_fwd_layout(q, k, v, o, lse, B, H, Hkv, N, d_qk, d_v, scale, causal, stream, dtype,
                       layout) -> int:
    """The general 16-bit C entry point (layout argument) with plain integers
    for pointers; returns the status."""
    return load_library().qm_attn_fwd_layout(q, k, v, o, lse, int(B), int(H), int(Hkv), int(N),
                                             int(d_qk), int(d_v), float(scale), int(causal),
                                             stream, int(dtype), int(layout))


def qm_attn_fwd_gqa(q, k, v, o, lse, B, H, Hkv, N, d, scale, causal, stream, dtype) -> int:
    """The grouped-query C entry point with plain integers for pointers; returns the status."""
    return load_library().qm_attn_fwd_gqa(q, k, v, o, lse, int(B), int(H), int(Hkv), int(N),
                                          int(d), float(scale), int(causal), stream, int(dtype))


def qm_attn_fwd_mla(q, k, v, o, lse, B, H, N, d_qk, d_v, scale, causal, stream, dtype) -> int:
    """The unequal-head-dimension C entry point with plain integers for pointers."""
    return load_library().qm_attn_fwd_mla(q, k, v, o, lse, int(B), int(H), int(N), int(d_qk),
                                          int(d_v), float(scale), int(causal), stream, int(dtype))


def qm_attn_fwd_fp8(q, k, v, o, lse, B, H, N, d, q_scale, k_scale, v_scale, scale, causal,
                    stream) -> int:
    """The FP8 C entry point with plain integers for pointers; returns the status."""
    return load_library().qm_attn_fwd_fp8(q, k, v, o, lse, int(B), int(H), int(N), int(d),
                                          float(q_scale), float(k_scale), float(v_scale),
                                          float(scale), int(causal), stream)


def fwd_fp8(q, k, v, scales, causal: bool = False, scale: float | None = None, out=None,
            lse=None, stream=None, layout: str = "bhnd"):
    """FP8 attention forward: q is [B, H, N, d], k and v [B, Hkv, N, d] (Hkv
    dividing H: grouped-query attention when Hkv < H) tensors of OCP E4M3 codes
    (``torch.float8_e4m3fn`` or ``uint8``) on a ROCm device; ``scales`` holds
    the three per-tensor factors (q_scale, k_scale, v_scale).  With
    ``layout="bnhd"`` the tensors are [B, N, heads, d] instead.  Returns
    (o, lse): o bf16 shaped like q, lse float32 [B, H, N] in either layout.
    ``scale`` defaults to 1/sqrt(d) rounded to float32.  Multi-head
    [B, H, N, d] calls go to ``qm_attn_fwd_fp8``, the others to
    ``qm_attn_fwd_fp8_layout``."""
    import torch

    if layout not in ("bhnd", "bnhd"):
        raise ValueError(f"layout must be 'bhnd' or 'bnhd', not {layout!r}")
    bnhd = layout == "bnhd"
    device = q.device
    for t in (q, k, v):
        if t.dim() != 4:
            names = "[B, N, H, d]" if bnhd else "[B, H, N, d]"
            raise ValueError(f"q, k and v must have shape {names}")
        if t.dtype not in (torch.uint8, torch.float8_e4m3fn):
            raise TypeError("FP8 inputs must be float8_e4m3fn or uint8 codes")
        if not t.is_cuda or t.device != device or not t.is_contiguous():
            raise ValueError("q, k and v must be contiguous tensors on one ROCm device")
    if bnhd:
        B, N, H, d = q.shape
        Bk, Nk, Hkv, dk = k.shape
    else:
        B, H, N, d = q.shape
        Bk, Hkv, Nk, dk = k.shape
    if v.shape != k.shape or Bk != B or Nk != N or dk != d:
        raise ValueError("k and v must hold Hkv heads matching q in B, N and d")
    scale = 1.0 / d ** 0.5 if scale is None else float(scale)   # rounded to float32 by the call
    with _pool_of(stream, out is None or lse is None):
        if out is None:
            out = torch.empty(q.shape, dtype=torch.bfloat16, device=device)
        elif out.shape != q.shape or out.dtype != torch.bfloat16 or not out.is_contiguous():
            raise ValueError("out must be a contiguous bfloat16 tensor shaped like q")
        lse = _lse(q, lse, B, H, N)
    _check_outputs_on(device, out, lse)
    qs, ks, vs = (float(t) for t in scales)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), B, H)
    if bnhd or Hkv != H:
        _enqueue(load_library().qm_attn_fwd_fp8_layout, device, stream,
                 args + (Hkv, N, d, qs, ks, vs, scale, 1 if causal else 0),
                 (QM_BNHD if bnhd else QM_BHND,))
    else:
        _enqueue(load_library().qm_attn_fwd_fp8, device, stream,
                 args + (N, d, qs, ks, vs, scale, 1 if causal else 0), ())
    return out, lse


def qm_attn_fwd_fp8_layout(q, k, v, o, lse, B, H, Hkv, N, d, q_scale, k_scale, v_scale, scale,
                           causal, stream, layout) -> int:
    """The general FP8 C entry point (key/value heads and layout as arguments)
    with plain integers for pointers; returns the status."""
    return load_library().qm_attn_fwd_fp8_layout(
        q, k, v, o, lse, int(B), int(H), int(Hkv), int(N), int(d), float(q_scale),
        float(k_scale), float(v_scale), float(scale), int(causal), stream, int(layout))


def _check_outputs_on(device, out, lse) -> None:
    """The kernel writes o and lse through device pointers: both must live on
    the inputs' device (a host tensor's address would be written by the GPU)."""
    for name, t in (("out", out), ("lse", lse)):
        if not t.is_cuda or t.device != device:
            raise ValueError(f"{name} must be on the inputs' device {device}, not {t.device}")


_CURRENT = contextlib.nullcontext()


def _pool_of(stream, new):
    """A context that takes new tensors, where there are any, from the pool of the stream
    that the call runs on.  From the current stream's pool, beside a `stream` of the
    caller's, their memory could still be in use by that stream's earlier work, and be given
    out to its later work while the kernel writes it: nothing orders the two."""
    if stream is None or not new:
        return _CURRENT
    import torch
    return torch.cuda.stream(stream)


def _lse(q, lse, B, H, N):
    """The log-sum-exp output: the caller's, checked, or a new tensor."""
    import torch
    if lse is None:
        return torch.empty(B, H, N, dtype=torch.float32, device=q.device)
    if lse.shape != (B, H, N) or lse.dtype != torch.float32 or not lse.is_contiguous():
        raise ValueError("lse must be a contiguous float32 tensor of shape [B, H, N]")
    return lse


def _enqueue(entry, device, stream, before, after) -> None:
    """Call a C entry point (arguments before and after its stream) with `device`
    current, on `stream` (a torch stream; None: the device's current one)."""
    import torch
    index = device.index
    # the current stream's handle alone, without a torch.cuda.Stream object around it
    if stream is None:
        raw = torch._C._cuda_getCurrentRawStream(index)
    elif stream.device.index == index:
        raw = stream.cuda_stream
    else:
        raise ValueError(f"stream must be one of the inputs' device {device}, not of {stream.device}")
    if index == torch._C._cuda_getDevice():   # (torch.cuda.current_device, without its checks)
        status = entry(*before, raw, *after)
    else:
        with torch.cuda.device(index):
            status = entry(*before, raw, *after)
    if status != QM_OK:
        raise QmAttnError(status, strerror(status))


def _dtype_code(t) -> int:
    import torch
    if t.dtype == torch.float16:
        return QM_F16
    if t.dtype == torch.bfloat16:
        return QM_BF16
    raise TypeError(f"q, k, v must be float16 or bfloat16, not {t.dtype}")


def _checked(q, k, v, scale, out, lse, stream, layout):
    """The checks that the 16-bit calls share.  Returns (the C arguments up to the
    query heads, Hkv, N, d, dv, scale, dtype code, o, lse)."""
    import torch

    if layout not in ("bhnd", "bnhd"):
        raise ValueError(f"layout must be 'bhnd' or 'bnhd', not {layout!r}")
    bnhd = layout == "bnhd"
    if q.dim() != 4:
        raise ValueError(f"q must have shape {'[B, N, H, d]' if bnhd else '[B, H, N, d]'}")
    # a head's rows lie along `rows`, heads along `heads`
    rows, heads = (1, 2) if bnhd else (2, 1)
    qs, ks, vs = q.shape, k.shape, v.shape
    if len(ks) != 4 or len(vs) != 4 or vs[:3] != ks[:3]:
        raise ValueError("k must hold Hkv heads of width d and v Hkv heads of width dv")
    B, H, N, d = qs[0], qs[heads], qs[rows], qs[3]
    Hkv, dv = ks[heads], vs[3]
    if ks[0] != B or ks[rows] != N or ks[3] != d:
        raise ValueError("k must match q in B, N and d")
    if not (q.is_cuda and k.is_cuda and v.is_cuda):
        raise ValueError("q, k and v must be on a ROCm device")
    if not (q.get_device() == k.get_device() == v.get_device()):
        raise ValueError("q, k and v must be on the same device")
    if not (q.dtype == k.dtype == v.dtype):
        raise TypeError("q, k and v must have the same dtype")
    if not (q.is_contiguous() and k.is_contiguous() and v.is_contiguous()):
        names = "[B, N, H, d]" if bnhd else "[B, H, N, d]"
        raise ValueError(f"q, k and v must be contiguous {names}")
    code = _dtype_code(q)
    # the C float argument rounds the scale to float32
    scale = 1.0 / d ** 0.5 if scale is None else float(scale)
    with _pool_of(stream, out is None or lse is None):
        if out is None:
            # (empty_like is a microsecond shorter, but would keep a subclass)
            if dv == d and type(q) is torch.Tensor:
                out = torch.empty_like(q)
            else:
                out = torch.empty((*qs[:3], dv), dtype=q.dtype, device=q.device)
        else:
            oshape = (*qs[:3], dv)
            if tuple(out.shape) != oshape or out.dtype != q.dtype or not out.is_contiguous():
                raise ValueError(f"out must be a contiguous {list(oshape)} tensor of q's dtype")
        lse = _lse(q, lse, B, H, N)
    _check_outputs_on(q.device, out, lse)
    args = (q.data_ptr(), k.data_ptr(), v.data_ptr(), out.data_ptr(), lse.data_ptr(), B, H)
    return args, Hkv, N, d, dv, scale, code, out, lse


def fwd(q, k, v, causal: bool = False, scale: float | None = None, out=None, lse=None,
        stream=None, layout: str = "bhnd"):
    """Attention forward on torch tensors on a ROCm device.

    q is [B, H, N, d]; k is [B, Hkv, N, d] and v [B, Hkv, N, dv] with Hkv
    dividing H.  Hkv = H and dv = d: multi-head attention (``qm_attn_fwd``);
    Hkv < H: grouped-query or multi-query attention (``qm_attn_fwd_gqa``);
    dv < d (d = 192, dv = 128, Hkv = H): the MLA shape (``qm_attn_fwd_mla``).
    With ``layout="bnhd"`` the tensors are [B, N, heads, width] instead (q
    [B, N, H, d], k [B, N, Hkv, d], v [B, N, Hkv, dv], o [B, N, H, dv];
    ``qm_attn_fwd_layout``).  Returns (o, lse): o of q's dtype, lse float32
    [B, H, N] in either layout.  ``scale`` defaults to 1/sqrt(d) rounded to
    float32.  ``stream`` defaults to the current stream of q's device.  Outputs that
    the call makes are tensors of the stream it runs on: work of another stream waits
    for it before it reads them, and, as for any tensor of another stream, the inputs and
    outputs live until the streams that use them are done (``Tensor.record_stream``).
    """
    args, Hkv, N, d, dv, scale, code, out, lse = _checked(q, k, v, scale, out, lse, stream, layout)
    lib, device = load_library(), q.device
    causal = 1 if causal else 0
    if layout == "bnhd":
        _enqueue(lib.qm_attn_fwd_layout, device, stream, args + (Hkv, N, d, dv, scale, causal),
                 (code, QM_BNHD))
    elif dv != d:
        if Hkv != args[6]:
            raise ValueError("unequal head dimensions need as many key/value heads as query heads")
        _enqueue(lib.qm_attn_fwd_mla, device, stream, args + (N, d, dv, scale, causal), (code,))
    elif Hkv == args[6]:
        _enqueue(lib.qm_attn_fwd, device, stream, args + (N, d, scale, causal), (code,))
    else:
        _enqueue(lib.qm_attn_fwd_gqa, device, stream, args + (Hkv, N, d, scale, causal), (code,))
    return out, lse


def fwd_window(q, k, v, window: int, sinks: int = 0, scale: float | None = None, out=None,
               lse=None, stream=None, layout: str = "bhnd"):
    """Causal attention forward with a sliding window: query i sees key j iff j <= i
    and (i - j < ``window`` or j < ``sinks``), the first ``sinks`` keys staying
    visible to every later query.  ``window`` counts the query's own key (at least
    1); a window that reaches every key gives exactly ``fwd(causal=True)``.
    Tensors, types, the other arguments and the results are those of :func:`fwd`
    (``qm_attn_fwd_window``; key blocks that no query sees cost nothing).  As there,
    every row must be finite, those that pad a batch of prompts among them: a hidden
    key has probability 0, but 0 times a NaN value is NaN."""
    args, Hkv, N, d, dv, scale, code, out, lse = _checked(q, k, v, scale, out, lse, stream, layout)
    _enqueue(load_library().qm_attn_fwd_window, q.device, stream,
             args + (Hkv, N, d, dv, scale, _int32(window, "window"), _int32(sinks, "sinks")),
             (code, QM_BNHD if layout == "bnhd" else QM_BHND))
    return out, lse


def _int32(x, name: str) -> int:
    """x as a C int: a value past its range would wrap unseen (a window of 2^32 + 1
    would be 1)."""
    x = operator.index(x)
    if not -2 ** 31 <= x < 2 ** 31:
        raise ValueError(f"{name} must fit 32 bits, not {x}")
    return x


def qm_attn_fwd_window(q, k, v, o, lse, B, H, Hkv, N, d_qk, d_v, scale, window, sinks, stream,
                       dtype, layout) -> int:
    """The sliding-window C entry point with plain integers for pointers; returns
    the status."""
    return load_library().qm_attn_fwd_window(q, k, v, o, lse, int(B), int(H), int(Hkv), int(N),
                                             int(d_qk), int(d_v), float(scale), int(window),
                                             int(sinks), stream, int(dtype), int(layout))
