"""The serving operators in 64 bits, from their definitions, and bounds on how far a
correct kernel may be from them (test infrastructure only; torch on whatever device the
inputs are on).

Bounds.  A value rounded to a type is off by at most half a step: ``HALF[t]`` times
itself (bf16 2^-8, f16 2^-11, E4M3 2^-4), or half a subnormal step (f16 2^-25, E4M3
2^-10).  fp32 arithmetic adds 2^-24 of each intermediate.

* norm and rotation: one rounding of the result, and fp32 errors of the products that
  make it: the mean of d squares, root, quotient and weight (relative, below
  (d / 8 + 16) 2^-24 with the lanes' sums of 16 squares) and the two products and the
  sum of the rotation, all below 2^-18 (|a| + |b|) for the pair (a, b).
* attention, o_i = sum_j p_ij v_j with p = e^(s - lse): weights rounded to the 16-bit
  type (HALF of each), scores formed in fp32 (a sum of d products is off by at most
  d 2^-24 sum_c |q_c k_c|; times the scale, the weight by that, the normaliser by as
  much again), exponentials and sums of fp32 (below 2^-18): together
  (HALF + 2 D + 2^-18) sum_j p_ij |v_j|, with D the largest score error of the row; f16
  weights below 2^-14 of the row's largest are off by 2^-25 of it; and the rounding of o.
* lse: D, and fp32 rounding of the maximum and the logarithm, 2^-21 (1 + |lse| + |max|).
"""
from __future__ import annotations

import math

import torch

HALF = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11, torch.float8_e4m3fn: 2.0 ** -4}
STEP = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25, torch.float8_e4m3fn: 2.0 ** -10}


def rotation_table(positions, rotary, base=10000.0, device="cuda"):
    half = rotary // 2
    rate = base ** (-torch.arange(half, dtype=torch.float64) / max(half, 1))
    phase = torch.arange(positions, dtype=torch.float64)[:, None] * rate
    return phase.cos().float().to(device), phase.sin().float().to(device)


def norm_rope(x, weight, cos, sin, positions, eps, interleaved):
    """x [B, N, heads, d] (any strides) in 64 bits, positions [B, N]; returns (y, bound
    on fp32 errors).  Rows of positions outside the table are NaN."""
    y = x.double()
    if weight is not None:
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + eps) * weight.double()
    out, size = y.clone(), y.abs()
    if cos is not None and cos.shape[1]:
        half = cos.shape[1]
        inside = (positions >= 0) & (positions < cos.shape[0])
        at = positions.clamp(0, cos.shape[0] - 1).long()
        c, s = (t.double()[at][:, :, None] for t in (cos, sin))
        first = slice(0, 2 * half, 2) if interleaved else slice(0, half)
        second = slice(1, 2 * half, 2) if interleaved else slice(half, 2 * half)
        a, b = y[..., first], y[..., second]
        out[..., first], out[..., second] = a * c - b * s, b * c + a * s
        size = size.clone()
        size[..., first] = size[..., second] = a.abs() + b.abs()
        out[~inside] = math.nan
    return out, 2.0 ** -18 * size


def check_rounded(got, want, slack, what=""):
    """got = want rounded to its type, up to `slack` before the rounding; NaNs alike."""
    g, t = got.double(), got.dtype
    assert torch.equal(torch.isnan(g), torch.isnan(want)), f"{what}: NaNs differ"
    bound = HALF[t] * (want.abs() + slack) + STEP[t] + slack
    over = (g - want).abs() - bound
    over = torch.where(torch.isnan(want), -1.0, over)
    assert over.numel() == 0 or over.max() <= 0, (
        f"{what}: off by {float((g - want).abs().flatten()[over.argmax()]):.3e}, bound "
        f"{float(bound.flatten()[over.argmax()]):.3e} at {int(over.argmax())}")


def attention_row_bounds(q, k, v, scale, seen, dtype):
    """One head in 64 bits: q [R, d], k [K, d], v [K, dv], seen [R, K].  Returns (o, lse,
    bound of o, bound of lse); rows that see nothing give o = 0 and lse = -inf."""
    q, k, v = q.double(), k.double(), v.double()
    s = (q @ k.T) * scale
    s = torch.where(seen, s, -math.inf)
    lse = torch.logsumexp(s, dim=1) if k.shape[0] else torch.full(q.shape[:1], -math.inf, dtype=q.dtype, device=q.device)
    p = torch.exp(s - torch.where(torch.isinf(lse), 0.0, lse)[:, None])
    v = torch.where(seen.any(0)[:, None], v, 0.0)
    o = p @ v
    D = (q.abs() @ k.abs().T) * abs(scale) * q.shape[1] * 2.0 ** -24
    D = torch.where(seen, D, 0.0).amax(1, keepdim=True) if k.shape[0] else torch.zeros_like(o[:, :1])
    top = torch.where(torch.isinf(lse), 0.0, s.amax(1)) if k.shape[0] else torch.zeros_like(lse)
    largest = torch.exp(top - torch.where(torch.isinf(lse), 0.0, lse))   # the row's largest weight
    o_bound = ((HALF[dtype] + 2 * D + 2.0 ** -18) * (p @ v.abs())
               + STEP[dtype] * largest[:, None] * (seen.double() @ v.abs()))
    o_bound = o_bound + HALF[dtype] * (o.abs() + o_bound) + STEP[dtype]
    lse_bound = D[:, 0] + 2.0 ** -21 * (1 + torch.where(torch.isinf(lse), 0.0, lse.abs()) + top.abs())
    return o, lse, o_bound, lse_bound


def check_attention(o, lse, want, what=""):
    ow, lw, ob, lb = want
    assert torch.isfinite(o).all(), f"{what}: o is not finite"
    over = (o.double() - ow).abs() - ob
    assert over.max() <= 0, f"{what}: o over its bound by {float(over.max()):.3e} at {int(over.argmax())}"
    hidden = torch.isinf(lw)
    assert torch.equal(torch.isinf(lse), hidden), f"{what}: lse of empty rows"
    assert (lse[hidden] < 0).all()
    over = torch.where(hidden, -1.0, (lse.double() - lw).abs() - lb)
    assert over.max() <= 0, f"{what}: lse over its bound by {float(over.max()):.3e}"


def tokens_of(cache, table_row, n, layout):
    """The first n tokens of one sequence, [n, Hkv, d] in 64 bits, from a paged cache."""
    t = cache.float() if cache.dtype != torch.uint8 else cache.view(torch.float8_e4m3fn).float()
    t = t if layout == "bnhd" else t.transpose(1, 2)
    page = t.shape[1]
    pages = table_row[:(n + page - 1) // page].long()
    return t[pages].flatten(0, 1)[:n].double()


def decode(q, k_cache, v_cache, table, lengths, scale, window, sinks, k_scale, v_scale, layout):
    """Yields (b, heads of one key/value head, the bounds of attention_row_bounds)."""
    B, H, _ = q.shape
    for b, n in enumerate(lengths):
        k = tokens_of(k_cache, table[b], n, layout) * k_scale
        v = tokens_of(v_cache, table[b], n, layout) * v_scale
        j = torch.arange(n, device=q.device)
        seen = torch.ones(n, dtype=torch.bool, device=q.device)
        if window:
            seen = (j >= n - window) | (j < sinks)
        k, v = (torch.where(seen[:, None, None], t, 0.0) for t in (k, v))
        G = H // k.shape[1]
        for g in range(k.shape[1]):
            heads = slice(g * G, (g + 1) * G)
            yield b, heads, attention_row_bounds(q[b, heads], k[:, g], v[:, g], scale,
                                                 seen.expand(G, n), q.dtype)


def window_mask(N, window, sinks, device="cuda"):
    i, j = torch.arange(N, device=device)[:, None], torch.arange(N, device=device)
    return (j <= i) & ((i - j < window) | (j < sinks))
