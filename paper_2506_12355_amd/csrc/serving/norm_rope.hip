// Head norms and the position rotation in one pass over q and k, and, where a paged
// cache is given, the keys and values written into its pages.
//
//   y_c = x_c w_c / sqrt(mean_c x_c^2 + eps)                      (per head, d columns)
//   (a, b) -> (a cos - b sin, b cos + a sin)     (first `rotary` columns, in pairs)
//
// in fp32 from the stored values to one rounding into the result's type.
//
// Bound: memory; every element is read and written once, 1-2 flops per byte.  A head's
// row belongs to d / 16 lanes, each with two 16-byte pieces: columns 8 i .. + 7 of each
// half of the rotated part (the pairs of the half-split rotation), or 16 consecutive
// columns (the pairs of the interleaved one, and columns that are not rotated).  Every
// pair then lies in one lane, whose angles are 8 consecutive table entries either way,
// and the only exchange is the norm's sum over d / 16 lanes.  A wavefront takes 64 /
// (d / 16) rows, in the order of the output, so consecutive rows are read and written as
// one stream; several rows in turn, angles and weights kept, were slower (two and four
// rows a lane, below).
//
// Measured (us, bf16, d = 128, over more inputs than the last-level cache holds; a plain copy runs
// at 5.1 TB/s): 72 heads of 8192 tokens 55-58 (5.2-5.5 TB/s; two and four rows a lane 4% and 8%
// more), head-major 61; one token 2.9 (two and four rows a lane 0.7 and 2.7 more); 4 ragged
// prompts of up to 2000 tokens into E4M3 pages 30-31 (4.7-4.9 TB/s), into bf16 ones 31.6 (5.0).
#include "serving_device.h"
#include "serving_launch.h"

namespace qm {
namespace {

// One of q, k and v, as a unit of rows sees it.
struct Stream {
  const uint16_t* x;
  uint16_t* out;          // NULL: not written (keys and values kept in the cache only)
  uint8_t* cache;         // NULL: not cached
  const uint16_t* weight;
  int64_t sb, sn, sh;     // input strides, elements
  FastDiv inner, outer;   // of a row index, in the order of the output
  uint32_t rows, units;
  float inv;              // cached values are multiplied by this
};

struct Params {
  Stream s[3];
  const float *cos, *sin;
  const int32_t *starts, *counts;
  const int32_t* table;
  int64_t page_stride;
  int token_stride, head_stride, num_pages, table_cols, fp8;
  FastDiv page;
  int rotary, table_rows, interleaved, bnhd;
  float eps;
};

// With positions of several axes.  (A struct of its own: calls of one axis, which are short,
// take no arguments that they do not read.)
struct AxesParams : Params {
  const int32_t* positions;
  int64_t axis_stride;
  int B, N, used_axes;
  uint64_t pair_axis[2];
  FastDiv blocks[3], head_blocks[3];   // of a unit's index in q, k and v, where a lane has several heads
};
template <bool AXES>
using ParamsOf = std::conditional_t<AXES, AxesParams, Params>;

// Sum over the L (4 or 8) neighbouring lanes that hold a row.
template <int L>
__device__ __forceinline__ float row_sum(float x) {
  auto add = [](float v, auto ctrl) {
    return v + __builtin_bit_cast(float, __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v),
                                                                   decltype(ctrl)::value, 0xf, 0xf, true));
  };
  x = add(x, std::integral_constant<int, 0xB1>{});             // quad_perm [1, 0, 3, 2]
  x = add(x, std::integral_constant<int, 0x4E>{});             // quad_perm [2, 3, 0, 1]
  if (L == 8) x = add(x, std::integral_constant<int, 0x141>{});   // row_half_mirror
  return x;
}

// The rows of one unit of q (KIND 0), k (1) or v (2).
template <int DT, int D, bool AXES, int HEADS, int KIND>
__device__ __forceinline__ void unit_rows(const ParamsOf<AXES>& p, const Stream& s, uint32_t unit) {
  using T = Type16<DT>;
  constexpr int L = D / 16;      // lanes of a row
  constexpr int R = 64 / L;      // rows of a wavefront at once
  const int lane = threadIdx.x & 63, i = lane % L;

  // this lane's two pieces of a row, and whether their columns are rotated
  const int half = p.rotary / 2;
  const bool turned = KIND < 2 && i < p.rotary / 16;
  const bool split = turned && !p.interleaved;
  const int c0 = split ? 8 * i : 16 * i, c1 = split ? half + 8 * i : 16 * i + 8;

  u32x4 w0, w1;
  const bool normed = KIND < 2 && s.weight;
  if (normed) {
    w0 = *reinterpret_cast<const u32x4*>(s.weight + c0);
    w1 = *reinterpret_cast<const u32x4*>(s.weight + c1);
  }

  uint32_t row = unit * R + lane / L, b, h, t;
  const uint32_t heads = p.bnhd ? s.inner.d : s.outer.d;
  if constexpr (HEADS > 1) {
    const FastDiv &blocks = p.blocks[KIND], &head_blocks = p.head_blocks[KIND];
    // a lane's rows: of one token, HEADS heads, R apart (a wavefront has R * HEADS of a token) or
    // neighbours (it has those of R tokens)
    const uint32_t token = p.bnhd ? blocks.div(unit) : 0, block = p.bnhd ? unit - token * blocks.d : blocks.div(unit);
    if (p.bnhd) {
      b = s.outer.div(token);
      t = token - b * s.outer.d;
      h = block * (R * HEADS) + lane / L;
    } else {   // blocks of R tokens the inner index, blocks of HEADS heads the next
      t = (unit - block * blocks.d) * R + lane / L;
      b = head_blocks.div(block);
      h = (block - b * head_blocks.d) * HEADS;
    }
    if (b >= (uint32_t)p.B || h >= heads || t >= (uint32_t)p.N) return;
  } else if (row >= s.rows) {
    return;
  } else if (p.bnhd) {
    const uint32_t token = s.inner.div(row);
    h = row - token * s.inner.d;
    b = s.outer.div(token);
    t = token - b * s.outer.d;
  } else {
    const uint32_t bh = s.inner.div(row);
    t = row - bh * s.inner.d;
    b = s.outer.div(bh);
    h = bh - b * s.outer.d;
  }
  const int64_t at = (int64_t)(p.starts ? p.starts[b] : 0) + t;
  const bool held = !p.counts || (int)t < p.counts[b];
  bool fits = !p.rotary || (at >= 0 && at < p.table_rows);
  int row0 = 0, row1 = 0, row2 = 0, row3 = 0;   // the token's row of the table on each axis
  if constexpr (AXES) if (held) {
    const int32_t* own = p.positions + (int64_t)b * p.N + t;
    if (p.used_axes & 1) row0 = own[0];
    if (p.used_axes & 2) row1 = own[p.axis_stride];
    if (p.used_axes & 4) row2 = own[2 * p.axis_stride];
    if (p.used_axes & 8) row3 = own[3 * p.axis_stride];
    auto inside = [&](int r) __attribute__((always_inline)) { return (uint32_t)r < (uint32_t)p.table_rows; };
    fits = inside(row0) && inside(row1) && inside(row2) && inside(row3);
  }

  f32x4 cv[2], sv[2];   // of this lane's pairs
  auto load_angles = [&]() __attribute__((always_inline)) {
    int64_t line = at;
    bool one = true;   // the lane's pairs lie in one row of the table
    if constexpr (AXES) {
      // the axes of pairs 8 i .. 8 i + 7
      const uint32_t of = (uint32_t)(p.pair_axis[i >= 4] >> (16 * (i & 3))) & 0xffffu;
      auto row_of = [&](uint32_t a) __attribute__((always_inline)) {
        const int low = a & 1 ? row1 : row0, high = a & 1 ? row3 : row2;
        return a & 2 ? high : low;
      };
      line = row_of(of & 3);
      one = of == (of & 3) * 0x5555u;
      if (!one) {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int64_t from = (int64_t)row_of(of >> (2 * j) & 3) * half + 8 * i + j;
          cv[j / 4][j % 4] = p.cos[from];
          sv[j / 4][j % 4] = p.sin[from];
        }
      }
    }
    if (one) {
      const float* ct = p.cos + line * half + 8 * i;
      const float* st = p.sin + line * half + 8 * i;
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        cv[j] = reinterpret_cast<const f32x4*>(ct)[j];
        sv[j] = reinterpret_cast<const f32x4*>(st)[j];
      }
    }
  };
  auto one_row = [&](uint32_t row, uint32_t h) __attribute__((always_inline)) {
    float x[8], y[8];
    if (held) {
      const uint16_t* src = s.x + (int64_t)b * s.sb + (int64_t)t * s.sn + (int64_t)h * s.sh;
      const u32x4 r0 = *reinterpret_cast<const u32x4*>(src + c0);
      const u32x4 r1 = *reinterpret_cast<const u32x4*>(src + c1);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const f32x2 e0 = T::unpack(r0[j]), e1 = T::unpack(r1[j]);
        x[2 * j] = e0[0], x[2 * j + 1] = e0[1];
        y[2 * j] = e1[0], y[2 * j + 1] = e1[1];
      }
      if (normed) {
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 8; ++j) sum = fmaf(x[j], x[j], fmaf(y[j], y[j], sum));
        const float r = 1.0f / sqrtf(row_sum<L>(sum) * (1.0f / D) + p.eps);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const f32x2 e0 = T::unpack(w0[j]), e1 = T::unpack(w1[j]);
          x[2 * j] *= r * e0[0], x[2 * j + 1] *= r * e0[1];
          y[2 * j] *= r * e1[0], y[2 * j + 1] *= r * e1[1];
        }
      }
      if (turned && fits) {
        if (HEADS == 1) load_angles();
        // Which product is rounded before the sum is said here, not left to the compiler, so that
        // every instance gives the same bytes.  (In interleaved pairs 4 to 6 of a lane the other one
        // is, in b cos + a sin: the bytes that calls of one axis gave while it was left.)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float cj = cv[j / 4][j % 4], sj = sv[j / 4][j % 4];
          if (p.interleaved) {
            float* z = j < 4 ? x : y;
            const int e = 2 * (j % 4);
            const float a0 = z[e], b0 = z[e + 1];
            z[e] = fmaf(a0, cj, -(b0 * sj));
            z[e + 1] = j < 4 || j == 7 ? fmaf(b0, cj, a0 * sj) : fmaf(a0, sj, b0 * cj);
          } else {
            const float a0 = x[j], b0 = y[j];
            x[j] = fmaf(a0, cj, -(b0 * sj));
            y[j] = fmaf(b0, cj, a0 * sj);
          }
        }
      }
    }
    if (!held || (!fits && KIND < 2)) {
      // no token, or one that the table has no angle for
      const float fill = held ? __builtin_nanf("") : 0.f;
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = y[j] = fill;
    }
    if (KIND == 0 || (KIND == 1 && s.out)) {
      uint16_t* dst = s.out + (size_t)row * D;
      u32x4 o0, o1;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        o0[j] = T::pack(x[2 * j], x[2 * j + 1]);
        o1[j] = T::pack(y[2 * j], y[2 * j + 1]);
      }
      *reinterpret_cast<u32x4*>(dst + c0) = o0;
      *reinterpret_cast<u32x4*>(dst + c1) = o1;
    }
    if (KIND > 0 && s.cache && held && fits && at >= 0 && at < (int64_t)p.table_cols * p.page.d) {
      const uint32_t n = p.page.div((uint32_t)at);
      const int page = p.table[(size_t)b * p.table_cols + n];
      if (page >= 0 && page < p.num_pages) {
        uint8_t* dst = s.cache + (int64_t)page * p.page_stride +
                       (int64_t)((uint32_t)at - n * p.page.d) * p.token_stride + (int64_t)h * p.head_stride;
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] *= s.inv, y[j] *= s.inv;
        if (p.fp8) {
          *reinterpret_cast<u32x2*>(dst + c0) = u32x2{pack_fp8(x[0], x[1], x[2], x[3]),
                                                      pack_fp8(x[4], x[5], x[6], x[7])};
          *reinterpret_cast<u32x2*>(dst + c1) = u32x2{pack_fp8(y[0], y[1], y[2], y[3]),
                                                      pack_fp8(y[4], y[5], y[6], y[7])};
        } else {
          u32x4 o0, o1;
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            o0[j] = T::pack(x[2 * j], x[2 * j + 1]);
            o1[j] = T::pack(y[2 * j], y[2 * j + 1]);
          }
          *reinterpret_cast<u32x4*>(dst + 2 * c0) = o0;
          *reinterpret_cast<u32x4*>(dst + 2 * c1) = o1;
        }
      }
    }
  };
  if constexpr (HEADS == 1) {
    one_row(row, h);
  } else {
    if (held && turned && fits) load_angles();
    for (int r = 0; r < HEADS; ++r) {
      const uint32_t of = h + (p.bnhd ? R : 1) * r;
      if (of < heads) one_row(p.bnhd ? ((uint32_t)b * p.N + t) * heads + of : (b * heads + of) * p.N + t, of);
    }
  }
}

template <int DT, int D, bool AXES, int HEADS>
__global__ __launch_bounds__(256) void norm_rope_kernel(ParamsOf<AXES> p) {
  uint32_t unit = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (unit < p.s[0].units) return unit_rows<DT, D, AXES, HEADS, 0>(p, p.s[0], unit);
  unit -= p.s[0].units;
  if (unit < p.s[1].units) return unit_rows<DT, D, AXES, HEADS, 1>(p, p.s[1], unit);
  unit -= p.s[1].units;
  if (unit < p.s[2].units) unit_rows<DT, D, AXES, HEADS, 2>(p, p.s[2], unit);
}

// With positions of several axes a lane takes four heads of its token in large calls, so that the
// angles, which lie in up to eight places of the table for its eight pairs, are fetched once
// for them (us, one, two, four and eight heads, over more inputs than the last-level cache holds;
// axes in turn over the pairs: 4 prompts of up to 1999 tokens into E4M3 pages 59.5, 45.8, 39.9,
// 40.9, 72 heads of 8192 tokens 96.5, 68.7, 63.8, 62.3; a run of pairs each: 35.1, 33.5, 31.3, 31.8
// and 61.6, 57.6, 58.3, 57.7).  Large: of 4096 wavefronts on (us, 32/8 heads, one and four heads a
// lane, axes in turn, token-major, and in runs: 400 tokens, 2000 wavefronts, 7.0, 9.4 and 5.6, 8.7;
// 800 9.9, 10.5 and 7.1, 9.4; 1600 15.8, 12.6 and 10.7, 10.4; 3200 27.6, 21.1 and 17.9, 16.2).
constexpr int kHeads = 4;

template <int DT, int D>
hipError_t launch(const NormRopeArgs& a, hipStream_t stream) {
  constexpr int kRows = 64 / (D / 16);   // rows of a wavefront
  AxesParams p = {};
  const uint16_t* in[3] = {a.q, a.k, a.v};
  uint16_t* out[3] = {a.q_out, a.k_out, nullptr};
  uint32_t units = 0;
  for (int i = 0; i < 3; ++i) {
    Stream& s = p.s[i];
    if (!in[i]) continue;
    s.x = in[i];
    s.out = out[i];
    s.cache = static_cast<uint8_t*>(i == 0 ? nullptr : i == 1 ? a.cache.k : a.cache.v);
    s.weight = i == 0 ? a.q_weight : i == 1 ? a.k_weight : nullptr;
    s.sb = a.stride[i][0], s.sn = a.stride[i][1], s.sh = a.stride[i][2];
    const int heads = i == 0 ? a.H : a.Hkv;
    s.inner = FastDiv(a.layout ? heads : a.N);
    s.outer = FastDiv(a.layout ? a.N : heads);
    s.rows = (uint32_t)((int64_t)a.B * a.N * heads);
    s.units = (s.rows + kRows - 1) / kRows;
    s.inv = i == 1 ? a.k_inv : a.v_inv;
    units += s.units;
  }
  p.cos = a.cos, p.sin = a.sin;
  p.starts = a.starts, p.counts = a.counts;
  p.table = a.cache.table;
  p.page_stride = a.cache.page_stride;
  p.token_stride = a.cache.token_stride, p.head_stride = a.cache.head_stride;
  p.num_pages = a.cache.num_pages, p.table_cols = a.cache.table_cols, p.fp8 = a.cache.fp8;
  p.page = FastDiv(a.cache.k ? a.cache.page_size : 1);
  p.rotary = a.rotary, p.table_rows = a.table_rows;
  p.interleaved = a.interleaved, p.bnhd = a.layout, p.eps = a.eps;
  if (a.positions) {
    p.positions = a.positions;
    p.axis_stride = (int64_t)a.B * a.N;
    p.B = a.B, p.N = a.N, p.used_axes = a.used_axes;
    p.pair_axis[0] = a.pair_axis[0], p.pair_axis[1] = a.pair_axis[1];
    // (blocks of rows of one token, or of one head, that would not fill a wavefront, and
    // launches of few wavefronts, keep one row a lane: see kHeads)
    const bool blocks = a.layout ? a.Hkv >= kRows && a.H >= kRows : a.N >= kRows;
    if (blocks && units >= 1024u * kHeads) {
      units = 0;
      for (int i = 0; i < 3; ++i) {
        Stream& s = p.s[i];
        if (!in[i]) continue;
        const int heads = i == 0 ? a.H : a.Hkv;
        const uint32_t token_blocks = (a.N + kRows - 1) / kRows, per = a.layout ? kRows * kHeads : kHeads;
        const uint32_t head_blocks = (heads + per - 1) / per;
        p.blocks[i] = FastDiv(a.layout ? head_blocks : token_blocks);
        p.head_blocks[i] = FastDiv(head_blocks);
        s.units = (uint32_t)((int64_t)a.B * head_blocks * (a.layout ? a.N : token_blocks));
        units += s.units;
      }
      hipLaunchKernelGGL((norm_rope_kernel<DT, D, true, kHeads>), dim3((units + 3) / 4), dim3(256), 0, stream, p);
      return hipGetLastError();
    }
    hipLaunchKernelGGL((norm_rope_kernel<DT, D, true, 1>), dim3((units + 3) / 4), dim3(256), 0, stream, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((norm_rope_kernel<DT, D, false, 1>), dim3((units + 3) / 4), dim3(256), 0, stream,
                     static_cast<const Params&>(p));
  return hipGetLastError();
}

template <int DT>
hipError_t launch_width(const NormRopeArgs& a, hipStream_t stream) {
  return a.d == 64 ? launch<DT, 64>(a, stream) : launch<DT, 128>(a, stream);
}

}  // namespace

hipError_t launch_norm_rope(const NormRopeArgs& a, hipStream_t stream) {
  return a.dtype == 0 ? launch_width<0>(a, stream) : launch_width<1>(a, stream);
}

}  // namespace qm
