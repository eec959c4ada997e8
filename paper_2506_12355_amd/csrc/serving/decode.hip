// Attention of one new token per sequence over a paged cache of keys and values.
//
// Bound: HBM.  Every visible key and value is read once, by one wavefront, for all
// query heads that share it (up to 16; more take further workgroups), straight from
// its page into matrix operands: there is no staging and no reuse to stage for.
//
// A wavefront walks 32-token blocks (two 16-token tiles, which a page, a multiple of
// 16 tokens, never splits):
//
//   S^T[key][head] = K Q^T   A operand: K rows as stored (lane l: row l % 16 of a tile,
//       16 bytes of columns 32 c + 8 (l / 16) ..), B operand: Q, resident.  Each lane
//       ends with one head, l % 16, and keys 4 (l / 16) .. + 3 of both tiles.
//   O^T[column][head] += V^T P^T   B operand: P^T as it lies, 8 keys of the lane's head.
//       A operand: the same 8 keys of V, for column l % 16 of each M tile.  Columns are
//       dealt so that a lane reads d / 16 consecutive ones of each of its 8 rows (16
//       lanes read a whole row) and M tile t takes the t-th of them; operands are then
//       pairs of rows' halves, one byte permute per register.
//
// The order of the contraction and of the M tiles is free, so neither K, V nor P moves
// between lanes.  E4M3 codes are widened to the query's type on the way (exact) and
// take the same path.  Scores, maxima and sums are in fp32, base 2 (c = scale log2 e);
// P is rounded to the query's 16-bit type for the second product, as the package's
// other attention kernels round it: the row sum keeps the unrounded values.
//
// Split: a workgroup's wavefronts take the blocks of a chunk in turn and join their
// (m, l, O) in LDS; where a sequence has several chunks, each workgroup writes its
// unnormalised O, m and l to the workspace and a second kernel joins them in order, so
// results do not depend on which finished first.  Chunks past a sequence's end cost an
// early exit.  Keys that are hidden (past the length, or before the window and past the
// first keys) get the score -inf and a zero V row: what their memory holds, NaN
// included, does not reach the result.
//
// Window: the blocks walked are those with first keys, then those from the window on;
// list index i is block i, or i + skip past the first keys' blocks.
#include <float.h>

#include "serving_device.h"
#include "serving_launch.h"

namespace qm {
namespace {

constexpr int kBlock = 32;   // tokens of a wavefront's step

struct Params {
  const uint16_t* q;
  uint16_t* o;
  float* lse;
  const int32_t* lengths;
  const uint8_t *k, *v;
  const int32_t* table;
  float* part_o;     // [B H][splits][d]
  float* part_ml;    // [B H][splits][2]
  int64_t page_stride;
  uint32_t token_stride, head_stride;
  int num_pages, table_cols;
  FastDiv page;
  int H, Hkv, group, tiles;   // query heads per key/value head, and 16-head tiles of them
  int splits, chunk;          // chunk: blocks of a workgroup
  int limit, window, sinks;
  float c, v_scale;
};

// The blocks of one sequence that hold visible tokens.
struct Blocks {
  int total, nsink, skip;
  __device__ __forceinline__ Blocks(const Params& p, int len) {
    total = (len + kBlock - 1) / kBlock;
    nsink = skip = 0;
    if (p.window > 0 && len > p.window) {
      const int first = (len - p.window) / kBlock;
      nsink = min(first, (min(p.sinks, len) + kBlock - 1) / kBlock);
      skip = first - nsink;
      total -= skip;
    }
  }
  __device__ __forceinline__ int token(int i) const { return (i < nsink ? i : i + skip) * kBlock; }
};

__device__ __forceinline__ float max_over_groups(float x) {
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_over_groups(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// Eight E4M3 codes as 16-bit values (exact in either type).
template <int DT>
__device__ __forceinline__ u32x4 widen(uint32_t lo, uint32_t hi) {
  u32x4 w;
  if constexpr (DT == 0) {
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, false));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(lo, 1.f, true));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, false));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(hi, 1.f, true));
  } else {
    w[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, false));
    w[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.f, true));
    w[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, false));
    w[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.f, true));
  }
  return w;
}

template <int BYTES>
struct Raw;
template <>
struct Raw<16> { using T = u32x4; };
template <>
struct Raw<8> { using T = u32x2; };
template <>
struct Raw<4> { using T = uint32_t; };

template <int DT, int D, bool FP8, int WAVES>
__global__ __launch_bounds__(64 * WAVES, (WAVES > 4 ? 1 : 2)) void decode_kernel(Params p) {
  using T = Type16<DT>;
  constexpr int ES = FP8 ? 1 : 2;
  constexpr int NC = D / 32;            // k-steps of the first product
  constexpr int NK = D * ES / 64;       // 16-byte K loads of a lane and tile
  constexpr int CV = D / 16;            // V columns of a lane, and M tiles
  using VRaw = typename Raw<CV * ES>::T;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);

  // workgroup: (sequence, key/value head, 16-head tile, chunk), chunks innermost
  int id = blockIdx.x;
  const int split = id % p.splits;
  id /= p.splits;
  const int tile = id % p.tiles;
  id /= p.tiles;
  const int hkv = id % p.Hkv, b = id / p.Hkv;

  const int len0 = p.lengths[b];
  const bool bad_len = len0 < 0 || len0 > p.limit;
  const int len = bad_len ? 0 : len0;
  const Blocks blocks(p, len);
  const int first = split * p.chunk;
  if (first >= blocks.total && split > 0) return;
  const int last = min(first + p.chunk, blocks.total);   // list indexes first .. last - 1
  const int lo_window = p.window > 0 ? len - p.window : 0;   // tokens from here on are visible

  // heads of this tile
  const int heads = min(16, p.group - 16 * tile);
  const int head0 = hkv * p.group + 16 * tile;
  u32x4 qf[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) qf[c] = u32x4{};
  if (n < heads) {
    const uint16_t* q = p.q + ((size_t)b * p.H + head0 + n) * D;
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      const int col = FP8 ? (c / 2) * 64 + g * 16 + (c % 2) * 8 : c * 32 + g * 8;
      qf[c] = *reinterpret_cast<const u32x4*>(q + col);
    }
  }

  const uint8_t* kh = p.k + (size_t)hkv * p.head_stride;
  const uint8_t* vh = p.v + (size_t)hkv * p.head_stride;
  const uint32_t k_lane = n * p.token_stride + g * 16;
  const uint32_t v_lane = 4 * g * p.token_stride + n * (CV * ES);

  // Offsets of the tiles of the wavefront's next 32 blocks: lane 2 i + t holds tile t of
  // the i-th.  A tile past the length borrows the first tile's (its keys are hidden).
  int off_lo = 0, off_hi = 0;
  bool bad = bad_len;
  auto look_up = [&](int i0) __attribute__((always_inline)) {
    const int li = i0 + WAVES * (lane >> 1);
    int64_t off = 0;
    if (li < last) {
      int token = blocks.token(li) + 16 * (lane & 1);
      if (token >= len) token -= 16;
      const uint32_t at = p.page.div((uint32_t)token);
      const int page = p.table[(size_t)b * p.table_cols + at];
      if (page >= 0 && page < p.num_pages)
        off = page * p.page_stride + (int64_t)((uint32_t)token - at * p.page.d) * p.token_stride;
      else
        bad = true;
    }
    off_lo = (int)(uint32_t)off;
    off_hi = (int)(off >> 32);
  };
  auto tile_off = [&](int i, int t) __attribute__((always_inline)) {
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_hi, 2 * i + t) << 32 |
                     (uint32_t)__builtin_amdgcn_readlane(off_lo, 2 * i + t));
  };

  u32x4 kr[2][NK];
  VRaw vr[8];
  auto load_k = [&](int64_t o0, int64_t o1) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < NK; ++c) {
      kr[0][c] = *reinterpret_cast<const u32x4*>(kh + o0 + (k_lane + 64 * c));
      kr[1][c] = *reinterpret_cast<const u32x4*>(kh + o1 + (k_lane + 64 * c));
    }
  };
  auto load_v = [&](int64_t o0, int64_t o1) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      vr[r] = *reinterpret_cast<const VRaw*>(vh + o0 + (v_lane + r * p.token_stride));
      vr[4 + r] = *reinterpret_cast<const VRaw*>(vh + o1 + (v_lane + r * p.token_stride));
    }
  };

  f32x4 acc[CV];
#pragma unroll
  for (int t = 0; t < CV; ++t) acc[t] = f32x4{};
  float m = -FLT_MAX, l = 0.f;   // of the lane's head; l: this lane's keys only

  int i = first + wave, slot = 0;
  if (i < last) {
    look_up(i);
    const int64_t o0 = tile_off(0, 0), o1 = tile_off(0, 1);
    load_k(o0, o1);
    load_v(o0, o1);
  }
  while (i < last) {
    const int token = blocks.token(i);
    const int next = i + WAVES;
    const bool more = next < last;
    int64_t o0 = 0, o1 = 0;
    if (more) {
      if (++slot == 32) {
        slot = 0;
        look_up(next);
      }
      o0 = tile_off(slot, 0);
      o1 = tile_off(slot, 1);
    }

    f32x4 s[2] = {f32x4{}, f32x4{}};
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u32x4 a;
        if constexpr (FP8) a = widen<DT>(kr[t][c / 2][2 * (c % 2)], kr[t][c / 2][2 * (c % 2) + 1]);
        else a = kr[t][c];
        s[t] = T::mfma(a, qf[c], s[t]);
      }
    }
    if (more) load_k(o0, o1);

    const bool edge = token + kBlock > len || (token < lo_window && token + kBlock > p.sinks);
    float x[8];
    bool hidden[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) x[j] = s[j / 4][j % 4] * p.c;
    if (edge) {
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const int key = token + 16 * (j / 4) + 4 * g + j % 4;
        hidden[j] = key >= len || (key < lo_window && key >= p.sinks);
        if (hidden[j]) x[j] = -INFINITY;
      }
    }
    float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                      fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    top = fmaxf(m, max_over_groups(top));
    if (__any(top > m)) {
      const float alpha = __builtin_amdgcn_exp2f(m - top);
      l *= alpha;
#pragma unroll
      for (int t = 0; t < CV; ++t) acc[t] *= alpha;
      m = top;
    }
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      e[j] = __builtin_amdgcn_exp2f(x[j] - m);
      l += e[j];
    }
    u32x4 pf;
#pragma unroll
    for (int w = 0; w < 4; ++w) pf[w] = T::pack(e[2 * w], e[2 * w + 1]);

    if (edge) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (hidden[j]) vr[j] = VRaw{};
    }
    // each row's columns as pairs of 16-bit values
    uint32_t rows[8][CV / 2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (!FP8) {
#pragma unroll
        for (int w = 0; w < CV / 2; ++w) rows[j][w] = vr[j][w];
      } else if constexpr (CV == 8) {
        const u32x4 r = widen<DT>(vr[j][0], vr[j][1]);
#pragma unroll
        for (int w = 0; w < 4; ++w) rows[j][w] = r[w];
      } else {
        const u32x4 r = widen<DT>(vr[j], 0);
        rows[j][0] = r[0], rows[j][1] = r[1];
      }
    }
#pragma unroll
    for (int t = 0; t < CV; ++t) {
      u32x4 a;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        a[w] = __builtin_amdgcn_perm(rows[2 * w + 1][t / 2], rows[2 * w][t / 2],
                                     t % 2 ? 0x07060302u : 0x05040100u);
      acc[t] = T::mfma(a, pf, acc[t]);
    }
    if (more) load_v(o0, o1);
    i = next;
  }

  // ---- join the wavefronts: each puts its O, scaled to the common maximum, into LDS ----
  extern __shared__ __attribute__((aligned(16))) float lds[];
  float* const ml = lds;                      // [WAVES][16][2]
  float* const part = lds + WAVES * 32;       // [WAVES][16][D]
  l = sum_over_groups(l);
  bad = __any(bad);
  if (bad) l = __builtin_nanf("");            // a length or page out of range
  if (g == 0) {
    ml[(wave * 16 + n) * 2] = m;
    ml[(wave * 16 + n) * 2 + 1] = l;
  }
  __syncthreads();
  float top = -FLT_MAX;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ml[(w * 16 + n) * 2]);
  float total = 0.f;
#pragma unroll
  for (int w = 0; w < WAVES; ++w)
    total += ml[(w * 16 + n) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(w * 16 + n) * 2] - top);
  const float weight = __builtin_amdgcn_exp2f(m - top);
#pragma unroll
  for (int r = 0; r < 4; ++r) {
    // columns (4 g + r) CV .. + CV - 1 of head n
    float* dst = part + (wave * 16 + n) * D + (4 * g + r) * CV;
#pragma unroll
    for (int t = 0; t < CV; t += 4)
      *reinterpret_cast<f32x4*>(dst + t) = f32x4{acc[t][r], acc[t + 1][r], acc[t + 2][r], acc[t + 3][r]} * weight;
  }
  __syncthreads();
  // totals by head, for the threads that finish it
  if (wave == 0 && g == 0) {
    ml[n * 2] = top;
    ml[n * 2 + 1] = total;
  }
  __syncthreads();
  const int active = p.splits == 1 ? 1 : (blocks.total + p.chunk - 1) / p.chunk;
  for (int e4 = threadIdx.x; e4 < heads * (D / 4); e4 += 64 * WAVES) {
    const int h = e4 / (D / 4), col = e4 % (D / 4) * 4;
    f32x4 sum = f32x4{};
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
      sum += *reinterpret_cast<const f32x4*>(part + (w * 16 + h) * D + col);
    const float mh = ml[h * 2], lh = ml[h * 2 + 1];
    const size_t row = (size_t)b * p.H + head0 + h;
    if (active <= 1) {
      // no visible token: l = 0 gives O = 0 and lse = -inf
      const float inv = lh == 0.f ? 0.f : p.v_scale / lh;
      sum *= inv;
      *reinterpret_cast<u32x2*>(p.o + row * D + col) = u32x2{T::pack(sum[0], sum[1]), T::pack(sum[2], sum[3])};
      if (col == 0) p.lse[row] = (mh + log2f(lh)) * 0.69314718055994531f;
    } else {
      *reinterpret_cast<f32x4*>(p.part_o + (row * p.splits + split) * D + col) = sum;
      if (col == 0) {
        p.part_ml[(row * p.splits + split) * 2] = mh;
        p.part_ml[(row * p.splits + split) * 2 + 1] = lh;
      }
    }
  }
}

// Joins the chunks of each (sequence, head), in order: one wavefront a row.
template <int DT, int D>
__global__ __launch_bounds__(256) void decode_join_kernel(Params p, int rows) {
  using T = Type16<DT>;
  const int lane = threadIdx.x & 63;
  const int row = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (row >= rows) return;
  const int len = p.lengths[row / p.H];
  if (len < 0 || len > p.limit) return;   // the chunk kernel wrote it
  const Blocks blocks(p, len);
  const int active = (blocks.total + p.chunk - 1) / p.chunk;
  if (active <= 1) return;
  const float* ml = p.part_ml + (size_t)row * p.splits * 2;
  float top = -FLT_MAX;
  for (int s = lane; s < active; s += 64) top = fmaxf(top, ml[2 * s]);
#pragma unroll
  for (int x = 1; x < 64; x *= 2) top = fmaxf(top, __shfl_xor(top, x));
  float total = 0.f;
  constexpr int C = D / 64;   // columns of a lane
  float o[C] = {};
  const float* part = p.part_o + (size_t)row * p.splits * D + lane * C;
#pragma unroll 8
  for (int s = 0; s < active; ++s) {
    const float w = __builtin_amdgcn_exp2f(ml[2 * s] - top);
    total += w * ml[2 * s + 1];
#pragma unroll
    for (int c = 0; c < C; ++c) o[c] += w * part[(size_t)s * D + c];
  }
  const float inv = p.v_scale / total;
  uint16_t* dst = p.o + (size_t)row * D + lane * C;
  if constexpr (C == 2) {
    *reinterpret_cast<uint32_t*>(dst) = T::pack(o[0] * inv, o[1] * inv);
  } else {
    *dst = (uint16_t)T::pack(o[0] * inv, 0.f);
  }
  if (lane == 0) p.lse[row] = (top + log2f(total)) * 0.69314718055994531f;
}

template <int DT, int D, bool FP8, int WAVES>
hipError_t launch_chunks(const Params& p, unsigned grid, hipStream_t stream) {
  constexpr size_t lds = (size_t)WAVES * (32 + 16 * D) * sizeof(float);
  static_assert(lds <= 64 * 1024, "within the LDS a kernel has without asking for more");
  hipLaunchKernelGGL((decode_kernel<DT, D, FP8, WAVES>), dim3(grid), dim3(64 * WAVES), lds, stream, p);
  return hipGetLastError();
}

template <int DT, int D>
hipError_t launch_width(const DecodeArgs& a, const DecodePlan& plan, hipStream_t stream) {
  Params p = {};
  p.q = a.q, p.o = a.o, p.lse = a.lse, p.lengths = a.lengths;
  p.k = static_cast<const uint8_t*>(a.cache.k);
  p.v = static_cast<const uint8_t*>(a.cache.v);
  p.table = a.cache.table;
  p.page_stride = a.cache.page_stride;
  p.token_stride = a.cache.token_stride, p.head_stride = a.cache.head_stride;
  p.num_pages = a.cache.num_pages, p.table_cols = a.cache.table_cols;
  p.page = FastDiv(a.cache.page_size);
  p.H = a.H, p.Hkv = a.Hkv, p.group = a.H / a.Hkv, p.tiles = (p.group + 15) / 16;
  p.splits = plan.splits, p.chunk = plan.chunk;
  p.limit = a.limit, p.window = a.window, p.sinks = a.sinks;
  p.c = a.c, p.v_scale = a.v_scale;
  p.part_o = a.workspace;
  p.part_ml = a.workspace + (size_t)a.B * a.H * plan.splits * a.d;
  const unsigned grid = (unsigned)a.B * a.Hkv * p.tiles * plan.splits;
  hipError_t e = a.cache.fp8 ? launch_chunks<DT, D, true, 4>(p, grid, stream)
                             : launch_chunks<DT, D, false, 4>(p, grid, stream);
  if (e == hipSuccess && plan.splits > 1) {
    const int rows = a.B * a.H;
    hipLaunchKernelGGL((decode_join_kernel<DT, D>), dim3((rows + 3) / 4), dim3(256), 0, stream, p, rows);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace

hipError_t launch_decode(const DecodeArgs& a, const DecodePlan& plan, hipStream_t stream) {
  if (a.d == 64) {
    return a.dtype == 0 ? launch_width<0, 64>(a, plan, stream) : launch_width<1, 64>(a, plan, stream);
  }
  return a.dtype == 0 ? launch_width<0, 128>(a, plan, stream) : launch_width<1, 128>(a, plan, stream);
}

}  // namespace qm
