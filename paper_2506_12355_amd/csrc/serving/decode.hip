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
// take the same path.  Scores, maxima and sums are in fp32, base 2 (c = scale log2 e).
// P enters the second product as two values of the query's 16-bit type, P rounded and
// what that left, one MFMA each: 2^-16 (bf16) or 2^-22 (f16) of a weight is lost, where
// one value loses 2^-8 or 2^-11, as much as the rounding of O.  The wavefronts wait for
// memory, so that the second MFMA costs little (us, one value -> two: 64 sequences of 0 to
// 8192 tokens 196.6 -> 197.2, one of 131072 in E4M3 58.4 -> 58.6, one of 1000 10.1 -> 10.3).
// f16's smallest step is 2^-24: there the operands are 2^15 times the weights (kWeight),
// the largest of which is 1, so that of those far below it 2^-40 each is lost.  Row sums
// take the weights in fp32.
//
// Keys that are hidden (past the length, or before the window and past the first keys)
// get the score -inf and a zero V row: what their memory holds, NaN included, does not
// reach the result.
//
// Work: a row is one (sequence, key/value head, 16-head tile), its work its blocks.
// Where rows are short, or many, a workgroup takes a whole row (decode_rules.h).  Else all rows'
// blocks, end to end, are dealt in equal shares to as many workgroups as the device
// holds, which evens out sequences of any lengths.  A workgroup's wavefronts take a
// piece's blocks in turn and join their (m, l, O) in LDS; of a row that was cut, each
// piece leaves its unnormalised O, m and l in the workspace, and a second kernel joins
// them in order, so results do not depend on which finished first.  A workgroup's range
// cuts at most its first row (slot 2 w: a piece that continues a row) and its last
// (slot 2 w + 1: a piece that begins one).
//
// Measured (us; a sum over 1 GiB reads 6.18 TB/s, a floor of 0.162 us a MB): 64 sequences
// of 0 to 8192 tokens, 64/8 heads, bf16, d = 128 199 (5.4 TB/s), all of 8192 (32 of them)
// 195 (5.5), of 32768 (64) 1405 (6.12); one of 131072 with E4M3 pages 58.7 (4.6); one of
// 1000 10.0, a chain of latencies: length, page numbers, rows, join, second kernel.
//
// Window: the blocks walked are those with first keys, then those from the window on;
// list index i is block i, or i + skip past the first keys' blocks.
#include <float.h>

#include "decode_rules.h"
#include "serving_device.h"
#include "serving_launch.h"

namespace qm {
namespace {

constexpr int kBlock = kDecodeBlock;   // tokens of a wavefront's step
constexpr int kMinShare = 4;           // least blocks of a workgroup's share: one a wavefront
// The second product's factor (see above); O is divided by it at the end.
template <int DT>
constexpr float kWeight = DT == 0 ? 32768.f : 1.f;
// What a row costs a workgroup beside its blocks, in blocks: its first loads and its
// join, 5-8 us, against 1.1 us a block.  Counted as 0, 6 and 12 (us): 512 rows of up to
// 8192 tokens 205, 198, 199; up to 2000 88, 64, 65; 8 rows of 2000 13.4, 10.8, 10.8.
constexpr int kRowCost = 6;

struct Params {
  const uint16_t* q;
  uint16_t* o;
  float* lse;
  const int32_t* lengths;
  const uint8_t *k, *v;
  const int32_t* table;
  float* part_o;     // [2 grid][16][d]
  float* part_ml;    // [2 grid][16][2]
  int32_t* desc;     // [rows][2]: first workgroup of a row, and its pieces
  int grid;          // workgroups of equal shares
  int64_t page_stride;
  uint32_t token_stride, head_stride;
  int num_pages, table_cols;
  FastDiv page;
  int B, H, Hkv, group, tiles;   // query heads per key/value head, and 16-head tiles of them
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

// Over the four lanes that hold a head: v_permlane16_swap and v_permlane32_swap of a
// value with itself leave each lane the values of both halves of its pair of rows, or
// of the wavefront.
template <typename F>
__device__ __forceinline__ float over_groups(float x, F f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];
  const uint32_t v = __builtin_bit_cast(uint32_t, (float)f(__builtin_bit_cast(float, a), __builtin_bit_cast(float, b)));
  const auto s = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  const uint32_t c = s[0], d = s[1];
  return f(__builtin_bit_cast(float, c), __builtin_bit_cast(float, d));
}
__device__ __forceinline__ float max_over_groups(float x) {
  return over_groups(x, [](float a, float b) { return fmaxf(a, b); });
}
__device__ __forceinline__ float sum_over_groups(float x) {
  return over_groups(x, [](float a, float b) { return a + b; });
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

// Four columns of a finished row: O = sum / (kWeight l), and lse.  No visible token (l = 0) gives
// O = 0 and lse = -inf.
template <int DT>
__device__ __forceinline__ void finish(const Params& p, size_t row, int d, int col, f32x4 sum, float m, float l) {
  sum *= l == 0.f ? 0.f : p.v_scale * (1.f / kWeight<DT>) / l;
  *reinterpret_cast<u32x2*>(p.o + row * d + col) =
      u32x2{Type16<DT>::pack(sum[0], sum[1]), Type16<DT>::pack(sum[2], sum[3])};
  if (col == 0) p.lse[row] = (m + log2f(l)) * 0.69314718055994531f;
}

// A row's blocks lo .. hi - 1 by one workgroup: joined into the result where they are
// the whole row, else into partial slot `slot`.
template <int DT, int D, bool FP8, int WAVES>
__device__ __forceinline__ void piece(const Params& p, float* lds, int b, int row, int len, bool bad,
                                      const Blocks& blocks, int lo, int hi, int slot) {
  using T = Type16<DT>;
  constexpr int ES = FP8 ? 1 : 2;
  constexpr int NC = D / 32;            // k-steps of the first product
  constexpr int NK = D * ES / 64;       // 16-byte K loads of a lane and tile
  constexpr int CV = D / 16;            // V columns of a lane, and M tiles
  using VRaw = typename Raw<CV * ES>::T;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int hkv = row / p.tiles, tile = row - hkv * p.tiles;
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
  // the i-th.  A tile without a visible key may have no page: it borrows its neighbour's
  // (a block on the list has a visible key in one of the two), and its keys are hidden.
  int off_lo = 0, off_hi = 0;
  auto look_up = [&](int i0) __attribute__((always_inline)) {
    const int li = i0 + WAVES * (lane >> 1);
    int64_t off = 0;
    if (li < hi) {
      int token = blocks.token(li) + 16 * (lane & 1);
      if (token >= len || (token + 16 <= lo_window && token >= p.sinks)) token ^= 16;
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

  // K and V of the block in hand, each replaced by the next block's as soon as its
  // operands are read.  (With two blocks in flight a wavefront, 248 registers instead of
  // 191, no case was faster: the memory system's queues are full either way.)
  u32x4 k[2][NK];
  VRaw v[8];
  auto load_k = [&](int64_t o0, int64_t o1) __attribute__((always_inline)) {
#pragma unroll
    for (int c = 0; c < NK; ++c) {
      k[0][c] = *reinterpret_cast<const u32x4*>(kh + o0 + (k_lane + 64 * c));
      k[1][c] = *reinterpret_cast<const u32x4*>(kh + o1 + (k_lane + 64 * c));
    }
  };
  auto load_v = [&](int64_t o0, int64_t o1) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      v[r] = *reinterpret_cast<const VRaw*>(vh + o0 + (v_lane + r * p.token_stride));
      v[4 + r] = *reinterpret_cast<const VRaw*>(vh + o1 + (v_lane + r * p.token_stride));
    }
  };

  f32x4 acc[CV];
#pragma unroll
  for (int t = 0; t < CV; ++t) acc[t] = f32x4{};
  float m = -FLT_MAX, l = 0.f;   // of the lane's head; l: this lane's keys only

  int i = lo + wave, nth = 0;   // nth: of the 32 blocks looked up, the one in hand
  if (i < hi) {
    look_up(i);
    const int64_t o0 = tile_off(0, 0), o1 = tile_off(0, 1);
    load_k(o0, o1);
    load_v(o0, o1);
  }
  for (; i < hi; i += WAVES) {
    const int token = blocks.token(i);
    const bool more = i + WAVES < hi;
    int64_t o0 = 0, o1 = 0;
    if (more) {
      if (++nth == 32) {
        nth = 0;
        look_up(i + WAVES);
      }
      o0 = tile_off(nth, 0);
      o1 = tile_off(nth, 1);
    }

    f32x4 s[2] = {f32x4{}, f32x4{}};
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u32x4 a;
        if constexpr (FP8) a = widen<DT>(k[t][c / 2][2 * (c % 2)], k[t][c / 2][2 * (c % 2) + 1]);
        else a = k[t][c];
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
    u32x4 pf, rest;   // the weights, and what rounding them left
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float e0 = e[2 * w] * kWeight<DT>, e1 = e[2 * w + 1] * kWeight<DT>;
      pf[w] = T::pack(e0, e1);
      const f32x2 near = T::unpack(pf[w]);
      rest[w] = T::pack(e0 - near[0], e1 - near[1]);
    }

    if (edge) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (hidden[j]) v[j] = VRaw{};
    }
    // each row's columns as pairs of 16-bit values
    uint32_t rows[8][CV / 2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (!FP8) {
#pragma unroll
        for (int w = 0; w < CV / 2; ++w) rows[j][w] = v[j][w];
      } else if constexpr (CV == 8) {
        const u32x4 r = widen<DT>(v[j][0], v[j][1]);
#pragma unroll
        for (int w = 0; w < 4; ++w) rows[j][w] = r[w];
      } else {
        const u32x4 r = widen<DT>(v[j], 0);
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
      acc[t] = T::mfma(a, rest, acc[t]);
    }
    if (more) load_v(o0, o1);
  }

  // ---- join the wavefronts: each scales its O to the common maximum; half of them put
  // theirs into LDS, the other half add their own ----
  constexpr int HALF = WAVES / 2;
  float* const ml = lds;                     // [WAVES][16][2]
  float* const part = lds + WAVES * 32;      // [HALF][16][D]
  l = sum_over_groups(l);
  if (__any(bad)) l = __builtin_nanf("");   // a length or page out of range
  if (g == 0) {
    ml[(wave * 16 + n) * 2] = m;
    ml[(wave * 16 + n) * 2 + 1] = l;
  }
  __syncthreads();
  float top = -FLT_MAX;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ml[(w * 16 + n) * 2]);
  const float weight = __builtin_amdgcn_exp2f(m - top);
  // columns (4 g + r) CV .. + CV - 1 of head n
  float* const mine = part + ((wave % HALF) * 16 + n) * D + 4 * g * CV;
#pragma unroll
  for (int phase = 0; phase < 2; ++phase) {
    if (wave / HALF == phase) {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int t = 0; t < CV; t += 4) {
          f32x4* dst = reinterpret_cast<f32x4*>(mine + r * CV + t);
          f32x4 x = f32x4{acc[t][r], acc[t + 1][r], acc[t + 2][r], acc[t + 3][r]} * weight;
          if (phase) x += *dst;
          *dst = x;
        }
      }
    }
    __syncthreads();
  }
  const bool whole = lo == 0 && hi >= blocks.total;
  for (int e4 = threadIdx.x; e4 < heads * (D / 4); e4 += 64 * WAVES) {
    const int h = e4 / (D / 4), col = e4 % (D / 4) * 4;
    f32x4 sum = f32x4{};
#pragma unroll
    for (int w = 0; w < HALF; ++w) sum += *reinterpret_cast<const f32x4*>(part + (w * 16 + h) * D + col);
    float mh = -FLT_MAX, lh = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) mh = fmaxf(mh, ml[(w * 16 + h) * 2]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
      lh += ml[(w * 16 + h) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(w * 16 + h) * 2] - mh);
    if (whole) {
      finish<DT>(p, (size_t)b * p.H + head0 + h, D, col, sum, mh, lh);
    } else {
      *reinterpret_cast<f32x4*>(p.part_o + ((size_t)slot * 16 + h) * D + col) = sum;
      if (col == 0) *reinterpret_cast<f32x2*>(p.part_ml + (slot * 16 + h) * 2) = f32x2{mh, lh};
    }
  }
}

// Quotients of the shares, nearly always of 32-bit values.
__device__ __forceinline__ int64_t quotient(int64_t x, int64_t d) {
  return (x | d) >> 32 ? x / d : (int64_t)((uint32_t)x / (uint32_t)d);
}

// Inclusive sum over the lanes up to each.
__device__ __forceinline__ int running_sum(int x) {
  x += __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false);   // row_shr:1, 2, 4, 8
  x += __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false);
  x += __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false);   // row_bcast:15, 31
  x += __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false);
  return x;
}

// One workgroup a row.
template <int DT, int D, bool FP8, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void decode_rows_kernel(Params p) {
  __shared__ __attribute__((aligned(16))) float lds[WAVES * 32 + WAVES / 2 * 16 * D];
  const int rows = p.Hkv * p.tiles;   // of a sequence
  const int b = blockIdx.x / rows;
  const int len = p.lengths[b];
  const bool bad = len < 0 || len > p.limit;
  const Blocks blocks(p, bad ? 0 : len);
  piece<DT, D, FP8, WAVES>(p, lds, b, blockIdx.x - b * rows, bad ? 0 : len, bad, blocks, 0, blocks.total, 0);
}

// Equal shares of all rows' blocks.
template <int DT, int D, bool FP8>
__global__ __launch_bounds__(256, 2) void decode_shares_kernel(Params p) {
  constexpr int WAVES = 4;
  __shared__ __attribute__((aligned(16))) float lds[WAVES * 32 + WAVES / 2 * 16 * D];
  const int rows = p.Hkv * p.tiles;   // of a sequence
  const int lane = threadIdx.x & 63;
  // a sequence's length, 0 where the join writes it (none, or one out of range)
  auto length_of = [&](int b) {
    const int len = b < p.B ? p.lengths[b] : 0;
    return len < 0 || len > p.limit ? 0 : len;
  };
  // What a sequence costs: its rows' blocks, and for each row what a piece costs beside
  // its blocks (kRowCost), so that a share of many short rows holds fewer blocks.
  auto cost_of = [&](int len) {
    const int n = Blocks(p, len).total;
    return n ? n + kRowCost : 0;
  };
  // All sequences' costs, and the one that this workgroup's share begins in: each
  // wavefront for itself, a sequence a lane, so that no barrier lies before the first loads.
  int len = length_of(lane);
  int sum = running_sum(cost_of(len));
  int64_t all = __builtin_amdgcn_readlane(sum, 63);
  for (int b0 = 64; b0 < p.B; b0 += 64)
    all += __builtin_amdgcn_readlane(running_sum(cost_of(length_of(b0 + lane))), 63);
  const int64_t total = all * rows;
  int64_t share = quotient(total + gridDim.x - 1, gridDim.x);
  share = share < kMinShare ? kMinShare : share;
  const int64_t begin = blockIdx.x * share, end = begin + share < total ? begin + share : total;
  if (begin >= total) return;
  const int64_t at = quotient(begin, rows);   // in costs of one row of each sequence
  int64_t upto = 0;                           // those of the sequences before
  int b = 0;
  while (upto + __builtin_amdgcn_readlane(sum, 63) <= at) {
    upto += __builtin_amdgcn_readlane(sum, 63);
    b += 64;
    if (b >= p.B) return;   // (only lengths that change under the call get here)
    len = length_of(b + lane);
    sum = running_sum(cost_of(len));
  }
  const int first = __builtin_ctzll(__ballot(upto + sum > at));
  if (first) upto += __builtin_amdgcn_readlane(sum, first - 1);
  b += first;
  len = __builtin_amdgcn_readlane(len, first);
  int64_t left = end - begin;
  int64_t before = begin - upto * rows;   // costs of the sequence's rows before the share
  for (;;) {
    const Blocks blocks(p, len);
    if (blocks.total) {
      const int cost = blocks.total + kRowCost;   // a row: its blocks, then what it costs beside
      int row = (int)quotient(before, cost);
      int lo = (int)(before - (int64_t)row * cost);
      for (; row < rows && left > 0; ++row, lo = 0) {
        const int cut = (int)(lo + left < cost ? lo + left : cost), hi = min(cut, blocks.total);
        left -= cut - lo;
        if (lo == 0 && threadIdx.x == 0) {
          int32_t* d = p.desc + 2 * ((size_t)b * rows + row);
          d[0] = blockIdx.x;
          d[1] = 1 + (int)quotient(blocks.total - hi + share - 1, share);
        }
        if (lo >= blocks.total) continue;
        piece<DT, D, FP8, WAVES>(p, lds, b, row, len, false, blocks, lo, hi, 2 * blockIdx.x + (lo == 0));
        if (left > 0) __syncthreads();   // the next piece's join refills the LDS
      }
      before = 0;
    }
    if (left <= 0 || ++b >= p.B) return;
    len = length_of(b);
  }
}

// Joins the pieces of each (sequence, head), in a fixed order, and writes the sequences
// that have no blocks.  T threads a head: 256 where rows have many pieces, 64 where few.
template <int DT, int D, int T>
__global__ __launch_bounds__(256) void decode_join_kernel(Params p, int heads) {
  constexpr int L = D / 4;     // threads of a piece, 4 columns each
  constexpr int G = T / L;     // pieces side by side
  __shared__ __attribute__((aligned(16))) float lds[256 / T][G][D + 4];
  const int own_head = T == 256 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int id = blockIdx.x * (256 / T) + own_head;
  if (id >= heads) return;
  const int b = id / p.H, h = id - b * p.H;
  const int len = p.lengths[b];
  const int thread = threadIdx.x % T, col = thread % L * 4, own = thread / L;
  if (len <= 0 || len > p.limit) {
    if (own == 0) finish<DT>(p, id, D, col, f32x4{}, -FLT_MAX, len == 0 ? 0.f : __builtin_nanf(""));
    return;
  }
  const int hkv = h / p.group, in_group = h - hkv * p.group;
  const int32_t* d = p.desc + 2 * (((size_t)b * p.Hkv + hkv) * p.tiles + in_group / 16);
  // (bounded by the partial results there are: lengths that change under the call can
  // give a row whose numbers were never written)
  const int first = d[0], pieces = first >= 0 && first < p.grid ? min(d[1], p.grid - first) : 0;
  if (pieces <= 1) return;
  float m = -FLT_MAX, l = 0.f;
  f32x4 o = f32x4{};
#pragma unroll 4
  for (int j = own; j < pieces; j += G) {
    const size_t at = (size_t)(j ? 2 * (first + j) : 2 * first + 1) * 16 + in_group % 16;
    const f32x2 ml = *reinterpret_cast<const f32x2*>(p.part_ml + at * 2);
    const f32x4 x = *reinterpret_cast<const f32x4*>(p.part_o + at * D + col);
    const float top = fmaxf(m, ml[0]);
    const float a = __builtin_amdgcn_exp2f(m - top), w = __builtin_amdgcn_exp2f(ml[0] - top);
    o = o * a + x * w;
    l = l * a + ml[1] * w;
    m = top;
  }
  float* mine = lds[own_head][own];
  *reinterpret_cast<f32x4*>(mine + col) = o;
  if (col == 0) mine[D] = m, mine[D + 1] = l;
  if (T == 256) {
    __syncthreads();
  } else {   // one wavefront: its LDS accesses only have to stay in order
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  }
  if (own) return;
  const int n = min(G, pieces);
  float top = -FLT_MAX;
  for (int i = 0; i < n; ++i) top = fmaxf(top, lds[own_head][i][D]);
  f32x4 sum = f32x4{};
  float total = 0.f;
  for (int i = 0; i < n; ++i) {
    const float* x = lds[own_head][i];
    const float w = __builtin_amdgcn_exp2f(x[D] - top);
    total += w * x[D + 1];
    sum += *reinterpret_cast<const f32x4*>(x + col) * w;
  }
  finish<DT>(p, id, D, col, sum, top, total);
}

template <int DT, int D, bool FP8>
hipError_t launch_kernels(const DecodeArgs& a, const DecodePlan& plan, Params& p, hipStream_t stream) {
  const unsigned rows = (unsigned)a.B * a.Hkv * p.tiles;
  if (plan.grid == 0) {
    hipLaunchKernelGGL((decode_rows_kernel<DT, D, FP8, 8>), dim3(rows), dim3(512), 0, stream, p);
    return hipGetLastError();
  }
  hipLaunchKernelGGL((decode_shares_kernel<DT, D, FP8>), dim3(plan.grid), dim3(256), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int heads = a.B * a.H;
  if (plan.grid > 8 * (int64_t)rows)
    hipLaunchKernelGGL((decode_join_kernel<DT, D, 256>), dim3(heads), dim3(256), 0, stream, p, heads);
  else
    hipLaunchKernelGGL((decode_join_kernel<DT, D, 64>), dim3((heads + 3) / 4), dim3(256), 0, stream, p, heads);
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
  p.B = a.B, p.H = a.H, p.Hkv = a.Hkv, p.group = a.H / a.Hkv, p.tiles = (p.group + 15) / 16;
  p.limit = a.limit, p.window = a.window, p.sinks = a.sinks;
  p.c = a.c, p.v_scale = a.v_scale;
  p.grid = plan.grid;
  p.part_o = a.workspace;
  p.part_ml = p.part_o + (size_t)2 * plan.grid * 16 * a.d;
  p.desc = reinterpret_cast<int32_t*>(p.part_ml + (size_t)2 * plan.grid * 16 * 2);
  return a.cache.fp8 ? launch_kernels<DT, D, true>(a, plan, p, stream)
                     : launch_kernels<DT, D, false>(a, plan, p, stream);
}

}  // namespace

hipError_t launch_decode(const DecodeArgs& a, const DecodePlan& plan, hipStream_t stream) {
  if (a.d == 64) {
    return a.dtype == 0 ? launch_width<0, 64>(a, plan, stream) : launch_width<1, 64>(a, plan, stream);
  }
  return a.dtype == 0 ? launch_width<0, 128>(a, plan, stream) : launch_width<1, 128>(a, plan, stream);
}

}  // namespace qm
