// Attention of one new token per sequence over a paged cache whose first tokens, the
// prefix, are the same pages for all sequences.
//
// With m, l, O the maximum, sum and unnormalised result of a part of the keys, softmax over
// prefix and own tokens is their join: m = max, l = sum l_i 2^(m_i - m), O alike (base 2).
//
// Prefix: the queries of all sequences that read a key/value head are the rows of one
// product, B H / Hkv of them, so keys and values are read once for many of them and not once
// a sequence.  Bound: HBM where rows are few, 4 d flops a row and key against 4 d bytes a key;
// from some 150 rows a head the matrix cores.  A workgroup takes a part of the prefix for a
// tile of rows and leaves m, l and O in the workspace.  All of the prefix is visible to all
// rows, so only its last block has hidden keys.  Two ways, by the number of rows
// (shared_rules.h):
//   16 or 32 rows a workgroup (prefix_piece): its wavefronts take blocks of 32 tokens in turn,
//     operands straight from memory as in decode.hip, each read meeting one or two 16-row
//     tiles, and join.
//   128 rows, 32 a wavefront (prefix_block_rows): the wavefronts go over the same blocks,
//     staged in LDS.
// Own tokens: equal shares of all sequences' blocks as in decode.hip, from the prefix on,
// by further workgroups of the same launch; then one kernel joins all parts in order.
//
// As in decode.hip each weight enters the second product as two 16-bit values, so that o is
// as far off as a result rounded once; on the matrix cores that is half as many products again.
//
// Measured (us, bf16, d = 128, 64/8 heads, no own tokens, with the join): 64 sequences behind
// 8192 tokens 44.2, behind 32768 108.4 (2.7 us a 1024 tokens: 800 TFLOP/s, 1200 of products); in
// prefix_piece alone 58.7 and 179.
#include "decode_device.h"
#include "shared_rules.h"

// Checking build: waits for all loads and a barrier more in each step of the rings.
#ifdef QM_DEBUG_SYNC
constexpr bool kDebugSync = true;
#else
constexpr bool kDebugSync = false;
#endif

namespace qm {
namespace {

// Weights are formed against a row's maximum so far, and redone against a new one where eight
// of them, a lane's, sum to more than kMostWeight (always in a row's first block): a step's
// weights then wait for no maximum, and the accumulators are scaled in few steps.  A row is
// redone by its own weights alone, so that what its neighbours hold changes none of its bits;
// then each of 32 rows has steps of its own, and room is what keeps them few (us, 64 sequences of
// 64/8 heads behind 32768 tokens, scores of a standard deviation of 1, 3 and 6: bf16, room 1024
// 110, 111, 124, 65536 107, 108, 116; E4M3 behind 65500 73, 73, 83, 72, 72, 76; f16, room 16 118, 131,
// 134, 256 117, 122, 127; with room 8, spread 1, bf16 117 where 1024 has 105).  bf16 has fp32's
// exponents; f16's factor brings the largest weights to 2^15, so that of those far below a
// row's largest 2^-32 each is lost: with 65536 tokens 2^-16 of their values.
template <int DT>
constexpr float kMostWeight = DT == 0 ? 256.f : 65536.f;
template <int DT>
constexpr float kFactor = DT == 0 ? 128.f : 1.f;

// a - the low half of w, b - the high half: what rounding a and b into w left, exactly.  (The
// factors stand in registers: written as constants, -1 in the low half is compiled into the
// immediate -1.0, which the instruction takes as -1 in the high one.)
template <int DT>
__device__ __forceinline__ f32x2 minus_halves(float a, float b, uint32_t w, uint32_t low, uint32_t high) {
  if constexpr (DT == 1) {
    const bf16x2 x = __builtin_bit_cast(bf16x2, w);
    return f32x2{__builtin_amdgcn_fdot2_f32_bf16(x, __builtin_bit_cast(bf16x2, low), a, false),
                 __builtin_amdgcn_fdot2_f32_bf16(x, __builtin_bit_cast(bf16x2, high), b, false)};
  } else {
    const f32x2 x = Type16<DT>::unpack(w);
    return f32x2{a - x[0], b - x[1]};
  }
}

struct SharedParams {
  Params own;
  const int32_t* prefix_table;
  float* prefix_o;    // [Hkv][tiles 16-row tiles][splits][16][d]
  float* prefix_ml;   // [..][16][2]
  int rows, tiles;    // of a key/value head; tiles of 16 rt rows
  int splits, blocks, prefix_grid;
};

// A part of the prefix, blocks lo .. hi - 1, for one tile of 16 RT rows.
template <int DT, int D, bool FP8, int RT, int WAVES>
__device__ __forceinline__ void prefix_piece(const SharedParams& sp, float* lds, int hkv, int tile, int split,
                                             int lo, int hi) {
  using T = Type16<DT>;
  constexpr int ES = FP8 ? 1 : 2;
  constexpr int NC = D / 32;            // k-steps of the first product
  constexpr int NK = D * ES / 64;       // 16-byte K loads of a lane and tile
  constexpr int CV = D / 16;            // V columns of a lane, and M tiles
  using VRaw = typename Raw<CV * ES>::T;
  const Params& p = sp.own;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int len = p.prefix;
  bool bad = false;

  u32x4 qf[RT][NC];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = (tile * RT + rt) * 16 + n;
#pragma unroll
    for (int c = 0; c < NC; ++c) qf[rt][c] = u32x4{};
    if (row < sp.rows) {
      const int b = row / p.group;
      const uint16_t* q = p.q + ((size_t)b * p.H + hkv * p.group + (row - b * p.group)) * D;
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int col = FP8 ? (c / 2) * 64 + g * 16 + (c % 2) * 8 : c * 32 + g * 8;
        qf[rt][c] = *reinterpret_cast<const u32x4*>(q + col);
      }
    }
  }

  const uint8_t* kh = p.k + (size_t)hkv * p.head_stride;
  const uint8_t* vh = p.v + (size_t)hkv * p.head_stride;
  const uint32_t k_lane = n * p.token_stride + g * 16;
  const uint32_t v_lane = 4 * g * p.token_stride + n * (CV * ES);

  // Offsets of the tiles of the wavefront's next 32 blocks: lane 2 i + t holds tile t of
  // the i-th.  The last block's second tile may have no token: it borrows the first's page.
  int off_lo = 0, off_hi = 0;
  auto look_up = [&](int i0) __attribute__((always_inline)) {
    const int li = i0 + WAVES * (lane >> 1);
    int64_t off = 0;
    if (li < hi) {
      int token = li * kBlock + 16 * (lane & 1);
      if (token >= len) token ^= 16;
      const uint32_t at = p.page.div((uint32_t)token);
      const int page = sp.prefix_table[at];
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

  f32x4 acc[RT][CV];
  float m[RT], l[RT];   // of the lane's rows; l: this lane's keys only
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = -FLT_MAX, l[rt] = 0.f;
#pragma unroll
    for (int t = 0; t < CV; ++t) acc[rt][t] = f32x4{};
  }

  int i = lo + wave, nth = 0;   // nth: of the 32 blocks looked up, the one in hand
  if (i < hi) {
    look_up(i);
    const int64_t o0 = tile_off(0, 0), o1 = tile_off(0, 1);
    load_k(o0, o1);
    load_v(o0, o1);
  }
  for (; i < hi; i += WAVES) {
    const int token = i * kBlock;
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

    f32x4 s[RT][2];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) s[rt][0] = s[rt][1] = f32x4{};
#pragma unroll
    for (int c = 0; c < NC; ++c) {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        u32x4 a;
        if constexpr (FP8) a = widen<DT>(k[t][c / 2][2 * (c % 2)], k[t][c / 2][2 * (c % 2) + 1]);
        else a = k[t][c];
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][t] = T::mfma(a, qf[rt][c], s[rt][t]);
      }
    }
    if (more) load_k(o0, o1);

    const bool edge = token + kBlock > len;
    u32x4 pf[RT], rest[RT];   // the weights, and what rounding them left
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      float x[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) x[j] = s[rt][j / 4][j % 4] * p.c;
      if (edge) {
#pragma unroll
        for (int j = 0; j < 8; ++j)
          if (token + 16 * (j / 4) + 4 * g + j % 4 >= len) x[j] = -INFINITY;
      }
      float top = fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])),
                        fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
      top = fmaxf(m[rt], max_over_groups(top));
      if (__any(top > m[rt])) {
        const float alpha = __builtin_amdgcn_exp2f(m[rt] - top);
        l[rt] *= alpha;
#pragma unroll
        for (int t = 0; t < CV; ++t) acc[rt][t] *= alpha;
        m[rt] = top;
      }
      float e[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        e[j] = __builtin_amdgcn_exp2f(x[j] - m[rt]);
        l[rt] += e[j];
      }
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float e0 = e[2 * w] * kWeight<DT>, e1 = e[2 * w + 1] * kWeight<DT>;
        pf[rt][w] = T::pack(e0, e1);
        const f32x2 near = T::unpack(pf[rt][w]);
        rest[rt][w] = T::pack(e0 - near[0], e1 - near[1]);
      }
    }

    if (edge) {
#pragma unroll
      for (int j = 0; j < 8; ++j)
        if (token + 16 * (j / 4) + 4 * g + j % 4 >= len) v[j] = VRaw{};
    }
    // each row's columns as pairs of 16-bit values
    uint32_t cols[8][CV / 2];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if constexpr (!FP8) {
#pragma unroll
        for (int w = 0; w < CV / 2; ++w) cols[j][w] = v[j][w];
      } else if constexpr (CV == 8) {
        const u32x4 r = widen<DT>(v[j][0], v[j][1]);
#pragma unroll
        for (int w = 0; w < 4; ++w) cols[j][w] = r[w];
      } else {
        const u32x4 r = widen<DT>(v[j], 0);
        cols[j][0] = r[0], cols[j][1] = r[1];
      }
    }
#pragma unroll
    for (int t = 0; t < CV; ++t) {
      u32x4 a;
#pragma unroll
      for (int w = 0; w < 4; ++w)
        a[w] = __builtin_amdgcn_perm(cols[2 * w + 1][t / 2], cols[2 * w][t / 2],
                                     t % 2 ? 0x07060302u : 0x05040100u);
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        acc[rt][t] = T::mfma(a, pf[rt], acc[rt][t]);
        acc[rt][t] = T::mfma(a, rest[rt], acc[rt][t]);
      }
    }
    if (more) load_v(o0, o1);
  }

  // ---- join the wavefronts, as in piece ----
  constexpr int HALF = WAVES / 2, R = 16 * RT;
  float* const ml = lds;                        // [WAVES][R][2]
  float* const part = lds + WAVES * R * 2;      // [HALF][R][D]
  const bool any_bad = __any(bad);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] = sum_over_groups(l[rt]);
    if (any_bad) l[rt] = __builtin_nanf("");   // a page out of range
    if (g == 0) *reinterpret_cast<f32x2*>(ml + (wave * R + rt * 16 + n) * 2) = f32x2{m[rt], l[rt]};
  }
  __syncthreads();
  float weight[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    float top = -FLT_MAX;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) top = fmaxf(top, ml[(w * R + rt * 16 + n) * 2]);
    weight[rt] = __builtin_amdgcn_exp2f(m[rt] - top);
  }
#pragma unroll
  for (int phase = 0; phase < 2; ++phase) {
    if (wave / HALF == phase) {
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        // columns (4 g + r) CV .. + CV - 1 of row n
        float* const mine = part + ((wave % HALF) * R + rt * 16 + n) * D + 4 * g * CV;
#pragma unroll
        for (int r = 0; r < 4; ++r) {
#pragma unroll
          for (int t = 0; t < CV; t += 4) {
            f32x4* dst = reinterpret_cast<f32x4*>(mine + r * CV + t);
            f32x4 x = f32x4{acc[rt][t][r], acc[rt][t + 1][r], acc[rt][t + 2][r], acc[rt][t + 3][r]} * weight[rt];
            if (phase) x += *dst;
            *dst = x;
          }
        }
      }
    }
    __syncthreads();
  }
  for (int e4 = threadIdx.x; e4 < R * (D / 4); e4 += 64 * WAVES) {
    const int r = e4 / (D / 4), col = e4 % (D / 4) * 4;
    f32x4 sum = f32x4{};
#pragma unroll
    for (int w = 0; w < HALF; ++w) sum += *reinterpret_cast<const f32x4*>(part + (w * R + r) * D + col);
    float mr = -FLT_MAX, lr = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) mr = fmaxf(mr, ml[(w * R + r) * 2]);
#pragma unroll
    for (int w = 0; w < WAVES; ++w)
      lr += ml[(w * R + r) * 2 + 1] * __builtin_amdgcn_exp2f(ml[(w * R + r) * 2] - mr);
    const size_t slot = ((((size_t)hkv * sp.tiles + tile) * RT + r / 16) * sp.splits + split) * 16 + r % 16;
    *reinterpret_cast<f32x4*>(sp.prefix_o + slot * D + col) = sum;
    if (col == 0) *reinterpret_cast<f32x2*>(sp.prefix_ml + slot * 2) = f32x2{mr, lr};
  }
}

// A block of keys or values in LDS: 32 rows of D 16-bit values, whose 16-byte units are
// turned about within each row so that what an operand's read takes lies in distinct banks:
// of keys one unit of each of 16 rows, of values two neighbouring units of each of 8 rows.
template <int D>
struct Tile {
  static constexpr int U = D / 8;   // units of a row
  static constexpr int kBytes = kBlock * D * 2;
  static __device__ __forceinline__ int key_turn(int row) { return U == 16 ? row & 15 : row >> 1 & 7; }
  static __device__ __forceinline__ int value_turn(int row) { return U == 16 ? 2 * (row & 7) : 2 * (row >> 1 & 3); }
};

// s_waitcnt immediate for vmcnt(n) alone: all but the last n memory operations have ended.
constexpr int wait_vm(int n) { return 0x0f70 | (n & 15) | ((n >> 4) << 14); }

// 16 bytes a lane from base + from straight into LDS, lane l's to `to` + 16 l.  Inline
// assembly, so that the compiler does not wait for all such loads before each LDS read; the
// waits are the explicit ones.  M0 holds `to`, and needs one wait state before the load.
__device__ __forceinline__ void load_to_lds(const uint8_t* base, uint32_t from, uint8_t* to) {
  const uint32_t m0 = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)to;
  asm volatile("s_nop 0\n\tglobal_load_lds_dwordx4 %0, %2" ::"v"(from), "{m0}"(m0), "s"(base) : "memory");
}

// A part of the prefix for one tile of 128 rows, 32 a wavefront: the wavefronts walk its
// blocks together through rings in LDS of three blocks of keys and three of values,
// whose loads go out two steps before they are read: from memory straight into LDS, or, of
// E4M3 codes, through registers, where they are widened.
template <int DT, int D, bool FP8>
__device__ __forceinline__ void prefix_block_rows(const SharedParams& sp, float* lds, int hkv, int tile, int split,
                                                  int lo, int hi) {
  using T = Type16<DT>;
  using L = Tile<D>;
  constexpr int RT = 2, NC = D / 32, CV = D / 16, U = L::U;
  constexpr int ES = FP8 ? 1 : 2;
  constexpr int NS = U / 8;             // units of a block of keys or values that a thread fetches
  const Params& p = sp.own;
  const int lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int len = p.prefix;
  bool bad = false;
  uint8_t* const keys = reinterpret_cast<uint8_t*>(lds);   // [3]
  uint8_t* const values = keys + 3 * L::kBytes;            // [3]

  const int tile0 = (tile * 4 + wave) * RT;   // the wavefront's first 16 rows
  const bool live = tile0 * 16 < sp.rows;
  const float c = fabsf(p.c);
  const uint32_t sign = p.c < 0.f ? 0x80008000u : 0u;   // of the scale, taken into q
  u32x4 qf[RT][NC];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int row = (tile0 + rt) * 16 + n;
#pragma unroll
    for (int i = 0; i < NC; ++i) qf[rt][i] = u32x4{};
    if (row < sp.rows) {
      const int b = row / p.group;
      const uint16_t* q = p.q + ((size_t)b * p.H + hkv * p.group + (row - b * p.group)) * D;
#pragma unroll
      for (int i = 0; i < NC; ++i) {
        qf[rt][i] = *reinterpret_cast<const u32x4*>(q + i * 32 + g * 8);
#pragma unroll
        for (int w = 0; w < 4; ++w) qf[rt][i][w] ^= sign;
      }
    }
  }

  // Offsets of the tiles of the next 32 blocks, as in prefix_piece (every wavefront all).
  int off_lo = 0, off_hi = 0;
  auto look_up = [&](int i0) __attribute__((always_inline)) {
    const int li = i0 + (lane >> 1);
    int64_t off = 0;
    if (li < hi) {
      int token = li * kBlock + 16 * (lane & 1);
      if (token >= len) token ^= 16;
      const uint32_t at = p.page.div((uint32_t)token);
      const int page = sp.prefix_table[at];
      if (page >= 0 && page < p.num_pages)
        off = page * p.page_stride + (int64_t)((uint32_t)token - at * p.page.d) * p.token_stride;
      else
        bad = true;
    }
    off_lo = (int)(uint32_t)off;
    off_hi = (int)(off >> 32);
  };
  struct Place { int64_t o0, o1; };   // of a block's two tiles
  auto place_of = [&](int i) __attribute__((always_inline)) {   // (in order, each once)
    const int nth = (i - lo) & 31;
    if (nth == 0) look_up(i);
    auto of = [&](int l) __attribute__((always_inline)) {
      return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane(off_hi, l) << 32 |
                       (uint32_t)__builtin_amdgcn_readlane(off_lo, l));
    };
    return Place{of(2 * nth), of(2 * nth + 1)};
  };

  // This thread's units: of LDS (16-bit), unit `col` of row `row` (and 16 rows on); what it
  // brings there is turned about at the source.  Of E4M3 codes it fetches unit `col`, and
  // puts it where the turn says.
  const int row = threadIdx.x / U, col = threadIdx.x % U;
  const int k_turned = col ^ L::key_turn(row), v_turned = col ^ L::value_turn(row);
  const uint32_t k_from = (row & 15) * p.token_stride + (FP8 ? col : k_turned) * 8 * ES;
  const uint32_t v_from = (row & 15) * p.token_stride + (FP8 ? col : v_turned) * 8 * ES;
  const uint8_t* const kh = p.k + (size_t)hkv * p.head_stride;
  const uint8_t* const vh = p.v + (size_t)hkv * p.head_stride;
  auto tile_of = [&](const Place& at, int j) __attribute__((always_inline)) {
    return NS == 2 ? (j ? at.o1 : at.o0) : (wave < 2 ? at.o0 : at.o1);
  };
  auto load = [&](const uint8_t* head, const Place& at, uint32_t from, uint8_t* to) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NS; ++j) load_to_lds(head + tile_of(at, j), from, to + (wave * 64 + 256 * j) * 16);
  };
  struct Codes { u32x2 u[NS]; };
  auto fetch = [&](const uint8_t* head, const Place& at, uint32_t from) __attribute__((always_inline)) {
    Codes x;
#pragma unroll
    for (int j = 0; j < NS; ++j) x.u[j] = *reinterpret_cast<const u32x2*>(head + tile_of(at, j) + from);
    return x;
  };
  auto put = [&](const Codes& x, uint8_t* to, int turned) __attribute__((always_inline)) {
#pragma unroll
    for (int j = 0; j < NS; ++j)
      *reinterpret_cast<u32x4*>(to + ((row + 16 * j) * U + turned) * 16) = widen<DT>(x.u[j][0], x.u[j][1]);
  };

  f32x4 acc[RT][CV];
  float m[RT], l[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m[rt] = -FLT_MAX, l[rt] = 0.f;
#pragma unroll
    for (int t = 0; t < CV; ++t) acc[rt][t] = f32x4{};
  }

  // this lane's operands in a block: of k-step 0 and M tile 0, others a turn of the units on
  const uint32_t k_at = (n * U + (g ^ L::key_turn(n))) * 16;
  const int v_row = 4 * g + (n >> 2);   // of the transposing read
  const uint32_t v_at = (v_row * U + ((n >> 1 & 1) ^ L::value_turn(v_row))) * 16 + (n & 1) * 8;
  typedef short i16x4 __attribute__((ext_vector_type(4)));
  typedef __attribute__((address_space(3))) i16x4 lds_i16x4;
  typedef __attribute__((address_space(3))) u32x4 lds_u32x4;
  const uint32_t keys_at = (uint32_t)(uintptr_t)(__attribute__((address_space(3))) void*)keys;
  const uint32_t values_at = keys_at + 3 * L::kBytes;

  // In step i the scores of block i + 1 and the second product of block i - 1 are formed,
  // on the matrix cores, beside the weights of block i: nothing of one waits for another.
  struct Weights { u32x4 near[RT], rest[RT]; };   // rounded, and what rounding them left
  struct Scores { f32x4 x[RT][2]; };
  auto scores = [&](Scores& to, int slot) __attribute__((always_inline)) {
    auto& s = to.x;
    const uint32_t base = keys_at + slot * L::kBytes;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) s[rt][0] = s[rt][1] = f32x4{};
#pragma unroll
    for (int x = 0; x < NC; ++x) {
      const uint32_t at = (k_at ^ 64 * x) + base;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const u32x4 a = *reinterpret_cast<lds_u32x4*>(at + t * 16 * U * 16);
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[rt][t] = T::mfma(a, qf[rt][x], s[rt][t]);
      }
    }
  };
  // (two M tiles at a time: a sum's next product is four instructions on)
  auto second = [&](const Weights& w, int slot) __attribute__((always_inline)) {
    const uint32_t base = values_at + slot * L::kBytes;
#pragma unroll
    for (int t = 0; t < CV; t += 2) {
      u32x4 a[2];
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const uint32_t at = (v_at ^ 32 * (t + y)) + base;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const u32x2 x = __builtin_bit_cast(u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16(
              reinterpret_cast<lds_i16x4*>(at + h * 16 * U * 16)));
          a[y][2 * h] = x[0], a[y][2 * h + 1] = x[1];
        }
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        acc[rt][t] = T::mfma(a[0], w.near[rt], acc[rt][t]);
        acc[rt][t + 1] = T::mfma(a[1], w.near[rt], acc[rt][t + 1]);
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        acc[rt][t] = T::mfma(a[0], w.rest[rt], acc[rt][t]);
        acc[rt][t + 1] = T::mfma(a[1], w.rest[rt], acc[rt][t + 1]);
      }
    }
  };

  // Block j of either ring lies in slot (j - lo) % 3.
  Place p1 = {}, p2 = {};   // of blocks i + 1 and i + 2
  Codes ku = {}, vu = {};   // E4M3: the keys of block i + 2 and the values of block i, on their way
  int slot = 0;             // of block i
  auto after = [](int slot, int by) __attribute__((always_inline)) { return slot + by < 3 ? slot + by : slot + by - 3; };
  const int last = hi - 1;

  uint32_t low = 0x0000bf80u, high = 0xbf800000u;   // see minus_halves
  asm("" : "+s"(low), "+s"(high));
  // A tile's weights against m, and the sum of this lane's.  The scaled score is rounded before m
  // is subtracted, as it was when m was taken: of scores past 2^24 a fused difference could
  // be far above 0.
  auto weigh = [&](const Scores& s, int rt, bool edge, int i, u32x4& near, u32x4& rest) __attribute__((always_inline)) {
#pragma clang fp contract(off)
    float e[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const float x = s.x[rt][j / 4][j % 4] * c;
      e[j] = __builtin_amdgcn_exp2f(x - m[rt]);
      if (edge && i * kBlock + 16 * (j / 4) + 4 * g + j % 4 >= len) e[j] = 0.f;
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float e0 = e[2 * w] * kFactor<DT>, e1 = e[2 * w + 1] * kFactor<DT>;
      near[w] = T::pack(e0, e1);
      const f32x2 left = minus_halves<DT>(e0, e1, near[w], low, high);
      rest[w] = T::pack(left[0], left[1]);
    }
    return ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
  };

  // Block i: from its scores to its weights, from block i - 1's weights to its second product,
  // and block i + 1's scores.  EDGE: it may end past the prefix (and is the last).
  auto step = [&](int i, auto edge, const Scores& s, const Weights& w, Scores& s1, Weights& w1) __attribute__((always_inline)) {
    constexpr bool EDGE = decltype(edge)::value;
    // keys of block i + 3 take the place of block i's, whose scores were formed a step ago, and
    // values of block i + 1 that of block i - 2's; past the last block, one again that is not read
    Place p3 = p2;
    if (i + 3 <= last) p3 = place_of(i + 3);
    Codes k1, v1;
    if constexpr (FP8) {
      k1 = fetch(kh, p3, k_from), v1 = fetch(vh, p1, v_from);
    } else {
      load(kh, p3, k_from, keys + slot * L::kBytes);
      load(vh, p1, v_from, values + after(slot, 1) * L::kBytes);
    }
    if (kDebugSync) {
      __builtin_amdgcn_s_waitcnt(wait_vm(0));
      __syncthreads();
    }
    if (live) {
      if (!EDGE) scores(s1, after(slot, 1));   // (of nothing after the last block)
      second(w, after(slot, 2));
      float sum[RT];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) sum[rt] = weigh(s, rt, EDGE, i, w1.near[rt], w1.rest[rt]);
      if (__any(fmaxf(sum[0], sum[1]) > kMostWeight<DT>)) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          float top = -FLT_MAX;
#pragma unroll
          for (int j = 0; j < 8; ++j)
            if (!EDGE || i * kBlock + 16 * (j / 4) + 4 * g + j % 4 < len) top = fmaxf(top, s.x[rt][j / 4][j % 4] * c);
          // (of the row's four lanes, by any; a row that is not redone keeps m, and its weights come
          // out as they were.  That is hidden from the compiler, which else branches by row.)
          top = max_over_groups(sum[rt]) > kMostWeight<DT> ? fmaxf(m[rt], max_over_groups(top)) : m[rt];
          asm("" : "+v"(top));
          const float alpha = __builtin_amdgcn_exp2f(m[rt] - top);
          l[rt] *= alpha;
#pragma unroll
          for (int t = 0; t < CV; ++t) acc[rt][t] *= alpha;
          m[rt] = top;
          sum[rt] = weigh(s, rt, EDGE, i, w1.near[rt], w1.rest[rt]);
        }
      }
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) l[rt] += sum[rt];
    }
    if constexpr (FP8) {
      put(ku, keys + after(slot, 2) * L::kBytes, k_turned);
      put(vu, values + slot * L::kBytes, v_turned);
      ku = k1, vu = v1;
    } else {
      __builtin_amdgcn_s_waitcnt(wait_vm(2 * NS));   // all but this step's loads have landed
    }
    __syncthreads();
    p1 = p2, p2 = p3;
    slot = after(slot, 1);
  };

  if (lo < hi) {
    const Place p0 = place_of(lo);
    p1 = lo + 1 <= last ? place_of(lo + 1) : p0;
    p2 = lo + 2 <= last ? place_of(lo + 2) : p1;
    if constexpr (FP8) {
      const Codes k0 = fetch(kh, p0, k_from), k1 = fetch(kh, p1, k_from);
      ku = fetch(kh, p2, k_from), vu = fetch(vh, p0, v_from);
      put(k0, keys, k_turned);
      put(k1, keys + L::kBytes, k_turned);
    } else {
      load(kh, p0, k_from, keys);
      load(kh, p1, k_from, keys + L::kBytes);
      load(kh, p2, k_from, keys + 2 * L::kBytes);
      load(vh, p0, v_from, values);
    }
  }
  // what stands for the values of the block before the first meets weights of 0
#pragma unroll
  for (int j = 0; j < NS; ++j)
    *reinterpret_cast<u32x4*>(values + 2 * L::kBytes + (threadIdx.x + 256 * j) * 16) = u32x4{};
  if (!FP8) __builtin_amdgcn_s_waitcnt(wait_vm(0));
  __syncthreads();
  if (lo < hi) {
    Scores s, s1;
    Weights w, w1;
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) w.near[rt] = w.rest[rt] = u32x4{};
    if (live) scores(s, 0);
    __syncthreads();
    const int whole = hi * kBlock > len ? last : hi;   // blocks of visible keys alone
    int i = lo;
    for (; i + 1 < whole; i += 2) {
      step(i, std::false_type{}, s, w, s1, w1);
      step(i + 1, std::false_type{}, s1, w1, s, w);
    }
    if (i < whole) {
      step(i, std::false_type{}, s, w, s1, w1);
      s = s1, w = w1;
      ++i;
    }
    if (i < hi) {
      step(i, std::true_type{}, s, w, s1, w1);
      w = w1;
      // values past the prefix: 0, as their weights are, whatever their memory holds
      const int at = after(slot, 2);
#pragma unroll
      for (int j = 0; j < NS; ++j)
        if (last * kBlock + row + 16 * j >= len)
          *reinterpret_cast<u32x4*>(values + at * L::kBytes + ((row + 16 * j) * U + col) * 16) = u32x4{};
      __syncthreads();
    }
    if (live) second(w, after(slot, 2));
  }
  if (!FP8) __builtin_amdgcn_s_waitcnt(wait_vm(0));   // no load is on its way into LDS when the workgroup ends

  const bool any_bad = __any(bad);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    l[rt] = sum_over_groups(l[rt]);
    if (any_bad) l[rt] = __builtin_nanf("");   // a page out of range
    const size_t slot = (((size_t)hkv * sp.tiles * 8 + tile0 + rt) * sp.splits + split) * 16 + n;
    // columns 16 t + 4 g .. + 3 of row n
#pragma unroll
    for (int t = 0; t < CV; ++t)
      *reinterpret_cast<f32x4*>(sp.prefix_o + slot * D + 16 * t + 4 * g) = acc[rt][t] * (kWeight<DT> / kFactor<DT>);
    if (g == 0) *reinterpret_cast<f32x2*>(sp.prefix_ml + slot * 2) = f32x2{m[rt], l[rt]};
  }
}

// RT: 16-row tiles of a workgroup's rows.
template <int DT, int D, bool FP8, int RT>
__global__ __launch_bounds__(256, 2) void shared_parts_kernel(SharedParams p) {
  constexpr int WAVES = 4;
  constexpr int kJoin = WAVES * 16 * RT * 2 + WAVES / 2 * 16 * RT * D, kRings = 6 * Tile<D>::kBytes / 4;
  __shared__ __attribute__((aligned(16))) float lds[RT == 8 ? kRings : kJoin];
  if ((int)blockIdx.x >= p.prefix_grid) {
    share_of<DT, D, FP8, true>(p.own, lds, blockIdx.x - p.prefix_grid, p.own.grid);
    return;
  }
  // workgroups of one XCD (every eighth) take the tiles of one head's part in turn
  const int at = blockIdx.x / 8;
  const int unit = at / p.tiles * 8 + blockIdx.x % 8, tile = at % p.tiles;
  if (unit >= p.own.Hkv * p.splits) return;
  const int hkv = unit / p.splits, split = unit - hkv * p.splits;
  const int lo = (int)((int64_t)p.blocks * split / p.splits), hi = (int)((int64_t)p.blocks * (split + 1) / p.splits);
  if constexpr (RT == 8) prefix_block_rows<DT, D, FP8>(p, lds, hkv, tile, split, lo, hi);
  else prefix_piece<DT, D, FP8, RT, WAVES>(p, lds, hkv, tile, split, lo, hi);
}

// Joins the parts of each (sequence, head), in a fixed order.  T threads a head: 64, or 256
// where heads are few (shared_rules.h).  The prefix's, which need no length, are on their
// way before the length and the number of the sequence's own parts are known.
template <int DT, int D, int RT, int T>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedParams sp, int heads) {
  constexpr int L = D / 4;     // threads of a part, 4 columns each
  constexpr int G = T / L;     // parts side by side
  constexpr int kAhead = 4;    // parts that a thread fetches at once
  __shared__ __attribute__((aligned(16))) float lds[256 / T][G][D + 4];
  const Params& p = sp.own;
  const int own_head = T == 256 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  const int id = blockIdx.x * (256 / T) + own_head;
  if (id >= heads) return;
  const int b = id / p.H, h = id - b * p.H;
  const int thread = threadIdx.x % T, col = thread % L * 4, own = thread / L;
  const int hkv = h / p.group, in_group = h - hkv * p.group, row = b * p.group + in_group;
  const size_t before = (((size_t)hkv * sp.tiles * RT + row / 16) * sp.splits) * 16 + row % 16;
  const int len = p.lengths[b];

  float m = -FLT_MAX, l = 0.f;
  f32x4 o = f32x4{};
  auto add = [&](f32x2 ml, f32x4 x) __attribute__((always_inline)) {
    const float top = fmaxf(m, ml[0]);
    const float a = __builtin_amdgcn_exp2f(m - top), w = __builtin_amdgcn_exp2f(ml[0] - top);
    o = o * a + x * w;
    l = l * a + ml[1] * w;
    m = top;
  };
  int j = own;
  for (; j + (kAhead - 1) * G < sp.splits; j += kAhead * G) {
    f32x2 ml[kAhead];
    f32x4 x[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const size_t at = before + (size_t)(j + i * G) * 16;
      ml[i] = *reinterpret_cast<const f32x2*>(sp.prefix_ml + at * 2);
      x[i] = *reinterpret_cast<const f32x4*>(sp.prefix_o + at * D + col);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) add(ml[i], x[i]);
  }
  for (; j < sp.splits; j += G) {
    const size_t at = before + (size_t)j * 16;
    add(*reinterpret_cast<const f32x2*>(sp.prefix_ml + at * 2), *reinterpret_cast<const f32x4*>(sp.prefix_o + at * D + col));
  }
  if (len < p.prefix || len > p.limit) {
    if (own == 0) finish<DT>(p, id, D, col, f32x4{}, -FLT_MAX, len == 0 ? 0.f : __builtin_nanf(""));
    return;
  }
  if (len > p.prefix) {
    const size_t at_row = ((size_t)b * p.Hkv + hkv) * p.tiles + in_group / 16;
    const int32_t* d = p.desc + 2 * at_row;
    // (bounded by the partial results there are, as lengths could change under the call)
    const int first = d[0], pieces = first >= 0 && first < p.grid ? min(d[1], p.grid - first) : 0;
#pragma unroll 2
    for (int i = own; i < pieces; i += G) {
      const size_t slot = pieces == 1 ? 2 * (size_t)p.grid + at_row : (size_t)(i ? 2 * (first + i) : 2 * first + 1);
      const size_t at = slot * 16 + in_group % 16;
      add(*reinterpret_cast<const f32x2*>(p.part_ml + at * 2), *reinterpret_cast<const f32x4*>(p.part_o + at * D + col));
    }
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
  float top = -FLT_MAX;
#pragma unroll
  for (int i = 0; i < G; ++i) top = fmaxf(top, lds[own_head][i][D]);
  f32x4 sum = f32x4{};
  float total = 0.f;
#pragma unroll
  for (int i = 0; i < G; ++i) {   // (those without a part have l = 0 and o = 0)
    const float* x = lds[own_head][i];
    const float w = __builtin_amdgcn_exp2f(x[D] - top);
    total += w * x[D + 1];
    sum += *reinterpret_cast<const f32x4*>(x + col) * w;
  }
  finish<DT>(p, id, D, col, sum, top, total);
}

template <int DT, int D, int RT>
hipError_t launch_rows(const SharedArgs& a, const SharedPlan& plan, const SharedParams& p, hipStream_t stream) {
  const dim3 grid(plan.prefix_grid + plan.own_grid);
  if (a.decode.cache.fp8)
    hipLaunchKernelGGL((shared_parts_kernel<DT, D, true, RT>), grid, dim3(256), 0, stream, p);
  else
    hipLaunchKernelGGL((shared_parts_kernel<DT, D, false, RT>), grid, dim3(256), 0, stream, p);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int heads = a.decode.B * a.decode.H;
  if (plan.join_threads == 256)
    hipLaunchKernelGGL((shared_join_kernel<DT, D, RT, 256>), dim3(heads), dim3(256), 0, stream, p, heads);
  else
    hipLaunchKernelGGL((shared_join_kernel<DT, D, RT, 64>), dim3((heads + 3) / 4), dim3(256), 0, stream, p, heads);
  return hipGetLastError();
}

template <int DT, int D>
hipError_t launch_width(const SharedArgs& s, const SharedPlan& plan, hipStream_t stream) {
  const DecodeArgs& a = s.decode;
  SharedParams p = {};
  const size_t slots = (size_t)a.Hkv * plan.tiles * plan.rt * plan.splits * 16;
  p.prefix_o = a.workspace;
  p.prefix_ml = p.prefix_o + slots * a.d;
  p.own = params_of(a, plan.own_grid, own_slots(plan, a.B, a.H, a.Hkv), p.prefix_ml + slots * 2);
  p.own.prefix = s.prefix;
  p.prefix_table = s.prefix_table;
  p.rows = a.B * p.own.group;
  p.tiles = plan.tiles;
  p.splits = plan.splits;
  p.blocks = (s.prefix + kBlock - 1) / kBlock;
  p.prefix_grid = plan.prefix_grid;
  return plan.rt == 1   ? launch_rows<DT, D, 1>(s, plan, p, stream)
         : plan.rt == 2 ? launch_rows<DT, D, 2>(s, plan, p, stream)
                        : launch_rows<DT, D, 8>(s, plan, p, stream);
}

}  // namespace

hipError_t launch_shared(const SharedArgs& a, const SharedPlan& plan, hipStream_t stream) {
  if (a.decode.d == 64)
    return a.decode.dtype == 0 ? launch_width<0, 64>(a, plan, stream) : launch_width<1, 64>(a, plan, stream);
  return a.decode.dtype == 0 ? launch_width<0, 128>(a, plan, stream) : launch_width<1, 128>(a, plan, stream);
}

}  // namespace qm
