// Attention of one new token per sequence over a paged cache whose first tokens, the
// prefix, are the same pages for all sequences.
//
// With m, l, O the maximum, sum and unnormalised result of a part of the keys, softmax over
// prefix and own tokens is their join: m = max, l = sum l_i e^(m_i - m), O alike.
//
// Prefix: the queries of all sequences that read a key/value head are the rows of one
// product, B H / Hkv of them, so each key and value is read once for 32 rows (16 where there
// are no more) and not once a sequence.  Bound: HBM where rows are few; from some 150 rows
// a head the matrix cores, 4 d flops a row and key against 4 d bytes a key.
// A wavefront walks 32-token blocks as in decode.hip, with 16-row tiles of queries in the
// place of 16 heads: each operand of K and V, read once, meets two tiles.  A workgroup's
// wavefronts take the blocks of its part in turn and join; every part leaves m, l and O
// in the workspace.  All tokens of the prefix are visible to all rows, so only its last block
// has hidden keys.
// Own tokens: equal shares of all sequences' blocks as in decode.hip, from the prefix on,
// by further workgroups of the same launch; then one kernel joins all parts in order.
#include "decode_device.h"
#include "shared_rules.h"

namespace qm {
namespace {

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

template <int DT, int D, bool FP8, int RT>
__global__ __launch_bounds__(256, 2) void shared_parts_kernel(SharedParams p) {
  constexpr int WAVES = 4;
  __shared__ __attribute__((aligned(16))) float lds[WAVES * 16 * RT * 2 + WAVES / 2 * 16 * RT * D];
  if ((int)blockIdx.x >= p.prefix_grid) {
    share_of<DT, D, FP8, true>(p.own, lds, blockIdx.x - p.prefix_grid, p.own.grid);
    return;
  }
  // workgroups of one XCD (every eighth) take the tiles of one head's part in turn
  const int at = blockIdx.x / 8;
  const int unit = at / p.tiles * 8 + blockIdx.x % 8, tile = at % p.tiles;
  if (unit >= p.own.Hkv * p.splits) return;
  const int hkv = unit / p.splits, split = unit - hkv * p.splits;
  prefix_piece<DT, D, FP8, RT, WAVES>(p, lds, hkv, tile, split, (int)((int64_t)p.blocks * split / p.splits),
                                      (int)((int64_t)p.blocks * (split + 1) / p.splits));
}

// Joins the parts of each (sequence, head), the prefix's first, in a fixed order.
template <int DT, int D, int RT>
__global__ __launch_bounds__(256) void shared_join_kernel(SharedParams sp) {
  constexpr int L = D / 4;     // threads of a part, 4 columns each
  constexpr int G = 256 / L;   // parts side by side
  __shared__ __attribute__((aligned(16))) float lds[G][D + 4];
  const Params& p = sp.own;
  const int id = blockIdx.x, b = id / p.H, h = id - b * p.H;
  const int len = p.lengths[b];
  const int col = threadIdx.x % L * 4, own = threadIdx.x / L;
  if (len < p.prefix || len > p.limit) {
    if (own == 0) finish<DT>(p, id, D, col, f32x4{}, -FLT_MAX, len == 0 ? 0.f : __builtin_nanf(""));
    return;
  }
  const int hkv = h / p.group, in_group = h - hkv * p.group, row = b * p.group + in_group;
  const size_t before = (((size_t)hkv * sp.tiles * RT + row / 16) * sp.splits) * 16 + row % 16;
  int first = 0, pieces = 0, row_slot = 0;
  if (len > p.prefix) {
    const int32_t* d = p.desc + 2 * (((size_t)b * p.Hkv + hkv) * p.tiles + in_group / 16);
    // (bounded by the partial results there are, as lengths could change under the call)
    first = d[0], pieces = first >= 0 && first < p.grid ? min(d[1], p.grid - first) : 0;
    row_slot = 2 * p.grid + (b * p.Hkv + hkv) * p.tiles + in_group / 16;
  }
  float m = -FLT_MAX, l = 0.f;
  f32x4 o = f32x4{};
#pragma unroll 4
  for (int j = own; j < sp.splits + pieces; j += G) {
    const int i = j - sp.splits;
    const float *xo, *xml;
    if (i < 0) {
      const size_t at = before + (size_t)j * 16;
      xo = sp.prefix_o + at * D, xml = sp.prefix_ml + at * 2;
    } else {
      const int slot = pieces == 1 ? row_slot : i ? 2 * (first + i) : 2 * first + 1;
      const size_t at = (size_t)slot * 16 + in_group % 16;
      xo = p.part_o + at * D, xml = p.part_ml + at * 2;
    }
    const f32x2 ml = *reinterpret_cast<const f32x2*>(xml);
    const f32x4 x = *reinterpret_cast<const f32x4*>(xo + col);
    const float top = fmaxf(m, ml[0]);
    const float a = __builtin_amdgcn_exp2f(m - top), w = __builtin_amdgcn_exp2f(ml[0] - top);
    o = o * a + x * w;
    l = l * a + ml[1] * w;
    m = top;
  }
  float* mine = lds[own];
  *reinterpret_cast<f32x4*>(mine + col) = o;
  if (col == 0) mine[D] = m, mine[D + 1] = l;
  __syncthreads();
  if (own) return;
  const int n = min(G, sp.splits + pieces);
  float top = -FLT_MAX;
  for (int i = 0; i < n; ++i) top = fmaxf(top, lds[i][D]);
  f32x4 sum = f32x4{};
  float total = 0.f;
  for (int i = 0; i < n; ++i) {
    const float* x = lds[i];
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
  hipLaunchKernelGGL((shared_join_kernel<DT, D, RT>), dim3(a.decode.B * a.decode.H), dim3(256), 0, stream, p);
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
  return plan.rt == 1 ? launch_rows<DT, D, 1>(s, plan, p, stream) : launch_rows<DT, D, 2>(s, plan, p, stream);
}

}  // namespace

hipError_t launch_shared(const SharedArgs& a, const SharedPlan& plan, hipStream_t stream) {
  if (a.decode.d == 64)
    return a.decode.dtype == 0 ? launch_width<0, 64>(a, plan, stream) : launch_width<1, 64>(a, plan, stream);
  return a.decode.dtype == 0 ? launch_width<0, 128>(a, plan, stream) : launch_width<1, 128>(a, plan, stream);
}

}  // namespace qm
