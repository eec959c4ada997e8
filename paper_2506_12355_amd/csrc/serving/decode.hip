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
#include "decode_device.h"

namespace qm {
namespace {

// One workgroup a row.
template <int DT, int D, bool FP8, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void decode_rows_kernel(Params p) {
  __shared__ __attribute__((aligned(16))) float lds[WAVES * 32 + WAVES / 2 * 16 * D];
  const int rows = p.Hkv * p.tiles;   // of a sequence
  const int b = blockIdx.x / rows;
  const int len = p.lengths[b];
  const bool bad = len < 0 || len > p.limit;
  const Blocks blocks(p, bad ? 0 : len);
  piece<DT, D, FP8, WAVES, false>(p, lds, b, blockIdx.x - b * rows, bad ? 0 : len, bad, blocks, 0, blocks.total, 0);
}

// Equal shares of all rows' blocks.
template <int DT, int D, bool FP8>
__global__ __launch_bounds__(256, 2) void decode_shares_kernel(Params p) {
  __shared__ __attribute__((aligned(16))) float lds[4 * 32 + 2 * 16 * D];
  share_of<DT, D, FP8, false>(p, lds, blockIdx.x, gridDim.x);
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
  Params p = params_of(a, plan.grid, (size_t)2 * plan.grid, a.workspace);
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
