// The residual's addition and the norm of whole rows in one pass, with a result in 16 bits
// or in E4M3 with scales.
//
//   s_c = x_c + r_c                                               (fp32; rounded into sum)
//   y_c = s_c w_c / sqrt(mean_c s_c^2 + eps)
//   E4M3: code_c = y_c / scale, scale = max(max |y| / 448, 2^-126) of a row or of a group
//   of columns, or given
//
// in fp32 from the stored values to one rounding into each result (y takes the unrounded s).
//
// Bound: memory; each element is read and written once.  A row belongs to T threads, each
// with V pieces of 8 columns that stay in registers from the one read to the last write: a
// part of a wavefront (T = 8 to 64, several rows a wavefront), or a workgroup.  One exchange:
// the sum of squares and, for a scale a row, max |s w|, which times 1 / sqrt(..) is max |y| to
// a rounding; rows whose products leave fp32's range, where y need not, take a second one, of
// y.  Maxima are taken of the values' bits without the sign, as whole numbers: a NaN is above
// every value there, where fmax would drop it.
//
// Measured (us, over more inputs than the last-level cache holds; a plain copy runs at 5.1 TB/s):
// 8192 rows of 8192 columns, bf16, with a residual 94 (5.7 TB/s), to E4M3 with a scale a row 84
// (5.6); 4097 of 5120, f16 to E4M3 in groups of 128 16.1 (4.0); one row of 4096 2.5, 64 of 8192 to
// E4M3 with a scale each 4.0: two latencies, of the row and of the sums.
#include "norm_rules.h"
#include "serving_device.h"
#include "serving_launch.h"

namespace qm {
namespace {

struct Params {
  const uint16_t *x, *residual, *weight;
  uint16_t* sum;
  void* out;
  float* scales;
  int64_t x_stride, residual_stride, sum_stride;   // elements from row to row
  int rows, width;
  float eps, inv_width;
  float inv;   // E4M3 with a given scale: its reciprocal; else 0
};

template <int T>
__device__ __forceinline__ float sum_over(float x) {
  return over_lanes<T>(x, [](float a, float b) { return a + b; });
}
template <int T>
__device__ __forceinline__ uint32_t max_over(uint32_t x) {
  return over_lanes<T>(x, [](uint32_t a, uint32_t b) { return a > b ? a : b; });
}
__device__ __forceinline__ uint32_t magnitude(float x) {
  return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu;
}

constexpr uint32_t kInfinite = 0x7f800000u, kLeastProduct = 0x0d800000u;   // bits of infinity and of 2^-100

// The scale of values up to m in magnitude: at least 2^-126, whose reciprocal is finite;
// NaN stays.
__device__ __forceinline__ float scale_of(float m) {
  const float s = m * (1.0f / 448.0f);
  return s < 0x1p-126f ? 0x1p-126f : s;
}

// GROUP: lanes of a scale's columns; 0: one a row, or the one given.
template <int DT, int T, int V, bool FP8, int GROUP>
__global__ __launch_bounds__(T < 256 ? 256 : T) void rms_norm_kernel(Params p) {
  using Ty = Type16<DT>;
  constexpr int kWaves = T / 64;
  const int lane = threadIdx.x % T;
  int row = T < 256 ? blockIdx.x * (256 / T) + threadIdx.x / T : blockIdx.x;
  const bool live = row < p.rows;   // (the last workgroup's further rows repeat the last one)
  row = live ? row : p.rows - 1;
  const int pieces = p.width / 8;

  float s[V][8];
  u32x4 w[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    const int at = j * T + lane;
    u32x4 x = u32x4{}, r = u32x4{};
    w[j] = u32x4{};
    if (at < pieces) {
      x = *reinterpret_cast<const u32x4*>(p.x + row * p.x_stride + 8 * at);
      if (p.residual) r = *reinterpret_cast<const u32x4*>(p.residual + row * p.residual_stride + 8 * at);
      if (p.weight) w[j] = *reinterpret_cast<const u32x4*>(p.weight + 8 * at);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 a = Ty::unpack(x[i]), b = Ty::unpack(r[i]);
      s[j][2 * i] = p.residual ? a[0] + b[0] : a[0];   // (-0 + 0 would lose the sign)
      s[j][2 * i + 1] = p.residual ? a[1] + b[1] : a[1];
    }
  }
  if (p.sum && live) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int at = j * T + lane;
      u32x4 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = Ty::pack(s[j][2 * i], s[j][2 * i + 1]);
      if (at < pieces) *reinterpret_cast<u32x4*>(p.sum + row * p.sum_stride + 8 * at) = o;
    }
  }

  float squares = 0.f;   // their mean: a sum could overflow where the mean does not
#pragma unroll
  for (int j = 0; j < V; ++j)
#pragma unroll
    for (int i = 0; i < 8; ++i) squares = fmaf(s[j][i] * p.inv_width, s[j][i], squares);
  uint32_t top = 0;   // of |s w|
  if (FP8 && GROUP == 0) {
#pragma unroll
    for (int j = 0; j < V; ++j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const f32x2 e = p.weight ? Ty::unpack(w[j][i]) : f32x2{1.f, 1.f};
        const uint32_t a = magnitude(s[j][2 * i] * e[0]), b = magnitude(s[j][2 * i + 1] * e[1]);
        const uint32_t ab = a > b ? a : b;
        top = top > ab ? top : ab;
      }
    }
  }
  squares = sum_over<(T < 64 ? T : 64)>(squares);
  if (FP8 && GROUP == 0) top = max_over<(T < 64 ? T : 64)>(top);
  __shared__ uint32_t tops[kWaves > 1 ? kWaves : 1];
  if constexpr (kWaves > 1) {
    __shared__ float parts[kWaves];
    if (threadIdx.x % 64 == 0) {
      parts[threadIdx.x / 64] = squares;
      if (FP8 && GROUP == 0) tops[threadIdx.x / 64] = top;
    }
    __syncthreads();
    squares = 0.f;
#pragma unroll
    for (int i = 0; i < kWaves; ++i) {
      squares += parts[i];
      if (FP8 && GROUP == 0) top = tops[i] > top ? tops[i] : top;
    }
  }
  const float r = 1.0f / sqrtf(squares + p.eps);
#pragma unroll
  for (int j = 0; j < V; ++j) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const f32x2 e = p.weight ? Ty::unpack(w[j][i]) : f32x2{1.f, 1.f};
      s[j][2 * i] *= r * e[0], s[j][2 * i + 1] *= r * e[1];
    }
  }

  if constexpr (!FP8) {
    if (!live) return;
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int at = j * T + lane;
      u32x4 o;
#pragma unroll
      for (int i = 0; i < 4; ++i) o[i] = Ty::pack(s[j][2 * i], s[j][2 * i + 1]);
      if (at < pieces)
        *reinterpret_cast<u32x4*>(static_cast<uint16_t*>(p.out) + (int64_t)row * p.width + 8 * at) = o;
    }
  } else {
    float scale = 1.f, inv = p.inv;
    if (GROUP == 0 && p.scales) {
      float most = __builtin_bit_cast(float, top) * r;
      // where the largest |s w| is past fp32's range, or so small that it lost bits, y need not be
      const bool lost = top - kLeastProduct >= kInfinite - kLeastProduct;
      if (__any(lost)) {   // (more than one wavefront: of all of them)
        uint32_t formed = 0;
#pragma unroll
        for (int j = 0; j < V; ++j)
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (j * T + lane < pieces && magnitude(s[j][i]) > formed) formed = magnitude(s[j][i]);
        formed = max_over<(T < 64 ? T : 64)>(formed);
        if constexpr (kWaves > 1) {
          __syncthreads();   // (tops has been read)
          if (threadIdx.x % 64 == 0) tops[threadIdx.x / 64] = formed;
          __syncthreads();
#pragma unroll
          for (int i = 0; i < kWaves; ++i) formed = tops[i] > formed ? tops[i] : formed;
        }
        if (lost) most = __builtin_bit_cast(float, formed);
      }
      scale = scale_of(most);
      if (live && lane == 0) p.scales[row] = scale;
      inv = 1.0f / scale;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int at = j * T + lane;
      if constexpr (GROUP > 0) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) m = magnitude(s[j][i]) > m ? magnitude(s[j][i]) : m;
        scale = scale_of(__builtin_bit_cast(float, max_over<GROUP>(m)));
        if (live && at < pieces && lane % GROUP == 0)
          p.scales[(int64_t)row * (pieces / GROUP) + at / GROUP] = scale;
        inv = 1.0f / scale;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s[j][i] *= inv;
      u32x2 codes;
      if (GROUP > 0 || p.scales) {
        // at most 448, to a rounding; NaN only where the scale is one, or infinite
#pragma unroll
        for (int i = 0; i < 8; ++i) s[j][i] = __builtin_amdgcn_fmed3f(s[j][i], -448.f, 448.f);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          int w = __builtin_amdgcn_cvt_pk_fp8_f32(s[j][4 * i], s[j][4 * i + 1], 0, false);
          w = __builtin_amdgcn_cvt_pk_fp8_f32(s[j][4 * i + 2], s[j][4 * i + 3], w, true);
          codes[i] = scale < INFINITY ? (uint32_t)w : 0x7f7f7f7fu;
        }
      } else {
        codes = u32x2{pack_fp8(s[j][0], s[j][1], s[j][2], s[j][3]), pack_fp8(s[j][4], s[j][5], s[j][6], s[j][7])};
      }
      if (live && at < pieces)
        *reinterpret_cast<u32x2*>(static_cast<uint8_t*>(p.out) + (int64_t)row * p.width + 8 * at) = codes;
    }
  }
}

template <int DT, int T, int V, bool FP8, int GROUP>
hipError_t launch(const Params& p, hipStream_t stream) {
  constexpr int kRows = T < 256 ? 256 / T : 1;
  Params part = p;
  for (int64_t first = 0; first < p.rows; first += rows_of_launch(T)) {
    const int64_t left = p.rows - first;
    part.rows = (int)(left < rows_of_launch(T) ? left : rows_of_launch(T));
    part.x = p.x + first * p.x_stride;
    if (p.residual) part.residual = p.residual + first * p.residual_stride;
    if (p.sum) part.sum = p.sum + first * p.sum_stride;
    part.out = static_cast<uint8_t*>(p.out) + first * p.width * (FP8 ? 1 : 2);
    if (p.scales) part.scales = p.scales + first * (GROUP ? p.width / (8 * GROUP) : 1);
    hipLaunchKernelGGL((rms_norm_kernel<DT, T, V, FP8, GROUP>), dim3((part.rows + kRows - 1) / kRows),
                       dim3(T < 256 ? 256 : T), 0, stream, part);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

// Threads and pieces of a row: four pieces at most, three where they hold it, from 256 threads
// on.  us, 4097 rows of 5120 columns to E4M3 in groups of 128: 256 threads and three pieces
// 16.0, and four 18.5, 128 and five 16.3, a wavefront with all 24.5; 4096 rows of 8192 with a
// residual: 256 threads and four pieces 41.2, 128 and eight 42.9, a wavefront with all 47.5.
template <int DT, bool FP8, int GROUP>
hipError_t launch_threads(const Params& p, hipStream_t stream) {
  const int pieces = p.width / 8;
  if constexpr (GROUP <= 8) {
    if (pieces <= 8) return launch<DT, 8, 1, FP8, GROUP>(p, stream);
  }
  if constexpr (GROUP <= 16) {
    if (pieces <= 16) return launch<DT, 16, 1, FP8, GROUP>(p, stream);
  }
  if (pieces <= 32) return launch<DT, 32, 1, FP8, GROUP>(p, stream);
  if (pieces <= 64) return launch<DT, 64, 1, FP8, GROUP>(p, stream);
  if (pieces <= 128) return launch<DT, 64, 2, FP8, GROUP>(p, stream);
  if (pieces <= 256) return launch<DT, 256, 1, FP8, GROUP>(p, stream);
  if (pieces <= 512) return launch<DT, 256, 2, FP8, GROUP>(p, stream);
  if (pieces <= 3 * 256) return launch<DT, 256, 3, FP8, GROUP>(p, stream);
  if (pieces <= 4 * 256) return launch<DT, 256, 4, FP8, GROUP>(p, stream);
  if (pieces <= 3 * 512) return launch<DT, 512, 3, FP8, GROUP>(p, stream);
  if (pieces <= 4 * 512) return launch<DT, 512, 4, FP8, GROUP>(p, stream);
  if (pieces <= 3 * 1024) return launch<DT, 1024, 3, FP8, GROUP>(p, stream);
  return launch<DT, 1024, 4, FP8, GROUP>(p, stream);
}

template <int DT>
hipError_t launch_type(const Params& p, const RmsNormArgs& a, hipStream_t stream) {
  if (!a.fp8) return launch_threads<DT, false, 0>(p, stream);
  switch (a.group) {
    case 32: return launch_threads<DT, true, 4>(p, stream);
    case 64: return launch_threads<DT, true, 8>(p, stream);
    case 128: return launch_threads<DT, true, 16>(p, stream);
    case 256: return launch_threads<DT, true, 32>(p, stream);
    default: return launch_threads<DT, true, 0>(p, stream);
  }
}

}  // namespace

hipError_t launch_rms_norm(const RmsNormArgs& a, hipStream_t stream) {
  Params p = {};
  p.x = a.x, p.residual = a.residual, p.weight = a.weight;
  p.sum = a.sum, p.out = a.out, p.scales = a.scales;
  p.x_stride = a.x_stride, p.residual_stride = a.residual_stride, p.sum_stride = a.sum_stride;
  p.rows = a.rows, p.width = a.width;
  p.eps = a.eps, p.inv_width = 1.0f / (float)a.width, p.inv = a.inv;
  return a.dtype == 0 ? launch_type<0>(p, a, stream) : launch_type<1>(p, a, stream);
}

}  // namespace qm
