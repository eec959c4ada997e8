// Device helpers that the serving kernels share: 16-bit and E4M3 conversions, exchanges
// between lanes, division.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

namespace qm {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// 16-bit storage types: 0 = fp16, 1 = bf16.  Packs round to nearest even.
template <int DT>
struct Type16;

template <>
struct Type16<0> {
  static __device__ __forceinline__ f32x2 unpack(uint32_t x) {
    return __builtin_convertvector(__builtin_bit_cast(f16x2, x), f32x2);
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, f16x2));
  }
  static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a),
                                                  __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
  }
};

template <>
struct Type16<1> {
  static __device__ __forceinline__ f32x2 unpack(uint32_t x) {
    return f32x2{__builtin_bit_cast(float, x << 16), __builtin_bit_cast(float, x & 0xffff0000u)};
  }
  static __device__ __forceinline__ uint32_t pack(float x, float y) {
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(f32x2{x, y}, bf16x2));
  }
  static __device__ __forceinline__ f32x4 mfma(u32x4 a, u32x4 b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a),
                                                   __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};

// To E4M3, to nearest even, beyond +-448 the largest value; NaN stays NaN.
__device__ __forceinline__ float to_range(float x) {
  return x != x ? x : fminf(fmaxf(x, -448.f), 448.f);
}
__device__ __forceinline__ uint32_t pack_fp8(float a, float b, float c, float d) {
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(to_range(a), to_range(b), 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(to_range(c), to_range(d), w, true);
}

// f over both values of each pair of 16-lane rows (over_rows), or of the wavefront's halves
// (over_halves): v_permlane16_swap and v_permlane32_swap of a value with itself leave each
// lane the values of both.
template <typename V, typename F>
__device__ __forceinline__ V over_rows(V x, F f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane16_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];
  return f(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b));
}
template <typename V, typename F>
__device__ __forceinline__ V over_halves(V x, F f) {
  const uint32_t u = __builtin_bit_cast(uint32_t, x);
  const auto r = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  const uint32_t a = r[0], b = r[1];
  return f(__builtin_bit_cast(V, a), __builtin_bit_cast(V, b));
}

// f (symmetric) over each aligned run of L lanes, 4 to 64, the same result in all of them.
template <int L, typename V, typename F>
__device__ __forceinline__ V over_lanes(V x, F f) {
  auto with = [&](V v, auto ctrl) __attribute__((always_inline)) {
    const int u = __builtin_amdgcn_mov_dpp(__builtin_bit_cast(int, v), decltype(ctrl)::value, 0xf, 0xf, true);
    return f(v, __builtin_bit_cast(V, u));
  };
  x = with(x, std::integral_constant<int, 0xB1>{});                 // quad_perm [1, 0, 3, 2]
  x = with(x, std::integral_constant<int, 0x4E>{});                 // quad_perm [2, 3, 0, 1]
  if (L >= 8) x = with(x, std::integral_constant<int, 0x141>{});    // row_half_mirror
  if (L >= 16) x = with(x, std::integral_constant<int, 0x140>{});   // row_mirror
  if (L >= 32) x = over_rows(x, f);
  if (L >= 64) x = over_halves(x, f);
  return x;
}

// Exact division of n < 2^31 by a constant of the launch: n d^-1 as a product with the
// rounded-up reciprocal, its 33rd bit added apart (the method of Granlund and Montgomery,
// "Division by invariant integers using multiplication", 1994; n + the product's high half
// fits 32 bits here, so their halving before the sum is not needed).
struct FastDiv {
  uint32_t d, mul, shift;
  FastDiv() = default;
  __host__ explicit FastDiv(uint32_t x) : d(x), shift(0) {
    while ((1ull << shift) < x) ++shift;
    mul = (uint32_t)(((1ull << 32) * ((1ull << shift) - x)) / x + 1);
  }
  __device__ __forceinline__ uint32_t div(uint32_t n) const {
    return (__umulhi(n, mul) + n) >> shift;
  }
};

}  // namespace
}  // namespace qm
