// Device helpers that the serving kernels share: 16-bit and E4M3 conversions.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

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
