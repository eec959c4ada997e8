// Argument checks that the C entry points share: host code only.
#pragma once

#include <stddef.h>
#include <stdint.h>
#include <string.h>

namespace qm {

inline bool overlaps(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
  return a0 < b0 + nb && b0 < a0 + na;
}

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

// finite iff the exponent field is not all ones (independent of fast-math flags)
inline bool finite_bits(float x) {
  uint32_t u;
  memcpy(&u, &x, sizeof(u));
  return (u & 0x7F800000u) != 0x7F800000u;
}

}  // namespace qm
