// How a call of row norms is divided: host code only.
#pragma once

#include <stdint.h>

namespace qm {

// Rows of one launch, of `threads` each (a power of two, 1024 at most): HIP refuses launches
// of 2^32 threads and more.
constexpr int rows_of_launch(int threads) { return (int)((int64_t{1} << 31) / threads); }

}  // namespace qm
