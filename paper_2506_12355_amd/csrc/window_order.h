// The key blocks that a tile of query rows walks under a sliding window, and their order
// (attn_fwd_kernel.h, WINDOW).
#pragma once

#include <hip/hip_runtime.h>

namespace qm {

// Key j is visible to query i iff j <= i and (j > i - window or j < sinks).  Of the
// 64-key blocks that some row of a tile sees there are four kinds: those of first keys
// before all windows, those at the left edges of the windows, those that every row sees
// whole, and those at the diagonal.
//
// Walked in ascending order, a tile starts where its rows see few keys, and the running
// maxima settle only after two or three steps.  So the whole ones come first; the others
// follow in ascending order, so that a wavefront can stop at its own rows' diagonal.
// Which blocks count as whole goes by 256 rows: a row meets its blocks in the same order
// in a tile of 128 rows and in one of 256.  (ascending: all blocks in that order, for the
// key groups of small grids.)
struct WindowOrder {
  int first = 0;      // first block of the tile's windows
  int nsink = 0;      // blocks of first keys before it
  int whole = 0;      // first block that all rows see whole,
  int nwhole = 0;     // how many they are, and
  int nedge = 0;      // blocks from `first` up to them; both 0 where there is none

  // The tile of rows row0 onward.
  __host__ __device__ __forceinline__ void set(int row0, int window, int sinks, bool ascending) {
    const int start = row0 - window + 1;   // of the first row's window
    first = (start > 0 ? start : 0) / 64;
    nsink = (sinks + 63) / 64;
    if (nsink > first) nsink = first;
    const int row = row0 & ~255, edge = row + 255 - window;   // the last key that some row does not see
    whole = (edge + 64 > 0 ? edge + 64 : 0) / 64;
    nwhole = ascending || whole == 0 || whole > row / 64 ? 0 : row / 64 - whole;
    nedge = nwhole > 0 ? whole - first : 0;
  }

  // Steps that cover the blocks up to block n - 1 (n past the windows' first block).
  __host__ __device__ __forceinline__ int steps(int n) const { return n - first + nsink; }

  // The block of step i.
  __host__ __device__ __forceinline__ int block(int i) const {
    int off = first - nsink;
    off = i < nwhole + nsink + nedge ? off - nwhole : off;
    off = i < nwhole + nsink ? -nwhole : off;
    off = i < nwhole ? whole : off;
    return i + off;
  }
  __host__ __device__ __forceinline__ int block_ascending(int i) const {
    return i < nsink ? i : i + first - nsink;
  }
};

}  // namespace qm
