// How a decode call splits the cached tokens, from its sizes and the device's CU
// count: host code only.
#pragma once

#include <stdint.h>

#include "serving_launch.h"

namespace qm {

constexpr int kDecodeBlock = 32;   // tokens of a wavefront's step
constexpr int kMinShare = 4;       // least blocks of a workgroup's share: one a wavefront
// What a row costs a workgroup beside its blocks, in blocks: its first loads and its
// join, 5-8 us, against 1.1 us a block.  Counted as 0, 6 and 12 (us): 512 rows of up to
// 8192 tokens 205, 198, 199; up to 2000 88, 64, 65; 8 rows of 2000 13.4, 10.8, 10.8.
constexpr int kRowCost = 6;

// Most 32-token blocks that hold visible tokens of a sequence of up to `limit`: those
// of the first keys, and those of a window that begins and ends inside a block.
inline int64_t decode_blocks(int64_t limit, int64_t window, int64_t sinks) {
  const int64_t all = (limit + kDecodeBlock - 1) / kDecodeBlock;
  if (window <= 0) return all;
  const int64_t seen = (sinks + kDecodeBlock - 1) / kDecodeBlock + window / kDecodeBlock + 2;
  return seen < all ? seen : all;
}

// rows: (sequence, key/value head, 16-head tile) triples, each of at most `blocks`.
//
// A workgroup of eight wavefronts for each row needs no second kernel, but a CU draws
// about 64 GB/s, and the longest row is waited for.  us, a workgroup a row -> equal
// shares (bf16, d = 128, rows x tokens, all of one length unless "up to" is said; blocks of
// d = 64 or E4M3, a half or a quarter of the bytes, are divided by the same lines, which
// were not measured for them):
// 8 x 300 8.7 -> 9.4, 8 x 1000 14.7 -> 9.9; 32 x 500 10.4 -> 10.7; 64 x 500 11.5 -> 13.4,
// 64 x 1000 16.0 -> 16.1; 128 x 1000 16.6 -> 19.6, 128 x 2000 37.8 -> 34.9; 256 x 2000
// 51.7 -> 59.3, 256 x 4000 95.3 -> 104.8; 512 x up to 2000 60.0 -> 63.6, x up to 8192
// 215 -> 198; 2048 x up to 4000 360 -> 378.
inline DecodePlan plan_decode(int64_t rows, int64_t blocks, int cus) {
  const bool whole = blocks <= 16 || (blocks <= 32 && 4 * rows >= cus) || (blocks <= 128 && rows >= cus);
  DecodePlan p;
  p.grid = whole ? 0 : 2 * cus;   // two workgroups a CU; with four, pieces are short and end in ramps
  return p;
}

}  // namespace qm
