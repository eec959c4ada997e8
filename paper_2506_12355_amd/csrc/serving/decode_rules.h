// How a decode call splits the cached tokens, from its sizes and the device's CU
// count: host code only.
#pragma once

#include <stdint.h>

#include "serving_launch.h"

namespace qm {

constexpr int kDecodeBlock = 32;   // tokens of a wavefront's step
constexpr int kDecodeWaves = 4;    // wavefronts of a workgroup

// Most 32-token blocks that hold visible tokens of a sequence of up to `limit`: those
// of the first keys, and those of a window that begins and ends inside a block.
inline int64_t decode_blocks(int64_t limit, int64_t window, int64_t sinks) {
  const int64_t all = (limit + kDecodeBlock - 1) / kDecodeBlock;
  if (window <= 0) return all;
  const int64_t seen = (sinks + kDecodeBlock - 1) / kDecodeBlock + window / kDecodeBlock + 2;
  return seen < all ? seen : all;
}

inline DecodePlan plan_decode(int64_t rows, int64_t blocks, int cus) {
  // rows: (sequence, key/value head, 16-head tile) triples
  const int64_t most = (blocks + 7) / 8;        // at least 256 tokens a workgroup
  const int64_t least = (blocks + 127) / 128;   // at most 4096
  int64_t splits = (4 * (int64_t)cus + rows - 1) / rows;
  if (splits < least) splits = least;
  if (splits > most) splits = most;
  if (splits < 1) splits = 1;
  int64_t chunk = (blocks + splits - 1) / splits;
  chunk = (chunk + kDecodeWaves - 1) / kDecodeWaves * kDecodeWaves;
  DecodePlan p;
  p.waves = kDecodeWaves;
  p.chunk = (int)chunk;
  p.splits = (int)((blocks + chunk - 1) / chunk);
  return p;
}

}  // namespace qm
