// How a call of decoding behind a shared prefix is divided, from its sizes and the device's
// CU count: host code only.
#pragma once

#include <stdint.h>

#include "decode_rules.h"
#include "serving_launch.h"

namespace qm {

constexpr int kLeastBlocks = 8;   // of a workgroup's part of the prefix: two a wavefront

// rows: queries of a key/value head, B * H / Hkv.
inline SharedPlan plan_shared(int64_t B, int64_t H, int64_t Hkv, int64_t limit, int64_t prefix, int cus) {
  SharedPlan p = {};
  const int64_t group = H / Hkv, rows = B * group, slots = 2 * (int64_t)cus;
  const int64_t blocks = (prefix + kDecodeBlock - 1) / kDecodeBlock;
  p.rt = rows <= 16 ? 1 : 2;
  const int64_t tiles = (rows + 16 * p.rt - 1) / (16 * p.rt);
  int64_t splits = slots / (Hkv * tiles);
  const int64_t most = (blocks + kLeastBlocks - 1) / kLeastBlocks;
  splits = splits < 1 ? 1 : splits;
  splits = splits > most ? most : splits;
  p.tiles = (int)tiles;
  p.splits = (int)splits;
  // eight (head, part) pairs side by side, one to an XCD, each with all of its tiles
  p.prefix_grid = (int)((Hkv * splits + 7) / 8 * 8 * tiles);
  const int64_t own_rows = B * Hkv * ((group + 15) / 16);
  const int64_t own_blocks = limit > prefix ? (limit + kDecodeBlock - 1) / kDecodeBlock - prefix / kDecodeBlock : 0;
  const int64_t shares = (own_rows * (own_blocks + 6) + 3) / 4;
  p.own_grid = own_blocks ? (int)(shares < slots ? shares : slots) : 0;
  return p;
}

// Slots for the partial results of 16 heads of the sequences' own tokens: two for each
// workgroup, which cuts at most its first row and its last, and one for each row, for one
// that lies whole in a share.
inline size_t own_slots(const SharedPlan& p, int64_t B, int64_t H, int64_t Hkv) {
  return p.own_grid ? 2 * (size_t)p.own_grid + (size_t)(B * Hkv * ((H / Hkv + 15) / 16)) : 0;
}

}  // namespace qm
