// How a call of decoding behind a shared prefix is divided, from its sizes and the device's
// CU count: host code only.
#pragma once

#include <stdint.h>

#include "decode_rules.h"
#include "serving_launch.h"

namespace qm {

constexpr int kLeastBlocks = 8;   // of a workgroup's part of the prefix: two a wavefront
constexpr int kPartCost = 4;      // a part's start, its results and their join, in blocks

// rows: queries of a key/value head, B * H / Hkv.
inline SharedPlan plan_shared(int64_t B, int64_t H, int64_t Hkv, int64_t limit, int64_t prefix, int cus) {
  SharedPlan p = {};
  const int64_t group = H / Hkv, rows = B * group, slots = 2 * (int64_t)cus;
  const int64_t blocks = (prefix + kDecodeBlock - 1) / kDecodeBlock;
  p.rt = rows <= 16 ? 1 : rows <= 64 || (rows <= 128 && blocks <= 64) ? 2 : 8;
  const int64_t tiles = (rows + 16 * p.rt - 1) / (16 * p.rt);
  // Parts that fill one to four rounds of the device's workgroups, or one part a tile: the
  // rounds' blocks, and what a part costs beside them.
  const int64_t base = Hkv * tiles, most = (blocks + kLeastBlocks - 1) / kLeastBlocks;
  int64_t splits = 1, least = -1;
  for (int64_t rounds = 0; rounds <= 4; ++rounds) {
    int64_t n = rounds ? rounds * slots / base : 1;
    n = n < 1 ? 1 : n > most ? most : n;
    const int64_t cost = (base * n + slots - 1) / slots * ((blocks + n - 1) / n + kPartCost);
    if (least < 0 || cost < least) least = cost, splits = n;
  }
  p.tiles = (int)tiles;
  p.splits = (int)splits;
  // eight (head, part) pairs side by side, one to an XCD, each with all of its tiles
  p.prefix_grid = (int)((Hkv * splits + 7) / 8 * 8 * tiles);
  const int64_t own_rows = B * Hkv * ((group + 15) / 16);
  const int64_t own_blocks = limit > prefix ? (limit + kDecodeBlock - 1) / kDecodeBlock - prefix / kDecodeBlock : 0;
  const int64_t shares = (own_rows * (own_blocks + 6) + 3) / 4;
  p.join_threads = B * H < 4 * (int64_t)cus ? 256 : 64;
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
