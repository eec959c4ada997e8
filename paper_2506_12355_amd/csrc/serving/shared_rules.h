// How a call of decoding behind a shared prefix is divided, from its sizes and the device's
// CU count: host code only.
#pragma once

#include <stdint.h>

#include "decode_rules.h"
#include "serving_launch.h"

namespace qm {

constexpr int kLeastBlocks = 8;   // of a workgroup's part of the prefix: two a wavefront
constexpr int kPartCost = 4;      // a part's start, its results and their join, in blocks

// es: bytes of a cached value.
inline SharedPlan plan_shared(int64_t B, int64_t H, int64_t Hkv, int d, int es, int64_t limit, int64_t prefix,
                              int cus) {
  SharedPlan p = {};
  const int64_t group = H / Hkv, rows = B * group;   // rows: queries of a key/value head
  const int64_t blocks = (prefix + kDecodeBlock - 1) / kDecodeBlock;
  p.rt = rows <= 16 ? 1 : rows <= 64 || (rows <= 128 && blocks <= 64) ? 2 : 8;
  const int64_t tiles = (rows + 16 * p.rt - 1) / (16 * p.rt);
  const int64_t own_rows = B * Hkv * ((group + 15) / 16);
  const int64_t own_blocks = limit > prefix ? (limit + kDecodeBlock - 1) / kDecodeBlock - prefix / kDecodeBlock : 0;
  // The prefix of many rows keeps the matrix cores busy, own tokens the memory: a workgroup of
  // each on a CU does both at once, where two of the prefix and own tokens after them are up to
  // a third slower; but the prefix alone takes a quarter longer with one workgroup a CU than with
  // two.  So one, where the prefix's work is at most four times what own tokens then cost nothing
  // and what half as many parts save, in units of a block of 128 rows (2.7 ns at d = 128; so much
  // is a block of own tokens of 16 KB; of their most, half is counted, as lengths vary).  Few
  // rows, which wait for memory, take one by the same rule, a tile's block as half a unit.
  // us, both ways, 64/8 heads, the prefix's tokens and the most own ones: 64 sequences
  // 8192 + 64 53.6, 47.9, + 500 58.2, 49.3, + 8000 241, 211; 32768 + 64 120, 127, + 8000 289, 229;
  // of E4M3 32768 + 2000 136, 142, + 8000 210, 173; d = 64 8192 + 2000 46.3, 37.8, 32768 + 2000 83.8,
  // 94.8; 8 sequences 16384 + 300 31.0, 24.1, 65536 + 300 66.4, 68.9, d = 64 35.8, 44.9.
  const double prefix_work = (double)(Hkv * tiles * blocks) * (p.rt == 8 ? 1.0 : 0.5) * (d == 128 ? 1.0 : 0.65);
  const double own_work = (double)(own_rows * own_blocks) * (d * es / 256.0), saved = 7600.0 * d / 128;
  const bool beside = own_blocks && prefix_work < own_work + saved;
  const int64_t slots = (beside ? 1 : 2) * (int64_t)cus;
  // Parts that fill one to four rounds of the workgroups that are on the device at once, or one
  // part a tile: the rounds' blocks, and what a part costs beside them.
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
  const int64_t shares = (own_rows * (own_blocks + kRowCost) + kMinShare - 1) / kMinShare;   // as share_of deals them
  p.join_threads = B * H < 4 * (int64_t)cus ? 256 : 64;
  // Beside few rows, own tokens' workgroups are those that are on the device with the prefix's, one a
  // CU at least (us, and with two a CU: 8 sequences 4000 + 1000 17.5, 21.6, + 4000 22.4, 27.2).  Beside
  // many, whose workgroups end first where own tokens are many, two (d = 64 and E4M3 up to 30%
  // faster, else 2-4% slower).
  const int64_t left = 2 * (int64_t)cus - (p.rt == 8 ? 0 : p.prefix_grid), grid = left < cus ? cus : left;
  p.own_grid = own_blocks ? (int)(shares < grid ? shares : grid) : 0;
  return p;
}

// Slots for the partial results of 16 heads of the sequences' own tokens: two for each
// workgroup, which cuts at most its first row and its last, and one for each row, for one
// that lies whole in a share.
inline size_t own_slots(const SharedPlan& p, int64_t B, int64_t H, int64_t Hkv) {
  return p.own_grid ? 2 * (size_t)p.own_grid + (size_t)(B * Hkv * ((H / Hkv + 15) / 16)) : 0;
}

}  // namespace qm
