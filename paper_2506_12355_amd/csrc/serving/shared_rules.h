// How a call of decoding behind a shared prefix is divided, from its sizes and the device's
// CU count: host code only.
#pragma once

#include <stdint.h>

#include "decode_rules.h"
#include "serving_launch.h"

namespace qm {

// Least blocks of a workgroup's part of the prefix: two a wavefront.  us, with 4, 8 and 16: 32
// sequences of 16/1 heads of d = 64 behind 16384 tokens 19.8, 19.9, 22.1; of 64/8 heads 4 behind 2048
// 12.2, 12.7, 14.6, 8 behind 1000 14.4, 15.0, 17.2, 20 behind 2048 22.3, 21.9, 26.2.
constexpr int kLeastBlocks = 8;
// A part's start, its results and their join, in blocks.  Counted as 0 to 16, no case of nine
// changed by 1.5%: what the rounds below leave to choose from is nearly equal.
constexpr int kPartCost = 4;

// es: bytes of a cached value.
inline SharedPlan plan_shared(int64_t B, int64_t H, int64_t Hkv, int d, int es, int64_t limit, int64_t prefix,
                              int cus) {
  SharedPlan p = {};
  const int64_t group = H / Hkv, rows = B * group;   // rows: queries of a key/value head
  const int64_t blocks = (prefix + kDecodeBlock - 1) / kDecodeBlock;
  // 16-row tiles of a workgroup: few rows take blocks straight from memory, 16 or 32 a workgroup;
  // many go over blocks in LDS, 128 a workgroup.  us, 16, 32, 128 rows a workgroup, 64/8 heads and up
  // to 300 own tokens: 16 rows a head behind 2048 tokens 12.5, 14.3, 16.9, behind 16384 23.4, 25.0, 27.7;
  // 32 rows 12.9, 15.2, 17.4, 27.2, 26.0, 29.6, behind 65536 64.9, 58.8, 68.3; 64 rows 15.3, 17.5, 18.7,
  // 36.5, 30.1, 30.2, 99.7, 67.5, 68.1, of E4M3 behind 16384 26.0, 26.7, 30.8, d = 64 23.0, 22.3, 22.4; 80 rows
  // 16.5, 18.1, 20.4, 43.6, 35.9, 31.7, 123, 88.4, 70.1; 128 rows 19.2, 19.4, 21.6, 56.1, 40.4, 34.1, behind
  // 4096 24.1, 22.5, 23.6.  (Behind 4096 and fewer, 16 rows a workgroup would be up to 18% faster.)
  p.rt = rows <= 16 ? 1 : rows <= 64 || (rows <= 128 && blocks <= 64) ? 2 : 8;
  const int64_t tiles = (rows + 16 * p.rt - 1) / (16 * p.rt);
  const int64_t own_rows = B * Hkv * ((group + 15) / 16);
  const int64_t own_blocks = limit > prefix ? (limit + kDecodeBlock - 1) / kDecodeBlock - prefix / kDecodeBlock : 0;
  // The prefix of many rows keeps the matrix cores busy, own tokens the memory: a workgroup of
  // each on a CU does both at once, where two of the prefix and own tokens after them are up to
  // a third slower; but the prefix alone takes up to a quarter longer with one workgroup a CU than
  // with two.  So one, where the prefix's work is at most four times what own tokens then cost nothing
  // and what half as many parts save, in units of a block of 128 rows (2.7 ns at d = 128; so much
  // is a block of own tokens of 16 KB; of their most, half is counted, as lengths vary).  Few
  // rows, which wait for memory, take one by the same rule, a tile's block as half a unit.
  // us, two and one, 64/8 heads, the prefix's tokens and the most own ones: 64 sequences
  // 8192 + 64 55.6, 48.8, + 500 61.5, 50.9, + 8000 243, 215; 32768 + 64 112, 129, + 8000 294, 231; of E4M3
  // 32768 + 2000 145, 149, + 8000 221, 171; d = 64 8192 + 2000 51.3, 43.4, 32768 + 2000 82.8, 100;
  // 8 sequences 16384 + 300 34.5, 30.4, 65536 + 300 69.6, 71.5, d = 64 41.3, 51.6.
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
  // Threads of a head in the join: with few heads four wavefronts, which share a head's parts (us, 64
  // and 256 threads, 64/8 heads: 2 sequences behind 2048 tokens 12.6, 12.3, 4 behind 16384 26.7, 25.3,
  // 8 behind 65536 70.6, 69.5, 16 behind 2048 19.0, 19.0, 32 22.4, 22.9, 64 behind 8192 48.0, 49.6).
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
