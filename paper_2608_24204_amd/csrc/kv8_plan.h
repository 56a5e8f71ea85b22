// Which kernel attends over the 8-bit cache, in which grid.  Host code alone (no HIP), so that
// a test can evaluate the rules.
#pragma once
#include <algorithm>
#include <cstddef>
#include <cstdint>

namespace wici {

constexpr int kCus = 256;         // compute units of the chip
constexpr int kTiles = 2;         // tiles of 16 positions that a wavefront takes at a time
constexpr int kStep = 16 * kTiles;
constexpr int kChunkTiles = 4;    // tiles of 16 positions a chunk of the row tiles
constexpr int kChunkPos = 16 * kChunkTiles;

// Workgroups that the chip holds at once: 4, 3 or 2 wavefronts a SIMD.
inline int resident(int hd, int terms) { return kCus * (hd == 64 ? 4 : terms == 1 ? 3 : 2); }
struct Kv8Plan {
  int row_tiles;  // prompts: tiles of 16 rows a wavefront; 0: a split of few rows
  int ntile, nsplit;
};
// The splits of the positions of `blocks` workgroups (of either cache).
inline int kv_splits(int hd, int terms, int row_tiles, int64_t blocks, int max_length) {
  const int64_t want = std::min<int64_t>((row_tiles ? 2 * kCus : resident(hd, terms)) / blocks, 128);
  if (want <= 1) return 1;
  if (row_tiles) {
    // eight chunks a split at least: partial results of 128 rows are the larger traffic
    const int64_t most = ((int64_t)max_length + 8 * kChunkPos - 1) / (8 * kChunkPos);
    return (int)std::max<int64_t>(1, std::min(want, most));
  }
  // Each wavefront as many steps: one at 16384 positions (8 bits a value) 16.4 us with 64 splits of two
  // steps a wavefront, 17.6 with the 96 that the chip holds.  Up to 512 positions, four
  // steps, no split: 256 7.7 us (one split) for 9.1 (two, and the merge), 512 9.5 for 9.1,
  // and a call's host work 3 us less; 700 would be 11.0 for 9.1.
  const int64_t steps = ((int64_t)max_length + kStep - 1) / kStep;
  const int64_t each = steps <= 16 ? 4 : (steps + 4 * want - 1) / (4 * want);
  return (int)std::max<int64_t>(1, (steps + 4 * each - 1) / (4 * each));
}
// Which kernel, from the rows x heads of a KV head, the workgroups of 128 of them and the
// 16 rows x 32 positions that all of them multiply (32 query on 8 KV heads of 128, bf16, us a
// call, split / 64 rows / 128 rows):
//  - below 128 rows the split: 16 new rows of each of 8 sequences of 2000: 28 / 28 / 33;
//    16 of 8000 positions: 21 / 23 / 29;
//  - where 128 rows fill the chip, or have long contexts to split: 2048 of 8192 positions:
//    636 / 379 / 288; 16 x 100 of 1000: 87 / 66 / 53; 128 of 8000: 57 / 48 / 48;
//  - a chip half full: 64 rows: 1024 of 1024: 39 / 29 / 57; 32 x 32 of 300: 32 / 19 / 22;
//  - few workgroups and little to do: the split: 333 of 333: 13 / 16 / 22; 256 of 512:
//    13 / 17 / 25.
// With two terms 128 rows' operands and results leave no registers to hold a chunk's operands
// in: 64 rows in their place (64 / 128 rows, while there were both: 2048 of 2048: 93 / 125;
// 8 x 500 of 1000: 105 / 127; 128 of 8000: 56 / 62; 2048 of 8192: 493 / 477, of 16384: 1038 / 997).
// (The farthest from the best of 24 such: 32 of 4000 in 4 sequences, 37 for 34.)
constexpr int kTileRows = 128, kFull = 400, kHalf = 200;
constexpr double kMuch = 60000;
inline Kv8Plan kv8_plan(int hd, int terms, int n_q, int n_kv, int n_seqs, int max_rows, int max_length) {
  const int64_t rows = (int64_t)max_rows * (n_q / n_kv), heads = (int64_t)n_seqs * n_kv;
  const int64_t tiles = heads * ((rows + 127) / 128);
  // (a double: 65535 sequences of the longest contexts pass 2^63)
  const double work = (double)heads * ((rows + 15) / 16) * (((int64_t)max_length + kStep - 1) / kStep);
  Kv8Plan p;
  p.row_tiles = rows < kTileRows ? 0
                : tiles >= kFull || work >= 2 * kMuch ? 2
                : tiles >= kHalf ? 1
                : work >= kMuch ? 2 : 0;
  if (terms == 2) p.row_tiles = std::min(p.row_tiles, 1);
  const int64_t per = p.row_tiles ? 64 * p.row_tiles : 16;
  p.ntile = std::max(1, (int)((rows + per - 1) / per));
  p.nsplit = kv_splits(hd, terms, p.row_tiles, heads * p.ntile, max_length);
  return p;
}

// Workgroups of the merge, one of 256 work-items for each of n rows x heads (1 or more), in two
// dimensions: along one there may be no more than 2^32 - 1 work-items, and n may be 2^24.  The
// last of y may pass n.
struct Kv8Merge {
  unsigned x, y;
};
inline Kv8Merge kv8_merge_grid(int n) {
  const unsigned x = std::min(n, 1 << 20);
  return {x, ((unsigned)n + x - 1) / x};
}

}  // namespace wici
