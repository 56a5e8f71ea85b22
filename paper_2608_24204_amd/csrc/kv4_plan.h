// Which kernel attends over the 4-bit cache, in which grid.  Host code alone (no HIP), so that
// a test can evaluate the rules.
#pragma once
#include "kv8_plan.h"

namespace wici {

// Which kernel, from the rows x heads of a KV head, the workgroups of 128 of them and the 16 rows x 32
// positions that all of them multiply (32 query on 8 KV heads of 128, bf16, us a call, split / 64 rows
// / 128 rows):
//  - below 128 rows the split: 16 new rows of each of 8 sequences of 2000: 26 / 29 / 34; 16 of 8000
//    positions: 20 / 23 / 28;
//  - where 128 rows fill the chip: 8 x 500 of 1000: 133 / 110 / 93; 16 x 100 of 1000: 68 / 66 / 55;
//  - a chip half full: 64 rows, up to the contexts that are worth splitting: 1024 of 2048: 61 / 53 / 71;
//    2 x 512 of 4096: 119 / 116 / 116; 1024 of 8192: 216 / 212 / 182 (heads of 64: 154 / 163 / 159);
//  - few workgroups: 128 rows with much to do, 512 of 8192: 126 / 132 / 106; with little the split: 333
//    of 333: 13 / 17 / 23; between them 128 of 8000: 45 / 50 / 47.
// (Farthest from the best of 40 such: 1300 of 3000, 121 for 111.)
// With three terms 128 rows' operands leave no registers: 64 in their place (3 x 333 of 333 27 for 34 by
// the split, 1024 of 1024 42 for 46).
inline Kv8Plan kv4_plan(int hd, int terms, int n_q, int n_kv, int n_seqs, int max_rows, int max_length) {
  const int64_t rows = (int64_t)max_rows * (n_q / n_kv), heads = (int64_t)n_seqs * n_kv;
  const int64_t tiles = heads * ((rows + 127) / 128);
  // (a double: 65535 sequences of the longest contexts pass 2^63)
  const double work = (double)heads * ((rows + 15) / 16) * (((int64_t)max_length + kStep - 1) / kStep);
  Kv8Plan p;
  p.row_tiles = rows < kTileRows ? 0
                : tiles >= kFull ? 2
                : tiles >= kHalf ? (work >= 5 * kMuch ? 2 : 1)
                : work >= kMuch ? 2 : 0;
  if (terms > 1) p.row_tiles = std::min(p.row_tiles, 1);
  const int64_t per = p.row_tiles ? 64 * p.row_tiles : 16;
  p.ntile = std::max(1, (int)((rows + per - 1) / per));
  p.nsplit = kv_splits(hd, terms, p.row_tiles, heads * p.ntile, max_length);
  return p;
}

}  // namespace wici
