// Which kernel attends over the 4-bit cache, in which grid.  Host code alone (no HIP), so that
// a test can evaluate the rules.
#pragma once
#include "kv8_plan.h"

namespace wici {

// Workgroups of the split that the chip holds at once: 4, 3 or 2 wavefronts a SIMD.
inline int resident4(int hd, int terms) { return kCus * (hd == 64 ? 4 : terms == 1 ? 3 : 2); }

inline Kv8Plan kv4_plan(int hd, int terms, int n_q, int n_kv, int n_seqs, int max_rows, int max_length) {
  const int64_t rows = (int64_t)max_rows * (n_q / n_kv), heads = (int64_t)n_seqs * n_kv;
  const int64_t tiles = heads * ((rows + 127) / 128);
  // (a double: 65535 sequences of the longest contexts pass 2^63)
  const double work = (double)heads * ((rows + 15) / 16) * (((int64_t)max_length + kStep - 1) / kStep);
  Kv8Plan p;
  p.row_tiles = rows < kTileRows ? 0
                : tiles >= kFull || work >= 2 * kMuch ? 2
                : tiles >= kHalf ? 1
                : work >= kMuch ? 2 : 0;
  if (terms > 1) p.row_tiles = std::min(p.row_tiles, 1);
  const int64_t per = p.row_tiles ? 64 * p.row_tiles : 16;
  p.ntile = std::max(1, (int)((rows + per - 1) / per));
  const int64_t blocks = heads * p.ntile;
  const int64_t want =
      std::min<int64_t>((p.row_tiles ? 2 * kCus : resident4(hd, terms)) / blocks, 128);
  if (want <= 1) {
    p.nsplit = 1;
  } else if (p.row_tiles) {
    // eight chunks a split at least: partial results of 128 rows are the larger traffic
    const int64_t most = ((int64_t)max_length + 8 * kChunkPos - 1) / (8 * kChunkPos);
    p.nsplit = (int)std::max<int64_t>(1, std::min(want, most));
  } else {
    // each wavefront as many steps
    const int64_t steps = ((int64_t)max_length + kStep - 1) / kStep;
    const int64_t each = steps <= 16 ? 4 : (steps + 4 * want - 1) / (4 * want);
    p.nsplit = (int)std::max<int64_t>(1, (steps + 4 * each - 1) / (4 * each));
  }
  return p;
}

}  // namespace wici
