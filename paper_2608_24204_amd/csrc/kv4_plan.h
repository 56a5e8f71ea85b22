// Which kernel attends over the 4-bit cache, in which grid.  Host code alone (no HIP), so that
// a test can evaluate the rules.
#pragma once
#include "kv8_plan.h"

namespace wici {

// Workgroups of the split that the chip holds at once: 4, 3 or 2 wavefronts a SIMD.
inline int resident4(int hd, int terms) { return kCus * (hd == 64 ? 4 : terms == 1 ? 3 : 2); }

inline Kv8Plan kv4_plan(int hd, int terms, int n_q, int n_kv, int n_seqs, int max_rows, int max_length) {
  const int64_t rows = (int64_t)max_rows * (n_q / n_kv), heads = (int64_t)n_seqs * n_kv;
  Kv8Plan p;
  p.row_tiles = 0;
  p.ntile = std::max(1, (int)((rows + 15) / 16));
  const int64_t blocks = heads * p.ntile;
  const int64_t want = std::min<int64_t>(resident4(hd, terms) / blocks, 128);
  if (want <= 1) {
    p.nsplit = 1;
  } else {
    // each wavefront as many steps
    const int64_t steps = ((int64_t)max_length + kStep - 1) / kStep;
    const int64_t each = steps <= 16 ? 4 : (steps + 4 * want - 1) / (4 * want);
    p.nsplit = (int)std::max<int64_t>(1, (steps + 4 * each - 1) / (4 * each));
  }
  return p;
}

}  // namespace wici
