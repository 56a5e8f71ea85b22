// Evaluates kv8_layout.h: each line of standard input is one question, each line of
// standard output its answer (see tests/test_kv8_host.py).
#include <cstdio>
#include <cstring>
#include <vector>

#include "kv8_layout.h"
#include "kv8_plan.h"

using namespace wici;

int main() {
  char what[16];
  long long a[7];
  while (std::scanf("%15s", what) == 1) {
    for (int i = 0; i < 7; ++i)
      if (std::scanf("%lld", &a[i]) != 1) return 1;
    if (!std::strcmp(what, "block")) {  // page, hd: byte of every code, key then value, then scale
      const int page = (int)a[0], hd = (int)a[1];
      std::printf("%zu", kv8_block_bytes(page, hd));
      for (int w = 0; w < 2; ++w)
        for (int s = 0; s < page; ++s)
          for (int d = 0; d < hd; ++d)
            std::printf(" %d", w ? kv8_value_at(s, d, hd) : kv8_key_at(s, d, hd));
      for (int s = 0; s < page; ++s) std::printf(" %d", kv8_scale_at(s, page, hd));
      std::printf("\n");
    } else if (!std::strcmp(what, "at")) {  // phys, which, h, n_kv, page, hd
      std::printf("%zu\n", kv8_block_at((int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)a[4], (int)a[5]));
    } else if (!std::strcmp(what, "page")) {  // logical page, max_pages, n_pages, table's entry
      // a table of exactly max_pages entries: an access past it is the sanitizer's to find
      std::vector<int32_t> table((size_t)a[1], (int32_t)a[3]);
      const int got = kv8_page(table.data(), a[0], (int)a[1], (int)a[2]);
      if (a[0] >= 0) {  // the look-up in two parts, of entries inside the table
        const uint32_t at = kv8_entry((uint32_t)a[0], (int)a[1]);
        const int two = kv8_named(table[at], (int)a[2]);
        if (a[0] < a[1] ? two != got : at != (uint32_t)a[1] - 1 || two >= (int)a[2]) return 3;
      }
      std::printf("%d\n", got);
    } else if (!std::strcmp(what, "range")) {  // from, to, n_rows
      int row0, rows;
      kv8_range((int)a[0], (int)a[1], (int)a[2], row0, rows);
      std::printf("%d %d\n", row0, rows);
    } else if (!std::strcmp(what, "seen")) {  // len, rows, i, cap
      std::printf("%d\n", kv8_seen((int)a[0], (int)a[1], (int)a[2], a[3]));
    } else if (!std::strcmp(what, "plan")) {  // hd, terms, heads, KV heads, sequences, rows, length
      const Kv8Plan p = kv8_plan((int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)a[4], (int)a[5], (int)a[6]);
      std::printf("%d %d %d\n", p.row_tiles, p.ntile, p.nsplit);
    } else {
      return 2;
    }
  }
  return 0;
}
