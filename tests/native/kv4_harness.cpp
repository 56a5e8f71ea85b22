// Evaluates the 4-bit cache's layout and launch rules (csrc/kv4_layout.h, kv4_plan.h) for a test:
// one question a line (a word and seven numbers), one line of answers.
#include <cstdio>
#include <iostream>
#include <string>

#include "kv4_layout.h"
#include "kv4_plan.h"

int main() {
  std::string what;
  long long a[7];
  while (std::cin >> what) {
    for (auto& x : a) std::cin >> x;
    if (what == "block") {  // page, hd: bytes; key, value places by (slot, byte); scale places
      const int page = (int)a[0], hd = (int)a[1];
      std::cout << wici::kv4_block_bytes(page, hd);
      for (int which = 0; which < 2; ++which)
        for (int s = 0; s < page; ++s)
          for (int d = 0; d < hd; d += 2)
            std::cout << ' ' << (which ? wici::kv4_value_at(s, d, hd) : wici::kv4_key_at(s, d, hd));
      for (int which = 0; which < 2; ++which)
        for (int s = 0; s < page; ++s)
          for (int g = 0; g < hd / wici::kKv4Group; ++g)
            std::cout << ' ' << (which ? wici::kv4_value_scale_at(s, g, page, hd)
                                       : wici::kv4_key_scale_at(s, g, page, hd));
    } else if (what == "at") {
      std::cout << wici::kv4_block_at((int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)a[4], (int)a[5]);
    } else if (what == "scale") {
      std::cout << wici::kv4_scale_byte((uint32_t)a[0]);
    } else {  // plan: hd, terms, query heads, KV heads, sequences, rows, length
      const wici::Kv8Plan p = wici::kv4_plan((int)a[0], (int)a[1], (int)a[2], (int)a[3], (int)a[4],
                                             (int)a[5], (int)a[6]);
      std::cout << p.row_tiles << ' ' << p.ntile << ' ' << p.nsplit;
    }
    std::cout << '\n';
  }
}
