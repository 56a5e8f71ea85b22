// Evaluates the arithmetic of csrc/kv8_layout.h and csrc/kv8_plan.h at the ends of its range: each
// line of standard input is one question, each line of standard output its answer (see
// tests/test_kv8_range_host.py).
#include <cstdio>
#include <cstring>

#include "kv8_layout.h"
#include "kv8_plan.h"

using namespace wici;

int main() {
  char what[16];
  long long a[3];
  while (std::scanf("%15s", what) == 1) {
    for (int i = 0; i < 3; ++i)
      if (std::scanf("%lld", &a[i]) != 1) return 1;
    if (!std::strcmp(what, "part")) {  // part, parts, hd: its output, its state, floats of all
      std::printf("%zu %zu %zu\n", kv8_part_out((size_t)a[0], (int)a[2]),
                  kv8_part_state((size_t)a[0], (size_t)a[1], (int)a[2]),
                  kv8_part_floats((size_t)a[1], (int)a[2]));
    } else if (!std::strcmp(what, "steps")) {  // n, step
      std::printf("%d\n", kv8_steps((int)a[0], (int)a[1]));
    } else if (!std::strcmp(what, "merge")) {  // rows x heads
      const Kv8Merge m = kv8_merge_grid((int)a[0]);
      std::printf("%u %u\n", m.x, m.y);
    } else {
      return 2;
    }
  }
  return 0;
}
