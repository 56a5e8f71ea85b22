// Evaluates what the attention over the 4-bit cache makes of large values (csrc/kv4_layout.h) for a test:
// positions in, and for weights as halves and in bf16 the first large scale byte and the lift out.
#include <iostream>

#include "kv4_layout.h"

int main() {
  long long n;
  while (std::cin >> n) {
    for (const wici::Room& r : {wici::kRoomHalf, wici::kRoomBf16})
      std::cout << r.most << ' ' << r.top << ' ' << r.log_most << ' ' << wici::kv4_large_byte(r, (int)n) << ' '
                << wici::kv4_lift(r, (int)n) << ' ';
    std::cout << '\n';
  }
}
