// Reads lines from standard input:
//   w address valid    -> the words that HalfWords asks for: byte addresses, lowest first
//   p part apart       -> part_at
#include <cstdio>
#include <iostream>

#include "../paper_2112_09335_b200/csrc/grouped_words.hpp"

int main() {
  char what;
  long long a, b;
  while (std::cin >> what >> a >> b) {
    if (what == 'p') {
      std::printf("%lld\n", (long long)gcn_admm_grouped::part_at((int)a, b));
      continue;
    }
    const gcn_admm_grouped::HalfWords w((std::uintptr_t)a, (int)b);
    for (int k = 0; k < 5; ++k)
      if (w.holds(k)) std::printf("%llu ", (unsigned long long)w.first + 4 * k);
    std::printf("\n");
  }
}
