// Reads lines from standard input:
//   w address valid    -> the words that HalfWords asks for: byte addresses, lowest first
//   p part apart       -> part_at
//   c slots flags      -> copies into so many slots in turn, one for each bit of `flags` below its highest, lowest first (set: one that brings rows behind an
//                         item): for each of the last that may be in flight its slot, whether it reports to `tail`, and the parity of the phase that it ends
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
    if (what == 'c') {
      gcn_admm_grouped::CopyLog log;
      const int slots = (int)a;
      for (int i = 0; b >> (i + 1) != 0; ++i) log.add(i % slots, (b >> i & 1) != 0);
      for (int i = log.started > slots ? log.started - slots : 0; i < log.started; ++i) {
        const int slot = i % slots;
        std::printf("%d %d %u ", slot, (int)log.is_tail(slot), log.is_tail(slot) ? log.tail_parity(slot) : gcn_admm_grouped::CopyLog::full_parity(i, slots));
      }
      std::printf("\n");
      continue;
    }
    const gcn_admm_grouped::HalfWords w((std::uintptr_t)a, (int)b);
    for (int k = 0; k < 5; ++k)
      if (w.holds(k)) std::printf("%llu ", (unsigned long long)w.first + 4 * k);
    std::printf("\n");
  }
}
