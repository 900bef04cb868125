// Prints, for lines "address valid" read from standard input, the words that HalfWords asks for: byte addresses, lowest first.
#include <cstdio>
#include <iostream>

#include "../paper_2112_09335_b200/csrc/grouped_words.hpp"

int main() {
  unsigned long long address;
  long long valid;
  while (std::cin >> address >> valid) {
    const gcn_admm_grouped::HalfWords w((std::uintptr_t)address, (int)valid);
    for (int k = 0; k < 5; ++k)
      if (w.holds(k)) std::printf("%llu ", (unsigned long long)w.first + 4 * k);
    std::printf("\n");
  }
}
