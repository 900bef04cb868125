// Which words of memory the loads and stores of the grouped products touch.  Arithmetic only, so that it can be tested without a GPU.
#pragma once
#include <cstdint>

#ifdef __CUDACC__
#define GROUPED_BOTH __host__ __device__ __forceinline__
#else
#define GROUPED_BOTH inline
#endif

namespace gcn_admm_grouped {

// Eight halves of a row on any boundary, the first `valid` of them inside of the matrix (none where it is not positive), as the aligned words that
// hold them.  Only words with a valid half may be loaded: where there is none, the address itself may lie anywhere.
struct HalfWords {
  std::uintptr_t first;   // address of word 0
  int some, odd;          // halves that are valid; whether the first of them is the second of its word
  GROUPED_BOTH HalfWords(std::uintptr_t address, int valid)
      : first(address & ~std::uintptr_t(3)), some(valid < 0 ? 0 : valid > 8 ? 8 : valid), odd(valid > 0 ? (int)(address >> 1 & 1) : 0) {}
  GROUPED_BOTH bool holds(int word) const { return 2 * word < some + odd; }
};

// Byte offset of part k of an element whose parts lie `apart` bytes from each other (images of split weights are longer than an int counts).
GROUPED_BOTH long long part_at(int k, long long apart) { return k * apart; }

// Copies that one thread has started, into the slots of a ring in turn: for each slot, which of two barriers its last copy reports to, and the phase of
// that barrier which the copy ends.  (full: every copy of the slot ends a phase of it, at its own end or when the rows behind an item are cleared;
// tail: only the copies that bring such rows.)
struct CopyLog {
  int started = 0;
  std::uint32_t tails = 0, odd_tails = 0;   // a bit for each slot: the last copy reports to `tail`; an odd number of copies have
  GROUPED_BOTH void add(int slot, bool tail) {
    const std::uint32_t bit = 1u << slot;
    tails = tail ? tails | bit : tails & ~bit;
    if (tail) odd_tails ^= bit;
    ++started;
  }
  GROUPED_BOTH bool is_tail(int slot) const { return (tails >> slot & 1u) != 0; }
  GROUPED_BOTH std::uint32_t tail_parity(int slot) const { return (odd_tails >> slot & 1u) ^ 1u; }
  static GROUPED_BOTH std::uint32_t full_parity(int copy, int slots) { return (std::uint32_t)(copy / slots) & 1u; }
};

}  // namespace gcn_admm_grouped
