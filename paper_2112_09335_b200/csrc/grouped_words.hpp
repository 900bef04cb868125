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
  int odd, some;          // whether the first half is the second of its word; halves that are valid
  GROUPED_BOTH HalfWords(std::uintptr_t address, int valid) : first(address & ~std::uintptr_t(3)), odd((int)(address >> 1 & 1)), some(valid < 0 ? 0 : valid > 8 ? 8 : valid) {}
  GROUPED_BOTH bool holds(int word) const { return some > 0 && 2 * word < some + odd; }
};

// Byte offset of part k of an element whose parts lie `apart` bytes from each other (images of split weights are longer than an int counts).
GROUPED_BOTH long long part_at(int k, long long apart) { return k * apart; }

}  // namespace gcn_admm_grouped
