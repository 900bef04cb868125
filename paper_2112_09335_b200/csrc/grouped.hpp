// Products grouped by expert and orthogonalised updates: what gcn_admm.cu calls of grouped.cu.
#pragma once
#include <cuda_runtime.h>

#include "grouped_plan.hpp"

namespace gcn_admm_grouped {

// What a call may use besides its operands.  `space` holds space_bytes(..) bytes, `tickets` tickets_of(..) counters that are zero between launches.
struct Room {
  void* space;
  unsigned* tickets;
  int* error_flag;       // raised by a bounded wait that ran out
  cudaStream_t stream;
  long long* launches;   // counted up
};
std::size_t space_bytes(const Product& p);
std::size_t space_bytes(const ProductTn& p);
std::size_t tickets_of(const ProductTn& p);
std::size_t space_bytes(const Orthogonal& p);

// These enqueue checked calls on the current device and return the first CUDA error.
cudaError_t enqueue(const Product& p, const Room& room);
cudaError_t enqueue(const ProductTn& p, const Room& room);
cudaError_t enqueue(const Orthogonal& p, const Room& room);

}  // namespace gcn_admm_grouped
