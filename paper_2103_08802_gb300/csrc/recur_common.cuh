// What the two forms of the gated recurrence share: the piece of time steps
// whose first state the forward saves, and the length of a sequence.
#pragma once
#include <cuda_bf16.h>

#include "../../include/pnn.h"

namespace pnn {

// steps of one thread's run; a piece is 8 runs
template <typename T>
constexpr int kRunSteps = sizeof(T) == 2 ? 11 : 6;

__device__ __forceinline__ int recur_len(const pnn_recur_args& a, int64_t b) {
  if (!a.lengths) return (int)a.time;
  const int64_t n = a.lengths[b];
  return (int)(n < 0 ? 0 : n > a.time ? a.time : n);
}

}  // namespace pnn
