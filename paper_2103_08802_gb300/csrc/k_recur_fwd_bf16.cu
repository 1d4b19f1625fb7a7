#include "recur_tile.cuh"

cudaError_t pnn::recur::run_fwd_bf16(const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st) {
  return dispatch<seq::bf16, false>(a, pl, gave_up, st);
}
