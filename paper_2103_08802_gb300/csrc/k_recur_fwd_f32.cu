#include "recur_tile.cuh"

cudaError_t pnn::recur::run_fwd_f32(const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st) {
  return dispatch<float, false>(a, pl, gave_up, st);
}
