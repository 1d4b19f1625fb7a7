#include "norm_rows.cuh"

namespace pnn {
cudaError_t norm::run_f32(const pnn_norm_args& a, bool back, float* ws, cudaStream_t st) {
  return a.res_dtype == PNN_DT_BF16 ? aligned<float, seq::bf16>(a, back, ws, st) : aligned<float, float>(a, back, ws, st);
}
}  // namespace pnn
