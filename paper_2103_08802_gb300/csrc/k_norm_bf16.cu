#include "norm_rows.cuh"

namespace pnn {
cudaError_t norm::run_bf16(const pnn_norm_args& a, bool back, float* ws, cudaStream_t st) {
  return a.res_dtype == PNN_DT_BF16 ? aligned<seq::bf16, seq::bf16>(a, back, ws, st) : aligned<seq::bf16, float>(a, back, ws, st);
}
}  // namespace pnn
