// Entry of the norms around a block; norm_rows.cuh has the kernels.
#include "norm_rows.cuh"

namespace pnn {

size_t norm_workspace(const pnn_norm_args& a) {
  if (!a.rows || !(a.weight || a.scales || a.next_weight)) return 0;
  const unsigned g = norm::plan(a, true, true).grid, h = norm::plan(a, true, false).grid;  // (whichever the rows' addresses allow)
  return (size_t)(g > h ? g : h) * 3 * a.width * 4;
}
cudaError_t launch_norm(const pnn_norm_args& a, bool back, void* ws, cudaStream_t st) {
  return a.dtype == PNN_DT_BF16 ? norm::run_bf16(a, back, static_cast<float*>(ws), st) : norm::run_f32(a, back, static_cast<float*>(ws), st);
}

}  // namespace pnn
