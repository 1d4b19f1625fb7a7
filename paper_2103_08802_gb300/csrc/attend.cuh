// What the kernels of the linear attention share: the pass that all of its
// directions are, the split of the time axis, powers of the decay.
//
// One pass over the rows x, y, z of a head (t ascending, or descending in a
// reverse one) is
//   out_i = fp sum_{j up to i} a^|i-j| (x_i . y_j) z_j  +  fo a^(p+1-rev) x_i^T S
//   S    := a^n S + fs sum_j a^(n-1-p+rev) y_j z_j^T
// for a piece of n tokens, p the place of a token in it in the pass's order, S
// (dx x dz) the state that comes from the pieces before.  With it
//   o  = forward (q, k, v),  S from s0, to s_last
//   dq = forward (dO, v, k), S from s0^T
//   dk = reverse (v, dO, q), S from ds_last^T
//   dv = reverse (k, q, dO), S from ds_last, to ds0
// (a reverse state has a token's own decay in it already, which is what ds0 is.)
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

#include "pnn_seq.h"
#include "seq_common.cuh"

namespace pnn {
namespace attend {

struct Rows {
  void* p;
  int64_t b, t, h;  // strides in elements
};
struct Pass {
  Rows x, y, z, out;
  int dx, dz;         // the state is dx x dz
  bool rev;
  float fp, fo, fs;
  const float* init;  // batch x heads x (dx x dz, or dz x dx if init_t)
  bool init_t;
  float* end;         // batch x heads x dx x dz
  float* carry;       // with segments: batch x heads x segments x dx x dz, a segment's own sum, then the state before it
};
struct Work {
  Pass pass[3];
  int passes, batch, time, heads;
  int dtype;
  const int* lengths;
  const float* decay;
  int segments, seg;  // tokens of a segment (a multiple of the kernel's chunk)
};

// a^n to 2^-46 n of itself: binary powers in pairs of fp32 numbers (the rest of every product is kept)
struct Df {
  float h, l;
};
__device__ __forceinline__ Df df_mul(Df a, Df b) {
  const float p = a.h * b.h;
  const float e = fmaf(a.h, b.l, fmaf(a.l, b.h, fmaf(a.h, b.h, -p)));
  Df r;
  r.h = p + e;
  r.l = e - (r.h - p);
  return r;
}
__device__ __forceinline__ float power(float a, uint32_t n) {
  Df r{1.f, 0.f}, x{a, 0.f};
  while (n) {
    if (n & 1) r = df_mul(r, x);
    n >>= 1;
    if (n) x = df_mul(x, x);
  }
  return r.h;
}
// a head's decay: outside [0, 1] (and NaN) clamped
__device__ __forceinline__ float decay_of(const Work& w, int head) { return fminf(fmaxf(w.decay[head], 0.f), 1.f); }
__device__ __forceinline__ int length_of(const Work& w, int b) {
  const int n = w.lengths ? w.lengths[b] : w.time;
  return n < 0 ? 0 : n > w.time ? w.time : n;
}

// the segments' own sums in `carry` become the states before them
cudaError_t launch_join(const Work& w, cudaStream_t st);
// bf16 rows of up to 128 on 16-byte boundaries: the tensor-core kernel.  *refused: the driver encodes no map for such
// strides, nothing has been launched.
bool tc_fits(const Work& w);
cudaError_t run_tc(const Work& w, cudaStream_t st, bool* refused);

}  // namespace attend
}  // namespace pnn
