// Element access and the gate shared by the token-sequence kernels.
#pragma once
#include <cuda_bf16.h>
#include <stdint.h>

namespace pnn {
namespace seq {

using bf16 = __nv_bfloat16;

__device__ __forceinline__ float ld(const float* p) { return *p; }
__device__ __forceinline__ float ld(const bf16* p) { return __bfloat162float(*p); }
__device__ __forceinline__ void st(float* p, float v) { *p = v; }
__device__ __forceinline__ void st(bf16* p, float v) { *p = __float2bfloat16_rn(v); }

// f = sigmoid(z) and g = 1 - f = sigmoid(-z), each with its own relative
// accuracy: 1 - f formed by subtraction would lose g where the gate is nearly
// open.  e = exp(-|z|) <= 1 never overflows; z = +-inf gives exactly 1 and 0.
__device__ __forceinline__ void gate(float z, float& f, float& g) {
  const float e = __expf(-fabsf(z));
  const float r = __fdividef(1.f, 1.f + e), s = e * r;
  const bool up = z >= 0.f;
  f = up ? r : s;
  g = up ? s : r;
}

}  // namespace seq
}  // namespace pnn
