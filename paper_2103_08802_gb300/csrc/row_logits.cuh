// Rows of logits held in registers: what the distillation and the policy loss
// share.  16-byte vectors of bf16 or fp32 logits, their maximum and exponentials,
// where a row lies in vectors, and sums that meet across warps and CTAs.
#pragma once
#include <math.h>

#include "seq_common.cuh"

namespace pnn {
namespace seq {

constexpr int kMaxCluster = 8;

// 2^y to 2^-22 of itself; below 2^-126 it is 0.  For fp32 logits too: a sum of such terms is no further off, nor is the logarithm
// that a loss takes of it.
__device__ __forceinline__ float ex2(float y) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}
__device__ __forceinline__ f2 ex2p(f2 y) {
  float a, b;
  upk(y, a, b);
  return pk(ex2(a), ex2(b));
}
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

// logits are read once: not kept in L1 (and not through the read-only path, since the gradient may replace them)
__device__ __forceinline__ uint4 ld_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
// the 2 * P pairs of a vector (bf16: 4, fp32: 2)
template <typename T> constexpr int kPairs = 8 / sizeof(T);
template <typename T> __device__ __forceinline__ f2 pair_of(const uint4& v, int i);
template <> __device__ __forceinline__ f2 pair_of<bf16>(const uint4& v, int i) {
  const uint32_t w = i == 0 ? v.x : i == 1 ? v.y : i == 2 ? v.z : v.w;
  return pk(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u));
}
template <> __device__ __forceinline__ f2 pair_of<float>(const uint4& v, int i) {
  return i == 0 ? pk(__uint_as_float(v.x), __uint_as_float(v.y)) : pk(__uint_as_float(v.z), __uint_as_float(v.w));
}
// the largest value of a vector (NaN passed over: the sums show it)
template <typename T> __device__ __forceinline__ float max_of(const uint4& v);
template <> __device__ __forceinline__ float max_of<bf16>(const uint4& v) {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
  const __nv_bfloat162 m = __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
  return fmaxf(__low2float(m), __high2float(m));
}
template <> __device__ __forceinline__ float max_of<float>(const uint4& v) {
  return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
}
template <typename T> __device__ __forceinline__ uint4 minus_inf();
template <> __device__ __forceinline__ uint4 minus_inf<bf16>() { return make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u); }
template <> __device__ __forceinline__ uint4 minus_inf<float>() { return make_uint4(0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u); }

// The base of the exponents: the maximum, or 0 where there is none (no value
// yet, or only masked ones: their sums are 0).
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// the factor that takes sums from the base of maximum m to base b
__device__ __forceinline__ float rebase(float m, float b, float k) { return m == -INFINITY ? 0.f : ex2((m - b) * k); }

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void put_remote(const float4* place, uint32_t rank, float4 v) {
  uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(place)), to;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(at), "r"(rank));
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(to), "f"(v.x), "f"(v.y), "f"(v.z), "f"(v.w) : "memory");
}

template <typename T>
__device__ __forceinline__ void put(T* to, const uint4& v, bool whole) {
  if (whole) {
    __stcs(reinterpret_cast<uint4*>(to), v);
  } else {
    const T* q = reinterpret_cast<const T*>(&v);
#pragma unroll
    for (int p = 0; p < (int)(16 / sizeof(T)); ++p) to[p] = q[p];
  }
}
template <typename T, int NV>
__device__ __forceinline__ float warp_max(const uint4 (&x)[NV], float m) {
#pragma unroll
  for (int i = 0; i < NV; ++i) m = fmaxf(m, max_of<T>(x[i]));
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// Where a row lies in 16-byte vectors: `head` values before the first, `all`
// vectors of which this CTA has nv from v0 on, and what is behind the last.
template <typename T>
struct Span {
  static constexpr int E = 16 / sizeof(T);
  const T* s;
  int head, all, each, v0, nv;
  __device__ __forceinline__ Span(const void* logits, int64_t stride, int V, int64_t row, int rank, int C) {
    s = static_cast<const T*>(logits) + row * stride;
    const int off = (int)((reinterpret_cast<uintptr_t>(s) & 15) / sizeof(T));
    head = off ? (E - off < V ? E - off : V) : 0;
    all = (V - head) / E;
    each = C > 1 ? (all + C - 1) / C : all;
    v0 = rank * each < all ? rank * each : all;
    nv = each < all - v0 ? each : all - v0;
  }
  __device__ __forceinline__ const uint4* vec() const { return reinterpret_cast<const uint4*>(s + head) + v0; }
  // the single value of thread tid: threads 0 .. head - 1, and E .. E + tail - 1, of rank 0; else -1
  __device__ __forceinline__ int lone(int V, int rank, int tid) const {
    const int done = head + all * E;
    if (rank != 0) return -1;
    return tid < head ? tid : tid >= E && tid - E < V - done ? done + tid - E : -1;
  }
};

}  // namespace seq
}  // namespace pnn
