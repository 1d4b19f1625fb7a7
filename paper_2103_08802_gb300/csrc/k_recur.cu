// Gated linear recurrence: forward scan, backward pass, single-token step.
#include "pnn_internal.h"
#include "pnn_seq.h"
#include "seq_common.cuh"

namespace pnn {
namespace {
using namespace seq;

constexpr int kChunk = 32;  // time steps between saved states

__device__ __forceinline__ int seq_len(const pnn_recur_args& a, int64_t b) {
  if (!a.lengths) return (int)a.time;
  const int64_t n = a.lengths[b];
  return (int)(n < 0 ? 0 : n > a.time ? a.time : n);
}

// One thread a channel, the whole sequence in order.
template <typename T>
__global__ void k_recur_fwd(pnn_recur_args a) {
  const int64_t D = a.heads * a.width, c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, b = blockIdx.y;
  if (c >= D) return;
  const int n = seq_len(a, b);
  const T* z = static_cast<const T*>(a.z) + b * a.z_stride_b + c / a.width;
  const T* x = static_cast<const T*>(a.x) + b * a.x_stride_b + c;
  T* h = static_cast<T*>(a.h) + b * a.h_stride_b + c;
  const int64_t chunks = (a.time + kChunk - 1) / kChunk;
  float s = a.h0 ? a.h0[b * D + c] : 0.f;
  for (int64_t t = 0; t < a.time; ++t) {
    if (a.saved && t % kChunk == 0) a.saved[(b * chunks + t / kChunk) * D + c] = s;
    if (t < n) {
      float f, g;
      gate(ld(z + t * a.z_stride_t), f, g);
      s = f * s + g * ld(x + t * a.x_stride_t);
    }
    st(h + t * a.h_stride_t, t < n ? s : 0.f);
  }
  if (a.h_last) a.h_last[b * D + c] = s;
}

// Backward, one thread a channel: chunk by chunk from the end, the states of a
// chunk recomputed in fp32 from its saved first state.  part: dz of each
// channel, batch x time x channels fp32, where a head has several channels.
template <typename T>
__global__ void k_recur_bwd(pnn_recur_args a, float* part) {
  const int64_t D = a.heads * a.width, c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, b = blockIdx.y;
  if (c >= D) return;
  const int n = seq_len(a, b);
  const T* z = static_cast<const T*>(a.z) + b * a.z_stride_b + c / a.width;
  const T* x = static_cast<const T*>(a.x) + b * a.x_stride_b + c;
  const T* dh = static_cast<const T*>(a.dh) + b * a.dh_stride_b + c;
  T* dx = static_cast<T*>(a.dx) + b * a.dx_stride_b + c;
  T* dz = static_cast<T*>(a.dz) + b * a.dz_stride_b + c;
  const int64_t chunks = (a.time + kChunk - 1) / kChunk;
  float r = a.dh_last ? a.dh_last[b * D + c] : 0.f;  // gradient of the state from the steps after
  for (int64_t k = chunks - 1; k >= 0; --k) {
    float hp[kChunk];
    const int64_t t0 = k * kChunk;
    float s = a.saved[(b * chunks + k) * D + c];
#pragma unroll
    for (int i = 0; i < kChunk; ++i) {
      hp[i] = s;
      if (t0 + i < n) {
        float f, g;
        gate(ld(z + (t0 + i) * a.z_stride_t), f, g);
        s = f * s + g * ld(x + (t0 + i) * a.x_stride_t);
      }
    }
#pragma unroll
    for (int i = kChunk - 1; i >= 0; --i) {
      const int64_t t = t0 + i;
      if (t < a.time) {
        float vx = 0.f, vz = 0.f;
        if (t < n) {
          float f, g;
          gate(ld(z + t * a.z_stride_t), f, g);
          const float G = ld(dh + t * a.dh_stride_t) + r;
          vx = g * G;
          vz = f * g * G * (hp[i] - ld(x + t * a.x_stride_t));
          r = f * G;
        }
        st(dx + t * a.dx_stride_t, vx);
        if (part) part[(b * a.time + t) * D + c] = vz;
        else st(dz + t * a.dz_stride_t, vz);
      }
    }
  }
  if (a.dh0) a.dh0[b * D + c] = r;
}

// dz of a head: the sum of its channels' parts
template <typename T>
__global__ void k_recur_dz(pnn_recur_args a, const float* part) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, total = a.batch * a.time * a.heads;
  if (i >= total) return;
  const int64_t k = i % a.heads, bt = i / a.heads;
  const float* p = part + (bt * a.heads + k) * a.width;
  float s = 0.f;
  for (int64_t j = 0; j < a.width; ++j) s += p[j];
  st(static_cast<T*>(a.dz) + bt / a.time * a.dz_stride_b + bt % a.time * a.dz_stride_t + k, s);
}

template <typename T>
__global__ void k_recur_step(pnn_recur_step_args a) {
  const int64_t D = a.heads * a.width, c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, i = blockIdx.y;
  if (c >= D) return;
  const int64_t k = a.slot ? (int64_t)a.slot[i] : i;
  float v = 0.f;
  if (k >= 0 && k < a.slots) {
    float f, g;
    float* s = a.state + k * a.state_stride + c;
    gate(ld(static_cast<const T*>(a.z) + i * a.z_stride + c / a.width), f, g);
    v = f * *s + g * ld(static_cast<const T*>(a.x) + i * a.x_stride + c);
    *s = v;
  }
  st(static_cast<T*>(a.h) + i * a.h_stride + c, v);
}

dim3 grid_of(int64_t D, int64_t rows, int threads) { return dim3((unsigned)((D + threads - 1) / threads), (unsigned)rows); }
}  // namespace

size_t recur_saved_floats(const pnn_recur_args& a) {
  return (size_t)a.batch * ((a.time + kChunk - 1) / kChunk) * a.heads * a.width;
}
size_t recur_workspace(const pnn_recur_args& a) {
  return a.width > 1 ? (size_t)a.batch * a.time * a.heads * a.width * 4 : 0;
}

cudaError_t launch_recur_fwd(const pnn_recur_args& a, cudaStream_t st) {
  const dim3 g = grid_of(a.heads * a.width, a.batch, 64);
  if (a.dtype == PNN_DT_BF16) k_recur_fwd<bf16><<<g, 64, 0, st>>>(a);
  else k_recur_fwd<float><<<g, 64, 0, st>>>(a);
  return cudaGetLastError();
}

cudaError_t launch_recur_bwd(const pnn_recur_args& a, void* ws, cudaStream_t st) {
  const dim3 g = grid_of(a.heads * a.width, a.batch, 64);
  float* part = a.width > 1 ? static_cast<float*>(ws) : nullptr;
  if (a.dtype == PNN_DT_BF16) k_recur_bwd<bf16><<<g, 64, 0, st>>>(a, part);
  else k_recur_bwd<float><<<g, 64, 0, st>>>(a, part);
  if (part) {
    const dim3 gd = grid_of(a.batch * a.time * a.heads, 1, 256);
    if (a.dtype == PNN_DT_BF16) k_recur_dz<bf16><<<gd, 256, 0, st>>>(a, part);
    else k_recur_dz<float><<<gd, 256, 0, st>>>(a, part);
  }
  return cudaGetLastError();
}

cudaError_t launch_recur_step(const pnn_recur_step_args& a, cudaStream_t st) {
  const dim3 g = grid_of(a.heads * a.width, a.batch, 128);
  if (a.dtype == PNN_DT_BF16) k_recur_step<bf16><<<g, 128, 0, st>>>(a);
  else k_recur_step<float><<<g, 128, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace pnn
