// Distillation from a teacher's top logits mixed with the labels' cross
// entropy: loss and gradient of one row by one CTA.
#include <math.h>

#include "pnn_internal.h"
#include "pnn_seq.h"
#include "seq_common.cuh"

namespace pnn {
namespace {
using namespace seq;

constexpr int kThreads = 256;

template <bool MAX>
__device__ __forceinline__ float block_reduce(float v, float* red) {
  for (int o = 16; o; o >>= 1) {
    const float u = __shfl_xor_sync(0xffffffffu, v, o);
    v = MAX ? fmaxf(v, u) : v + u;
  }
  __syncthreads();
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = v;
  __syncthreads();
  v = red[0];
  for (int i = 1; i < kThreads / 32; ++i) v = MAX ? fmaxf(v, red[i]) : v + red[i];
  return v;
}

template <typename T, typename TT>
__global__ void k_distill(pnn_distill_args a) {
  __shared__ float red[kThreads / 32];
  __shared__ int id[1024];
  __shared__ float p[1024], sv[1024];
  const int64_t row = blockIdx.x;
  const int V = (int)a.vocab, tid = threadIdx.x;
  const T* s = static_cast<const T*>(a.logits) + row * a.logits_stride;
  const float it = 1.f / a.tau;

  float m = -INFINITY;
  for (int v = tid; v < V; v += kThreads) m = fmaxf(m, ld(s + v));
  m = block_reduce<true>(m, red);
  if (m == -INFINITY) m = 0.f;
  float s1 = 0.f, st_ = 0.f;
  for (int v = tid; v < V; v += kThreads) {
    const float y = ld(s + v) - m;
    s1 += __expf(y);
    st_ += __expf(y * it);
  }
  s1 = block_reduce<false>(s1, red);
  st_ = block_reduce<false>(st_, red);

  // the teacher's softmax over the pairs that are there
  const TT* t = static_cast<const TT*>(a.teacher) + row * a.k;
  float mt = -INFINITY;
  for (int j = tid; j < a.k; j += kThreads) {
    const int v = a.ids[row * a.k + j];
    const bool ok = v >= 0 && v < V;
    id[j] = ok ? v : -1;
    p[j] = ok ? ld(t + j) : -INFINITY;
    sv[j] = ok ? ld(s + v) : 0.f;
    mt = fmaxf(mt, p[j]);
  }
  mt = block_reduce<true>(mt, red);
  if (mt == -INFINITY) mt = 0.f;
  float w = 0.f;
  for (int j = tid; j < a.k; j += kThreads) w += __expf((p[j] - mt) * it);
  w = block_reduce<false>(w, red);
  const int label = a.labels ? a.labels[row] : -1;
  const bool soft = a.alpha > 0.f && w != 0.f && st_ != 0.f;
  const bool hard = a.alpha < 1.f && label >= 0 && label < V && s1 != 0.f;
  const float slabel = hard ? ld(s + label) : 0.f;
  float loss = 0.f;
  for (int j = tid; j < a.k; j += kThreads) {
    const float y = (p[j] - mt) * it, q = __expf(y) / w;
    if (soft && q != 0.f) loss += q * ((y - logf(w)) - ((sv[j] - m) * it - logf(st_)));
    p[j] = q;
  }
  loss = block_reduce<false>(loss, red);
  if (tid == 0) {
    float l = 0.f;
    if (soft) l += a.alpha * a.tau * a.tau * loss;
    if (hard) l += (1.f - a.alpha) * (logf(s1) - (slabel - m));
    a.loss[row] = l;
  }
  if (!a.dlogits) return;
  T* d = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
  const float wt = a.weight ? a.weight[row] : 1.f;
  const float ct = a.alpha * a.tau, ch = 1.f - a.alpha;
  auto grad = [&](float x, float pt, bool hot) {
    float v = 0.f;
    if (soft) v += ct * (__expf((x - m) * it) / st_ - pt);
    if (hard) v += ch * (__expf(x - m) / s1 - (hot ? 1.f : 0.f));
    return wt * v;
  };
  for (int v = tid; v < V; v += kThreads) st(d + v, soft || hard ? grad(ld(s + v), 0.f, v == label) : 0.f);
  __syncthreads();
  if (soft)
    for (int j = tid; j < a.k; j += kThreads)
      if (id[j] >= 0) {
        float sum = 0.f;
        for (int i = 0; i < a.k; ++i) sum += id[i] == id[j] ? p[i] : 0.f;
        st(d + id[j], grad(sv[j], sum, id[j] == label));
      }
}
}  // namespace

cudaError_t launch_distill(const pnn_distill_args& a, cudaStream_t st) {
  const dim3 g((unsigned)a.rows);
  if (a.dtype == PNN_DT_BF16) {
    if (a.teacher_dtype == PNN_DT_BF16) k_distill<bf16, bf16><<<g, kThreads, 0, st>>>(a);
    else k_distill<bf16, float><<<g, kThreads, 0, st>>>(a);
  } else {
    if (a.teacher_dtype == PNN_DT_BF16) k_distill<float, bf16><<<g, kThreads, 0, st>>>(a);
    else k_distill<float, float><<<g, kThreads, 0, st>>>(a);
  }
  return cudaGetLastError();
}

}  // namespace pnn
