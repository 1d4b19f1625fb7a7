// Embedding lookup with scaling, and its gradient by sorted tokens.
#include "pnn_internal.h"
#include "pnn_seq.h"
#include "seq_common.cuh"

namespace pnn {
namespace {
using namespace seq;

__device__ __forceinline__ int64_t token_id(const pnn_embed_args& a, int64_t n) {
  return a.ids_bits == 64 ? static_cast<const int64_t*>(a.ids)[n] : (int64_t)static_cast<const int32_t*>(a.ids)[n];
}

template <typename TI, typename TO>
__global__ void k_embed_fwd(pnn_embed_args a) {
  const int64_t n = blockIdx.x, v = token_id(a, n);
  const bool ok = v >= 0 && v < a.vocab;
  const TI* src = static_cast<const TI*>(a.table) + (ok ? v : 0) * a.table_stride;
  TO* dst = static_cast<TO*>(a.out) + n * a.out_stride;
  for (int64_t c = threadIdx.x; c < a.width; c += blockDim.x) st(dst + c, ok ? a.scale * ld(src + c) : 0.f);
}

// Stable sort of (id, position) by id, least significant digit first, by one
// CTA.  Each of the 32 warps owns a contiguous range of the tokens; a pass
// counts digits per warp, forms every warp's first place for every digit
// (digits in order, warps in order within a digit), and walks its range again
// to place each pair.  Padding sorts behind every id (key = vocab).
constexpr int kSortThreads = 1024, kDigit = 8, kBins = 1 << kDigit;

__global__ void k_embed_sort(pnn_embed_args a, uint2* buf0, uint2* buf1, int passes) {
  __shared__ uint32_t cnt[kSortThreads / 32][kBins];
  __shared__ uint32_t tot[kBins];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, nw = kSortThreads / 32;
  const int64_t N = a.tokens, per = ((N + nw * 32 - 1) / (nw * 32)) * 32;
  const int64_t lo = warp * per < N ? warp * per : N, hi = lo + per < N ? lo + per : N;
  for (int64_t i = threadIdx.x; i < N; i += kSortThreads) {
    const int64_t v = token_id(a, i);
    buf0[i] = make_uint2(v >= 0 && v < a.vocab ? (uint32_t)v : (uint32_t)a.vocab, (uint32_t)i);
  }
  __syncthreads();
  for (int p = 0; p < passes; ++p) {
    const uint2* in = p & 1 ? buf1 : buf0;
    uint2* out = p & 1 ? buf0 : buf1;
    for (int i = threadIdx.x; i < nw * kBins; i += kSortThreads) cnt[i / kBins][i % kBins] = 0;
    __syncthreads();
    for (int64_t i = lo + lane; i < hi; i += 32) atomicAdd(&cnt[warp][(in[i].x >> (p * kDigit)) & (kBins - 1)], 1u);
    __syncthreads();
    if (threadIdx.x < kBins) {
      uint32_t s = 0;
      for (int w = 0; w < nw; ++w) { const uint32_t c = cnt[w][threadIdx.x]; cnt[w][threadIdx.x] = s; s += c; }
      tot[threadIdx.x] = s;
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t s = 0;
      for (int i = 0; i < kBins; ++i) { const uint32_t c = tot[i]; tot[i] = s; s += c; }
    }
    __syncthreads();
    for (int64_t i0 = lo; i0 < hi; i0 += 32) {
      const int64_t i = i0 + lane;
      const bool on = i < hi;
      const uint2 v = on ? in[i] : make_uint2(0, 0);
      const uint32_t d = on ? (v.x >> (p * kDigit)) & (kBins - 1) : 0xffffffffu;
      const uint32_t same = __match_any_sync(0xffffffffu, d), before = __popc(same & ((1u << lane) - 1));
      uint32_t at = on ? tot[d] + cnt[warp][d] + before : 0;
      __syncwarp();
      if (on && before == 0) cnt[warp][d] += __popc(same);
      __syncwarp();
      if (on) out[at] = v;
    }
    __syncthreads();
  }
}

// One CTA a row of the table: its run in the sorted pairs, added in order.
template <typename TI, typename TO>
__global__ void k_embed_sum(pnn_embed_args a, const uint2* sorted) {
  const uint32_t v = blockIdx.x;
  auto first = [&](uint32_t key) {  // first place whose id is >= key
    int64_t lo = 0, hi = a.tokens;
    while (lo < hi) {
      const int64_t mid = (lo + hi) / 2;
      if (sorted[mid].x < key) lo = mid + 1;
      else hi = mid;
    }
    return lo;
  };
  const int64_t b = first(v), e = first(v + 1);
  TO* dst = static_cast<TO*>(a.dtable) + (int64_t)v * a.dtable_stride;
  if (a.accumulate && b == e) return;
  for (int64_t c = threadIdx.x; c < a.width; c += blockDim.x) {
    float s = 0.f;
    for (int64_t i = b; i < e; ++i) s += ld(static_cast<const TI*>(a.dout) + (int64_t)sorted[i].y * a.dout_stride + c);
    s *= a.scale;
    if (a.accumulate) s += ld(dst + c);
    st(dst + c, s);
  }
}
}  // namespace

cudaError_t launch_embed_fwd(const pnn_embed_args& a, cudaStream_t st) {
  const unsigned g = (unsigned)a.tokens;
  const bool ti = a.table_dtype == PNN_DT_BF16, to = a.out_dtype == PNN_DT_BF16;
  if (ti && to) k_embed_fwd<bf16, bf16><<<g, 256, 0, st>>>(a);
  else if (ti) k_embed_fwd<bf16, float><<<g, 256, 0, st>>>(a);
  else if (to) k_embed_fwd<float, bf16><<<g, 256, 0, st>>>(a);
  else k_embed_fwd<float, float><<<g, 256, 0, st>>>(a);
  return cudaGetLastError();
}

size_t embed_workspace(const pnn_embed_args& a) { return (size_t)a.tokens * 16; }

cudaError_t launch_embed_bwd(const pnn_embed_args& a, void* ws, cudaStream_t st) {
  uint2 *b0 = static_cast<uint2*>(ws), *b1 = b0 + a.tokens;
  int passes = 0;
  for (int64_t v = a.vocab; v; v >>= kDigit) ++passes;
  k_embed_sort<<<1, kSortThreads, 0, st>>>(a, b0, b1, passes);
  const uint2* s = passes & 1 ? b1 : b0;
  const unsigned g = (unsigned)a.vocab;
  const bool ti = a.dout_dtype == PNN_DT_BF16, to = a.dtable_dtype == PNN_DT_BF16;
  if (ti && to) k_embed_sum<bf16, bf16><<<g, 256, 0, st>>>(a, s);
  else if (ti) k_embed_sum<bf16, float><<<g, 256, 0, st>>>(a, s);
  else if (to) k_embed_sum<float, bf16><<<g, 256, 0, st>>>(a, s);
  else k_embed_sum<float, float><<<g, 256, 0, st>>>(a, s);
  return cudaGetLastError();
}

}  // namespace pnn
