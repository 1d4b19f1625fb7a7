// Distillation from a teacher's top logits mixed with the labels' cross
// entropy: loss and gradient in one pass over the logits.
//
// A team of threads (a warp, a CTA, or a cluster of CTAs) holds one row in its
// registers: the row is read once, every warp forms the softmax sums from its
// own maximum, the warps' (maximum, sums) meet once in shared memory
//   S = sum_w s_w exp((m_w - m) / tau),
// and the gradient is written from the registers.  The row's few places that
// the teacher or the label names are written again after that with what they
// take off; pairs of the same id add up in the order of the list.
//
// Bound: HBM (one read, one write of the row), and the exponentials, two for
// an element at each temperature.
#include <math.h>

#include "pnn_internal.h"
#include "pnn_seq.h"
#include "seq_common.cuh"

namespace pnn {
namespace {
using namespace seq;

constexpr int kVecs = 8;          // 16-byte vectors of a thread: 32 registers of logits
constexpr int kMaxCluster = 8;

// ---------------------------------------------------------------- small pieces
using f2 = unsigned long long;
__device__ __forceinline__ f2 pk(float a, float b) {
  f2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void upk(f2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f2 mul2(f2 a, f2 b) {
  f2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 add2(f2 a, f2 b) {
  f2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f2 fma2(f2 a, f2 b, f2 c) {
  f2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
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

// A maximum with the sums of exp((s - m) / tau) and exp(s - m) from it.  No
// value yet, or only masked ones: m = -inf and sums 0.
struct Stat {
  float m, t, h;
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
__device__ __forceinline__ Stat merge(const Stat& a, const Stat& b, float kt) {
  const float m = fmaxf(a.m, b.m), s = base_of(m);
  return Stat{m, a.t * ex2((a.m - s) * kt) + b.t * ex2((b.m - s) * kt), a.h * ex2((a.m - s) * kLog2e) + b.h * ex2((b.m - s) * kLog2e)};
}
__device__ __forceinline__ Stat merge_warp(Stat s, float kt) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
    s = merge(s, Stat{__shfl_xor_sync(0xffffffffu, s.m, o), __shfl_xor_sync(0xffffffffu, s.t, o), __shfl_xor_sync(0xffffffffu, s.h, o)}, kt);
  return s;
}

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

// A pair of the teacher, or the label, as a place of the row.
struct Entry {
  int id;
  float t, s;  // the teacher's logit (then its probability), the student's
};

// TEAM threads a row; a CTA of 128 threads has four warp-wide teams.  TWO: the
// teacher's term and the label's need the softmax at two temperatures.
template <typename T, int TEAM, bool TWO, bool CL>
__global__ void __launch_bounds__(TEAM == 32 ? 128 : TEAM) k_distill(const __grid_constant__ pnn_distill_args a, int C) {
  constexpr int E = 16 / sizeof(T), P = kPairs<T>, W = TEAM / 32;
  extern __shared__ Entry entries[];
  __shared__ float4 stats[TEAM == 32 ? 1 : (CL ? kMaxCluster : 1) * W];
  const int tid = threadIdx.x % TEAM, team = threadIdx.x / TEAM, warp = tid >> 5, lane = threadIdx.x & 31;
  const int rank = CL ? (int)cluster_rank() : 0;
  const int64_t row = CL ? blockIdx.x / C : (int64_t)blockIdx.x * (TEAM == 32 ? 4 : 1) + team;
  if (CL) asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  if (TEAM == 32 && row >= a.rows) return;
  const int V = (int)a.vocab, K = a.k;
  const T* s = static_cast<const T*>(a.logits) + row * a.logits_stride;
  Entry* ent = entries + team * (K + 1);
  const float it = 1.f / a.tau;

  // this CTA's 16-byte vectors of the row; the values before the first boundary and behind the last are rank 0's
  const int off = (int)((reinterpret_cast<uintptr_t>(s) & 15) / sizeof(T));
  const int head = off ? (E - off < V ? E - off : V) : 0, all = (V - head) / E, tail = V - head - all * E;
  const int each = CL ? (all + C - 1) / C : all;
  const int v0 = rank * each < all ? rank * each : all, nv = each < all - v0 ? each : all - v0;
  const uint4* vec = reinterpret_cast<const uint4*>(s + head) + v0;
  const int chunks = (nv + kVecs * TEAM - 1) / (kVecs * TEAM);  // 1: the row stays in registers

  // the single values: lanes 0 .. head - 1 of the first warp, and E .. E + tail - 1
  const int lone = rank == 0 ? (tid < head ? tid : tid >= E && tid < E + tail ? head + all * E + tid - E : -1) : -1;
  uint4 x[kVecs];
  auto load = [&](int c) {
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int j = (c * kVecs + i) * TEAM + tid;
      x[i] = j < nv ? ld_once(vec + j) : minus_inf<T>();
    }
  };
  load(0);
  const float one = lone >= 0 ? ld(s + lone) : -INFINITY;
  // the teacher's pairs and the label (entry K)
  const bool teach = K > 0 && a.alpha > 0.f;
  const int label = a.labels && a.alpha < 1.f ? a.labels[row] : -1;
  for (int j = tid; j <= K; j += TEAM) {
    int id = j < K ? (teach ? a.ids[row * K + j] : -1) : label;
    if (id < 0 || id >= V) id = -1;
    float t = -INFINITY;
    if (j < K && id >= 0)
      t = a.teacher_dtype == PNN_DT_BF16 ? ld(static_cast<const bf16*>(a.teacher) + row * K + j) : ld(static_cast<const float*>(a.teacher) + row * K + j);
    ent[j] = Entry{id, t, id >= 0 ? ld(s + id) : 0.f};
  }

  // sums at k = log2(e) / tau; TWO: also at log2(e)
  const float kt = (teach ? it : 1.f) * kLog2e;
  Stat st{-INFINITY, 0.f, 0.f};
  for (int c = 0; c < chunks || c == 0; ++c) {
    if (c) load(c);
    float m = c ? -INFINITY : one;
#pragma unroll
    for (int i = 0; i < kVecs; ++i) m = fmaxf(m, max_of<T>(x[i]));
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float b = base_of(m);
    const f2 nb = pk(-b, -b), k2 = pk(kt, kt), k1 = pk(kLog2e, kLog2e);
    f2 at = 0, ah = 0;
#pragma unroll
    for (int i = 0; i < kVecs; ++i)
      if ((c * kVecs + i) * TEAM < nv) {
#pragma unroll
        for (int p = 0; p < P; ++p) {
          const f2 y = add2(pair_of<T>(x[i], p), nb);
          at = add2(at, ex2p(mul2(y, k2)));
          if (TWO) ah = add2(ah, ex2p(mul2(y, k1)));
        }
      }
    float t0, t1, h0, h1;
    upk(at, t0, t1);
    upk(ah, h0, h1);
    if (c == 0 && lone >= 0) {
      t0 += ex2((one - b) * kt);
      if (TWO) h0 += ex2((one - b) * kLog2e);
    }
    const Stat mine{m, t0 + t1, h0 + h1};
    st = c ? merge(st, mine, kt) : mine;
  }
  // all lanes have the warp's maximum: plain sums
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    st.t += __shfl_xor_sync(0xffffffffu, st.t, o);
    if (TWO) st.h += __shfl_xor_sync(0xffffffffu, st.h, o);
  }
  if (TEAM == 32) {
    __syncwarp();
  } else {
    if (CL) {
      asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // every peer has started
      if (lane < C) put_remote(&stats[rank * W + warp], lane, make_float4(st.m, st.t, st.h, 0.f));
      asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
      if (lane == 0) stats[warp] = make_float4(st.m, st.t, st.h, 0.f);
      __syncthreads();
    }
    st = Stat{-INFINITY, 0.f, 0.f};
    for (int i = lane; i < (CL ? C : 1) * W; i += 32) st = merge(st, Stat{stats[i].x, stats[i].y, stats[i].z}, kt);
    st = merge_warp(st, kt);
  }
  if (!TWO) st.h = st.t;  // one temperature serves both terms (tau = 1, or only one term)

  // the teacher's softmax over the pairs that are there, by every warp for itself
  float mt = -INFINITY, w = 0.f;
  for (int j = lane; j < K; j += 32) mt = fmaxf(mt, ent[j].t);
#pragma unroll
  for (int o = 16; o; o >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, o));
  mt = base_of(mt);
  for (int j = lane; j < K; j += 32) w += ex2((ent[j].t - mt) * kt);
#pragma unroll
  for (int o = 16; o; o >>= 1) w += __shfl_xor_sync(0xffffffffu, w, o);
  const float base = base_of(st.m);
  const bool soft = teach && w != 0.f && st.t != 0.f, hard = ent[K].id >= 0 && st.h != 0.f;

  if (rank == 0 && warp == 0) {
    float sum = 0.f;
    if (soft) {
      const float lw = log2f(w), ls = log2f(st.t);
      for (int j = lane; j < K; j += 32) {
        const float y = (ent[j].t - mt) * kt, p = ex2(y);
        if (p != 0.f) sum += p * ((y - lw) - ((ent[j].s - base) * kt - ls));
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    if (lane == 0) {
      float l = 0.f;
      if (soft) l = a.alpha * a.tau * a.tau * (kLn2 * (sum / w));
      if (hard) l += (1.f - a.alpha) * (logf(st.h) - (ent[K].s - base));
      a.loss[row] = l;
    }
  }
  if (!a.dlogits) return;

  // gradient = gt exp((s - m) / tau) + gh exp(s - m), then what the entries take off
  const float wt = a.weight ? a.weight[row] : 1.f;
  const float ct = soft ? wt * a.alpha * a.tau : 0.f, ch = hard ? wt * (1.f - a.alpha) : 0.f;
  const float gt = (TWO || soft ? ct / (soft ? st.t : 1.f) : 0.f) + (!TWO && hard ? ch / st.h : 0.f), gh = TWO && hard ? ch / st.h : 0.f;
  const bool none = !soft && !hard;
  auto grad = [&](float v) {
    const float y = v - base;
    float g = gt != 0.f || !TWO ? gt * ex2(y * kt) : 0.f;
    if (TWO && gh != 0.f) g = fmaf(gh, ex2(y * kLog2e), g);
    return none ? 0.f : g;
  };
  T* d = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
  const bool same = ((reinterpret_cast<uintptr_t>(d) ^ reinterpret_cast<uintptr_t>(s)) & 15) == 0;  // the same vectors
  const f2 nb = pk(-base, -base), k2 = pk(kt, kt), k1 = pk(kLog2e, kLog2e), gt2 = pk(gt, gt), gh2 = pk(gh, gh);
  for (int c = 0; c < chunks; ++c) {
    if (chunks > 1) load(c);
#pragma unroll
    for (int i = 0; i < kVecs; ++i) {
      const int j = (c * kVecs + i) * TEAM + tid;
      if (j >= nv) continue;
      float g[E];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        f2 v = 0;
        if (!none) {
          const f2 y = add2(pair_of<T>(x[i], p), nb);
          v = mul2(gt2, ex2p(mul2(y, k2)));
          if (TWO) v = fma2(gh2, ex2p(mul2(y, k1)), v);
        }
        upk(v, g[2 * p], g[2 * p + 1]);
      }
      T* to = d + head + (int64_t)(v0 + j) * E;
      if (same) {
        uint4 o;
        if constexpr (sizeof(T) == 2) {
          __nv_bfloat162* h = reinterpret_cast<__nv_bfloat162*>(&o);
#pragma unroll
          for (int p = 0; p < P; ++p) h[p] = __floats2bfloat162_rn(g[2 * p], g[2 * p + 1]);
        } else {
          o = make_uint4(__float_as_uint(g[0]), __float_as_uint(g[1]), __float_as_uint(g[2]), __float_as_uint(g[3]));
        }
        *reinterpret_cast<uint4*>(to) = o;
      } else {
#pragma unroll
        for (int p = 0; p < E; ++p) ::pnn::seq::st(to + p, g[p]);
      }
    }
  }
  if (lone >= 0) ::pnn::seq::st(d + lone, grad(one));
  // The places that entries name, each in the CTA that has just written it.
  if (none) return;
  if (TEAM == 32) __syncwarp();
  else __syncthreads();
  const float rw = soft ? ct / w : 0.f;
  for (int j = tid; j <= K; j += TEAM) {
    const int id = ent[j].id;
    if (id < 0) continue;
    if (CL) {  // whose?
      const int p = id - head;
      const int owner = p < 0 || p >= all * E ? 0 : p / E / each;
      if (owner != rank) continue;
    }
    float off_ = 0.f;
    if (soft)
      for (int i = 0; i < K; ++i)
        if (ent[i].id == id) off_ += ex2((ent[i].t - mt) * kt);
    float g = grad(ent[j].s) - rw * off_;
    if (hard && id == ent[K].id) g -= ch;
    ::pnn::seq::st(d + id, g);
  }
}

template <typename T, int TEAM, bool TWO, bool CL>
cudaError_t launch(const pnn_distill_args& a, int C, cudaStream_t st) {
  cudaLaunchConfig_t cfg = {};
  const int teams = TEAM == 32 ? 4 : 1;
  cfg.gridDim = dim3((unsigned)(TEAM == 32 ? (a.rows + 3) / 4 : a.rows * C));
  cfg.blockDim = dim3(TEAM == 32 ? 128 : TEAM);
  cfg.dynamicSmemBytes = (size_t)(a.k + 1) * sizeof(Entry) * teams;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = C > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, k_distill<T, TEAM, TWO, CL>, a, C);
}

// The smallest team whose registers hold the row: a warp (2048 bf16 values), a
// CTA of 128 or 512 threads (8192, 32768), a cluster of up to 8 such CTAs;
// longer rows are read a second time for the gradient.
template <typename T, bool TWO>
cudaError_t pick(const pnn_distill_args& a, cudaStream_t st) {
  const int64_t per = kVecs * 16 / sizeof(T), n = a.vocab;
  if (n <= 32 * per && a.k <= 512) return launch<T, 32, TWO, false>(a, 1, st);
  if (n <= 128 * per) return launch<T, 128, TWO, false>(a, 1, st);
  int C = 1;
  while (C < kMaxCluster && C * 512 * per < n) C *= 2;
  return C > 1 ? launch<T, 512, TWO, true>(a, C, st) : launch<T, 512, TWO, false>(a, 1, st);
}
}  // namespace

cudaError_t launch_distill(const pnn_distill_args& a, cudaStream_t st) {
  const bool two = a.k > 0 && a.alpha > 0.f && a.labels && a.alpha < 1.f && a.tau != 1.f;
  if (a.dtype == PNN_DT_BF16) return two ? pick<bf16, true>(a, st) : pick<bf16, false>(a, st);
  return two ? pick<float, true>(a, st) : pick<float, false>(a, st);
}

}  // namespace pnn
