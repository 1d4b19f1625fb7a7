// Gated linear recurrence: forward scan, backward pass, single-token step.
//
// The scan and backward pass here take rows of any alignment and heads of any
// width; rows that a tensor map can describe go to the tiled form
// (k_recur_tile.cu, which also states the mathematics).  A CTA takes 32
// channels and a piece of 8 runs of time steps at a time: each thread solves
// its run of one or two channels from zero out of registers while the next
// piece is loaded, one warp composes the runs along time and hands every
// thread its true first state, and the threads run their steps again from it.
// With few (sequence, tile) pairs a cluster of CTAs shares one, exchanging the
// pieces' results through distributed shared memory.
#include <algorithm>

#include "pnn_internal.h"
#include "pnn_seq.h"
#include "recur_common.cuh"
#include "seq_common.cuh"

namespace pnn {
namespace {
using namespace seq;

constexpr int kTile = 32, kGroups = 8, kMaxCluster = 16;
template <int V>
constexpr int kThreads = kGroups * kTile / V;
template <typename T>
constexpr int kPiece = kGroups * kRunSteps<T>;

// CTAs an SM holds: what leaves each thread the registers of its arrays
template <int V>
constexpr int kFwdCtas = 3 * V;
template <int V>
constexpr int kBwdCtas = 2 * V;

// V neighbouring values as they lie in memory
template <typename T, int V> struct Raw;
template <> struct Raw<bf16, 2> {
  uint32_t v;
  __device__ void load(const bf16* p) { v = *reinterpret_cast<const uint32_t*>(p); }
  __device__ void fill(float a) { const __nv_bfloat162 h = __float2bfloat162_rn(a); v = *reinterpret_cast<const uint32_t*>(&h); }
  __device__ float at(int i) const { return __uint_as_float(i ? v & 0xffff0000u : v << 16); }
  static __device__ void store(bf16* p, const float* a) { *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(a[0], a[1]); }
};
template <> struct Raw<bf16, 1> {
  bf16 v;
  __device__ void load(const bf16* p) { v = *p; }
  __device__ void fill(float a) { v = __float2bfloat16_rn(a); }
  __device__ float at(int) const { return __bfloat162float(v); }
  static __device__ void store(bf16* p, const float* a) { *p = __float2bfloat16_rn(a[0]); }
};
template <> struct Raw<float, 2> {
  float2 v;
  __device__ void load(const float* p) { v = *reinterpret_cast<const float2*>(p); }
  __device__ void fill(float a) { v = make_float2(a, a); }
  __device__ float at(int i) const { return i ? v.y : v.x; }
  static __device__ void store(float* p, const float* a) { *reinterpret_cast<float2*>(p) = make_float2(a[0], a[1]); }
};
template <> struct Raw<float, 1> {
  float v;
  __device__ void load(const float* p) { v = *p; }
  __device__ void fill(float a) { v = a; }
  __device__ float at(int) const { return v; }
  static __device__ void store(float* p, const float* a) { *p = a[0]; }
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// 8 bytes into the same shared-memory place of CTA `rank` of the cluster
__device__ __forceinline__ void put_remote(const float2* place, uint32_t rank, float2 v) {
  uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(place)), to;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(at), "r"(rank));
  asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(to), "f"(v.x), "f"(v.y) : "memory");
}

// The place of a thread: its channels, its group along time.
template <int V>
struct Place {
  int group, lane;      // lane: which V channels of the tile
  int64_t c, D;         // first channel, all channels
  bool on;
  __device__ Place(int64_t D_, int64_t tile) : group(threadIdx.x / (kTile / V)), lane(threadIdx.x % (kTile / V)), D(D_) {
    c = tile * kTile + lane * V;
    on = c < D;
  }
};

// SH: a gate is shared by `width` channels.  CL: a cluster of C CTAs a tile.
template <typename T, int V, bool SH, bool CL>
__global__ void __launch_bounds__(kThreads<V>, kFwdCtas<V>) k_recur_fwd(pnn_recur_args a, int C) {
  constexpr int S = kRunSteps<T>, G = kGroups, L = kPiece<T>;
  __shared__ float2 agg[G][kTile];
  __shared__ float first[G][kTile];
  __shared__ float2 peer[CL ? 2 : 1][CL ? kMaxCluster : 1][kTile];
  const int rank = CL ? (int)cluster_rank() : 0;
  const int64_t b = blockIdx.y;
  const Place<V> p(a.heads * a.width, CL ? blockIdx.x / C : blockIdx.x);
  const int n = recur_len(a, b), span = L * C;
  const int64_t pieces = (a.time + L - 1) / L;
  const int off = rank * L + p.group * S;  // this thread's first step of a round
  using RZ = Raw<T, SH ? 1 : V>;
  using RX = Raw<T, V>;
  RZ z[S];
  RX x[S];
  const T* zp = static_cast<const T*>(a.z) + b * a.z_stride_b + (SH ? p.c / a.width : p.c) + off * a.z_stride_t;
  const T* xp = static_cast<const T*>(a.x) + b * a.x_stride_b + p.c + off * a.x_stride_t;
  T* hp = static_cast<T*>(a.h) + b * a.h_stride_b + p.c + off * a.h_stride_t;
  // steps behind the end keep the state: gate +inf, input 0
  auto load = [&](int64_t t) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      z[i].fill(INFINITY);
      x[i].fill(0.f);
      if (p.on && t + i < n) {
        z[i].load(zp + i * a.z_stride_t);
        x[i].load(xp + i * a.x_stride_t);
      }
    }
    zp += span * a.z_stride_t;
    xp += span * a.x_stride_t;
  };
  load(off);
  // warp 0 carries the state of the tile's channels, one a lane
  const int64_t cj = (CL ? blockIdx.x / C : blockIdx.x) * (int64_t)kTile + (threadIdx.x & 31);
  const bool join = threadIdx.x < 32;
  float s = join && a.h0 && cj < p.D ? a.h0[b * p.D + cj] : 0.f;
  if (CL) cluster_sync();  // every CTA of the cluster runs before its shared memory is written
  int buf = 0;
  for (int64_t t0 = 0; t0 < a.time; t0 += span) {
    const int64_t t = t0 + off;
    if (t0 >= n) {  // the whole round lies behind the end
      const float zero[V] = {};
#pragma unroll
      for (int i = 0; i < S; ++i)
        if (p.on && t + i < a.time) RX::store(hp + i * a.h_stride_t, zero);
      hp += span * a.h_stride_t;
      continue;
    }
    float f[S][V], u[S][V], A[V], B[V];
#pragma unroll
    for (int v = 0; v < V; ++v) A[v] = 1.f, B[v] = 0.f;
#pragma unroll
    for (int i = 0; i < S; ++i) {
      float g;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        if (SH && v) f[i][v] = f[i][0];
        else gate(z[i].at(v), f[i][v], g);
        u[i][v] = g * x[i].at(v);
        A[v] *= f[i][v];
        B[v] = fmaf(f[i][v], B[v], u[i][v]);
      }
    }
    load(t + span);
#pragma unroll
    for (int v = 0; v < V; ++v) agg[p.group][p.lane * V + v] = make_float2(A[v], B[v]);
    __syncthreads();
    if (CL) {
      if (join) {
        float2 m = make_float2(1.f, 0.f);
#pragma unroll
        for (int g = 0; g < G; ++g) {
          const float2 q = agg[g][threadIdx.x];
          m = make_float2(q.x * m.x, fmaf(q.x, m.y, q.y));
        }
        for (int r = 0; r < C; ++r) put_remote(&peer[buf][rank][threadIdx.x], r, m);
      }
      cluster_sync();
    }
    if (join) {
      float q = s;
      if (CL)
        for (int r = 0; r < rank; ++r) q = fmaf(peer[buf][r][threadIdx.x].x, q, peer[buf][r][threadIdx.x].y);
      const int64_t piece = t0 / L + rank;
      if (a.saved && cj < p.D && piece < pieces) a.saved[(b * pieces + piece) * p.D + cj] = q;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        first[g][threadIdx.x] = q;
        q = fmaf(agg[g][threadIdx.x].x, q, agg[g][threadIdx.x].y);
      }
      if (CL)
        for (int r = rank + 1; r < C; ++r) q = fmaf(peer[buf][r][threadIdx.x].x, q, peer[buf][r][threadIdx.x].y);
      s = q;
    }
    __syncthreads();
    float h[V];
#pragma unroll
    for (int v = 0; v < V; ++v) h[v] = first[p.group][p.lane * V + v];
#pragma unroll
    for (int i = 0; i < S; ++i) {
      float w[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        h[v] = fmaf(f[i][v], h[v], u[i][v]);
        w[v] = t + i < n ? h[v] : 0.f;
      }
      if (p.on && t + i < a.time) RX::store(hp + i * a.h_stride_t, w);
    }
    hp += span * a.h_stride_t;
    buf ^= 1;
  }
  if (join && rank == 0 && a.h_last && cj < p.D) a.h_last[b * p.D + cj] = s;
}

// part: where a head spans several groups of `part_width` channels, the fp32
// sums of dz over each group, [batch][time][channels / part_width]; else NULL.
// part_width: channels whose dz is summed here (1, 16 or 32).
template <typename T, int V, bool SH, bool CL>
__global__ void __launch_bounds__(kThreads<V>, kBwdCtas<V>) k_recur_bwd(pnn_recur_args a, int C, float* part, int part_width) {
  constexpr int S = kRunSteps<T>, G = kGroups, L = kPiece<T>;
  __shared__ float2 aggf[G][kTile], aggb[G][kTile];
  __shared__ float first[G][kTile], last[G][kTile];
  __shared__ float2 peer[CL ? 2 : 1][CL ? kMaxCluster : 1][kTile];
  const int rank = CL ? (int)cluster_rank() : 0;
  const int64_t b = blockIdx.y;
  const Place<V> p(a.heads * a.width, CL ? blockIdx.x / C : blockIdx.x);
  const int n = recur_len(a, b), span = L * C;
  const int64_t pieces = (a.time + L - 1) / L, rounds = (a.time + span - 1) / span;
  using RZ = Raw<T, SH ? 1 : V>;
  using RX = Raw<T, V>;
  RZ z[S];
  RX x[S], d[S];
  const int64_t tl = (rounds - 1) * span + rank * L + p.group * S;  // first step of the last round
  const T* zp = static_cast<const T*>(a.z) + b * a.z_stride_b + (SH ? p.c / a.width : p.c) + tl * a.z_stride_t;
  const T* xp = static_cast<const T*>(a.x) + b * a.x_stride_b + p.c + tl * a.x_stride_t;
  const T* dp = static_cast<const T*>(a.dh) + b * a.dh_stride_b + p.c + tl * a.dh_stride_t;
  T* dxp = static_cast<T*>(a.dx) + b * a.dx_stride_b + p.c + tl * a.dx_stride_t;
  T* dzp = static_cast<T*>(a.dz) + b * a.dz_stride_b + (SH ? p.c / a.width : p.c) + tl * a.dz_stride_t;
  auto load = [&](int64_t t) {
#pragma unroll
    for (int i = 0; i < S; ++i) {
      z[i].fill(INFINITY);
      x[i].fill(0.f);
      d[i].fill(0.f);
      if (p.on && t >= 0 && t + i < n) {
        z[i].load(zp + i * a.z_stride_t);
        x[i].load(xp + i * a.x_stride_t);
        d[i].load(dp + i * a.dh_stride_t);
      }
    }
    zp -= span * a.z_stride_t;
    xp -= span * a.x_stride_t;
    dp -= span * a.dh_stride_t;
  };
  load(tl);
  // warp 0 joins the states, warp 1 the gradients R, one channel a lane
  const int jl = threadIdx.x & 31;
  const int64_t cj = (CL ? blockIdx.x / C : blockIdx.x) * (int64_t)kTile + jl;
  const bool joinf = threadIdx.x < 32, joinb = threadIdx.x >= 32 && threadIdx.x < 64;
  float r = joinb && a.dh_last && cj < p.D ? a.dh_last[b * p.D + cj] : 0.f;
  if (CL) cluster_sync();
  int buf = 0;
  for (int64_t k = rounds - 1; k >= 0; --k) {
    const int64_t t = k * span + rank * L + p.group * S;
    const bool live = k * span < n;
    float f[S][V], g[S][V], xv[S][V], dv[S][V];
    if (live) {
      float A[V], Bf[V], Bb[V];
#pragma unroll
      for (int v = 0; v < V; ++v) A[v] = 1.f, Bf[v] = 0.f, Bb[v] = 0.f;
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          if (SH && v) f[i][v] = f[i][0], g[i][v] = g[i][0];
          else gate(z[i].at(v), f[i][v], g[i][v]);
          xv[i][v] = x[i].at(v);
          dv[i][v] = d[i].at(v);
          A[v] *= f[i][v];
          Bf[v] = fmaf(f[i][v], Bf[v], g[i][v] * xv[i][v]);
        }
#pragma unroll
      for (int i = S - 1; i >= 0; --i)
#pragma unroll
        for (int v = 0; v < V; ++v) Bb[v] = f[i][v] * (dv[i][v] + Bb[v]);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        aggf[p.group][p.lane * V + v] = make_float2(A[v], Bf[v]);
        aggb[p.group][p.lane * V + v] = make_float2(A[v], Bb[v]);
      }
    }
    load(t - span);
    if (live) {
      __syncthreads();
      if (CL) {
        if (joinb) {
          float2 m = make_float2(1.f, 0.f);
#pragma unroll
          for (int q = G - 1; q >= 0; --q) {
            const float2 w = aggb[q][jl];
            m = make_float2(w.x * m.x, fmaf(w.x, m.y, w.y));
          }
          for (int q = 0; q < C; ++q) put_remote(&peer[buf][rank][jl], q, m);
        }
        cluster_sync();
      }
      if (joinf) {
        const int64_t piece = k * C + rank;
        float s = cj < p.D && piece < pieces && piece * L < n ? a.saved[(b * pieces + piece) * p.D + cj] : 0.f;
#pragma unroll
        for (int q = 0; q < G; ++q) {
          first[q][jl] = s;
          s = fmaf(aggf[q][jl].x, s, aggf[q][jl].y);
        }
      }
      if (joinb) {
        float w = r;
        if (CL)
          for (int q = C - 1; q > rank; --q) w = fmaf(peer[buf][q][jl].x, w, peer[buf][q][jl].y);
#pragma unroll
        for (int q = G - 1; q >= 0; --q) {
          last[q][jl] = w;
          w = fmaf(aggb[q][jl].x, w, aggb[q][jl].y);
        }
        if (CL)
          for (int q = rank - 1; q >= 0; --q) w = fmaf(peer[buf][q][jl].x, w, peer[buf][q][jl].y);
        r = w;
      }
      __syncthreads();
      float hb[S][V], s[V], w[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        s[v] = first[p.group][p.lane * V + v];
        w[v] = last[p.group][p.lane * V + v];
      }
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          hb[i][v] = s[v];
          s[v] = fmaf(f[i][v], s[v], g[i][v] * xv[i][v]);
        }
#pragma unroll
      for (int i = S - 1; i >= 0; --i)
#pragma unroll
        for (int v = 0; v < V; ++v) {
          const bool in = t + i < n;
          const float Gt = dv[i][v] + w[v];
          w[v] = f[i][v] * Gt;
          dv[i][v] = in ? g[i][v] * Gt : 0.f;
          xv[i][v] = in ? g[i][v] * w[v] * (hb[i][v] - xv[i][v]) : 0.f;
        }
    } else {
#pragma unroll
      for (int i = 0; i < S; ++i)
#pragma unroll
        for (int v = 0; v < V; ++v) dv[i][v] = xv[i][v] = 0.f;
    }
    // dx in dv, dz of each channel in xv
#pragma unroll
    for (int i = 0; i < S; ++i)
      if (p.on && t + i < a.time) RX::store(dxp + i * a.dx_stride_t, dv[i]);
    if (!SH) {
#pragma unroll
      for (int i = 0; i < S; ++i)
        if (p.on && t + i < a.time) RX::store(dzp + i * a.dz_stride_t, xv[i]);
    } else if (part_width == 1) {
#pragma unroll
      for (int i = 0; i < S; ++i)
        if (p.on && t + i < a.time)
#pragma unroll
          for (int v = 0; v < V; ++v) part[(b * a.time + t + i) * p.D + p.c + v] = xv[i][v];
    } else {
      const int lanes = part_width / V;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        float q = 0.f;
#pragma unroll
        for (int v = 0; v < V; ++v) q += xv[i][v];
        for (int o = lanes / 2; o; o >>= 1) q += __shfl_xor_sync(0xffffffffu, q, o);
        if (p.on && t + i < a.time && p.lane % lanes == 0) {
          if (part) part[(b * a.time + t + i) * (p.D / part_width) + p.c / part_width] = q;
          else st(dzp + i * a.dz_stride_t, q);
        }
      }
    }
    dxp -= span * a.dx_stride_t;
    dzp -= span * a.dz_stride_t;
    buf ^= live;
  }
  if (joinb && rank == 0 && a.dh0 && cj < p.D) a.dh0[b * p.D + cj] = r;
}

// dz of a head: the sum of its `parts` parts
template <typename T>
__global__ void k_recur_dz(pnn_recur_args a, const float* part, int64_t parts) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, total = a.batch * a.time * a.heads;
  if (i >= total) return;
  const int64_t k = i % a.heads, bt = i / a.heads;
  const float* p = part + i * parts;
  float s = 0.f;
  for (int64_t j = 0; j < parts; ++j) s += p[j];
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
    v = fmaf(f, *s, g * ld(static_cast<const T*>(a.x) + i * a.x_stride + c));
    *s = v;
  }
  st(static_cast<T*>(a.h) + i * a.h_stride + c, v);
}

dim3 grid_of(int64_t D, int64_t rows, int threads) { return dim3((unsigned)((D + threads - 1) / threads), (unsigned)rows); }

int piece_of(const pnn_recur_args& a) { return a.dtype == PNN_DT_BF16 ? kPiece<bf16> : kPiece<float>; }

// Channels whose dz one CTA sums: as many as divide a head and lie in its
// tile.  The tiled form sums 64, 32, 16 or 8, this file's one 32, 16 or 1.
int part_width(const pnn_recur_args& a, bool tile) {
  if (tile)
    for (int w = 64; w >= 8; w /= 2)
      if (a.width % w == 0) return w;
  return a.width % 32 == 0 ? 32 : a.width % 16 == 0 ? 16 : 1;
}

// CTAs of a cluster: the time of a launch is about its waves over the CTA
// slots of the GPU times a CTA's share of the pieces; clusters cost a little
// at every piece.
int cluster_of(const pnn_recur_args& a, int ctas_per_sm) {
  const int64_t tiles = (a.heads * a.width + kTile - 1) / kTile * a.batch;
  const int64_t pieces = (a.time + piece_of(a) - 1) / piece_of(a);
  const int64_t slots = (int64_t)device_sm_count() * ctas_per_sm;
  int best = 1;
  double least = 0;
  for (int c = 1, l = 0; c <= kMaxCluster; c *= 2, ++l) {
    if (c > 1 && c / 2 >= pieces) break;
    const double cost = (double)((tiles * c + slots - 1) / slots) * (double)((pieces + c - 1) / c) * (1 + 0.04 * l);
    if (c == 1 || cost < least) best = c, least = cost;
  }
  return best;
}

template <typename K, typename... A>
cudaError_t launch(K kernel, int threads, int C, int64_t tiles, int64_t batch, cudaStream_t st, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * C), (unsigned)batch);
  cfg.blockDim = dim3(threads);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  if (C > 1) {
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = C;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    cfg.attrs = at;
    cfg.numAttrs = 1;
    if (C > 8) {  // more than the portable size
      const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
      if (e != cudaSuccess) return e;
    }
  }
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <int V>
bool even(const void* p, int64_t sb, int64_t st, size_t esz) {
  return (reinterpret_cast<uintptr_t>(p) & (V * esz - 1)) == 0 && sb % V == 0 && st % V == 0;
}

template <typename T, int V, bool SH>
cudaError_t run_fwd(const pnn_recur_args& a, int C, int64_t tiles, cudaStream_t st) {
  return C > 1 ? launch(k_recur_fwd<T, V, SH, true>, kThreads<V>, C, tiles, a.batch, st, a, C)
               : launch(k_recur_fwd<T, V, SH, false>, kThreads<V>, C, tiles, a.batch, st, a, C);
}
template <typename T, int V, bool SH>
cudaError_t run_bwd(const pnn_recur_args& a, int C, int64_t tiles, float* part, int pw, cudaStream_t st) {
  return C > 1 ? launch(k_recur_bwd<T, V, SH, true>, kThreads<V>, C, tiles, a.batch, st, a, C, part, pw)
               : launch(k_recur_bwd<T, V, SH, false>, kThreads<V>, C, tiles, a.batch, st, a, C, part, pw);
}

// Two channels a thread where every row allows the wider access (and, with a
// shared gate, both lie in one head); else one.
template <typename T>
cudaError_t fwd(const pnn_recur_args& a, cudaStream_t st) {
  const int64_t D = a.heads * a.width, tiles = (D + kTile - 1) / kTile;
  const bool sh = a.width > 1;
  const bool two = D % 2 == 0 && (sh ? a.width % 2 == 0 : even<2>(a.z, a.z_stride_b, a.z_stride_t, sizeof(T))) &&
                   even<2>(a.x, a.x_stride_b, a.x_stride_t, sizeof(T)) && even<2>(a.h, a.h_stride_b, a.h_stride_t, sizeof(T));
  const int C = cluster_of(a, two ? kFwdCtas<2> : kFwdCtas<1>);
  if (two) return sh ? run_fwd<T, 2, true>(a, C, tiles, st) : run_fwd<T, 2, false>(a, C, tiles, st);
  return sh ? run_fwd<T, 1, true>(a, C, tiles, st) : run_fwd<T, 1, false>(a, C, tiles, st);
}
template <typename T>
cudaError_t bwd(const pnn_recur_args& a, float* part, int pw, cudaStream_t st) {
  const int64_t D = a.heads * a.width, tiles = (D + kTile - 1) / kTile;
  const bool sh = a.width > 1;
  const bool two = D % 2 == 0 &&
                   (sh ? a.width % 2 == 0
                       : even<2>(a.z, a.z_stride_b, a.z_stride_t, sizeof(T)) &&
                             even<2>(a.dz, a.dz_stride_b, a.dz_stride_t, sizeof(T))) &&
                   even<2>(a.x, a.x_stride_b, a.x_stride_t, sizeof(T)) &&
                   even<2>(a.dh, a.dh_stride_b, a.dh_stride_t, sizeof(T)) &&
                   even<2>(a.dx, a.dx_stride_b, a.dx_stride_t, sizeof(T));
  const int C = cluster_of(a, two ? kBwdCtas<2> : kBwdCtas<1>);
  if (two) return sh ? run_bwd<T, 2, true>(a, C, tiles, part, pw, st) : run_bwd<T, 2, false>(a, C, tiles, part, pw, st);
  return sh ? run_bwd<T, 1, true>(a, C, tiles, part, pw, st) : run_bwd<T, 1, false>(a, C, tiles, part, pw, st);
}
}  // namespace

size_t recur_saved_floats(const pnn_recur_args& a) {
  return (size_t)a.batch * ((a.time + piece_of(a) - 1) / piece_of(a)) * a.heads * a.width;
}
// (the same for every alignment: the narrowest part either form may write)
size_t recur_workspace(const pnn_recur_args& a) {
  const int pw = part_width(a, false);
  return a.width > 1 && a.width != pw ? (size_t)a.batch * a.time * (a.heads * a.width / pw) * 4 : 0;
}

cudaError_t launch_recur_fwd(const pnn_recur_args& a, cudaStream_t st) {
  if (recur_tile_fwd_ok(a)) return launch_recur_tile_fwd(a, st);
  return a.dtype == PNN_DT_BF16 ? fwd<bf16>(a, st) : fwd<float>(a, st);
}

cudaError_t launch_recur_bwd(const pnn_recur_args& a, void* ws, cudaStream_t st) {
  const bool tile = recur_tile_bwd_ok(a);
  const int pw = part_width(a, tile);
  float* part = a.width > 1 && a.width != pw ? static_cast<float*>(ws) : nullptr;
  cudaError_t e = tile                      ? launch_recur_tile_bwd(a, part, pw, st)
                  : a.dtype == PNN_DT_BF16 ? bwd<bf16>(a, part, pw, st)
                                            : bwd<float>(a, part, pw, st);
  if (e != cudaSuccess || !part) return e;
  const dim3 g = grid_of(a.batch * a.time * a.heads, 1, 256);
  if (a.dtype == PNN_DT_BF16) k_recur_dz<bf16><<<g, 256, 0, st>>>(a, part, a.width / pw);
  else k_recur_dz<float><<<g, 256, 0, st>>>(a, part, a.width / pw);
  return cudaGetLastError();
}

cudaError_t launch_recur_step(const pnn_recur_step_args& a, cudaStream_t st) {
  const dim3 g = grid_of(a.heads * a.width, a.batch, 128);
  if (a.dtype == PNN_DT_BF16) k_recur_step<bf16><<<g, 128, 0, st>>>(a);
  else k_recur_step<float><<<g, 128, 0, st>>>(a);
  return cudaGetLastError();
}

}  // namespace pnn
