// The norm after a block with its gate and residual scale, and the norm before
// the next block: forward, and backward with the gradients of the weights.
//
// A team of 8 to 1024 threads holds a row in its registers, 8 values a thread
// (16 in rows of more than 8192), and every tensor is read and written once.  The
// backward computes h again from the forward's inputs instead of reading what
// the forward stored, which is rounded.  With t = x w silu(g) scale,
//   D  = dh + rh (dn w2 - h rh^2 mean(dn w2 h))          (what reaches h)
//   dx = rx (q w - x rx^2 mean(q w x)),   q = D scale silu(g),   sum q w x = sum D t,
// so that after rx (one meeting of the team) all sums meet at once:
//   sum h^2, sum dn w2 h, sum t dh, sum t dn w2, sum t h.
// A thread keeps its columns' weight gradients over all its rows; the CTAs'
// parts are added in order by a second launch.
//
// Bound: HBM.
#include <math.h>

#include "pnn_internal.h"
#include "pnn_seq.h"
#include "seq_common.cuh"

namespace pnn {
namespace {
using namespace seq;

// Values e of a thread's N: columns in vectors of VE (8: 16 bytes of bf16; 2; 1: any alignment)
template <int VE>
__device__ __forceinline__ int col_of(int e, int lane, int team) { return (e / VE) * team * VE + lane * VE + e % VE; }

template <typename T, int VE, int N>
__device__ __forceinline__ void load(float (&v)[N], const T* p, int lane, int team, int width) {
#pragma unroll
  for (int e = 0; e < N; e += VE) {
    const int c = col_of<VE>(e, lane, team);
    if (c >= width) {
#pragma unroll
      for (int i = 0; i < VE; ++i) v[e + i] = 0.f;
      continue;
    }
    if constexpr (VE == 8 && sizeof(T) == 2) {
      const uint4 u = *reinterpret_cast<const uint4*>(p + c);
      const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        v[e + 2 * i] = __uint_as_float(w[i] << 16);
        v[e + 2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
    } else if constexpr (VE == 8) {
      const float4 a = *reinterpret_cast<const float4*>(p + c), b = *reinterpret_cast<const float4*>(p + c + 4);
      v[e] = a.x, v[e + 1] = a.y, v[e + 2] = a.z, v[e + 3] = a.w;
      v[e + 4] = b.x, v[e + 5] = b.y, v[e + 6] = b.z, v[e + 7] = b.w;
    } else if constexpr (VE == 2 && sizeof(T) == 2) {
      const uint32_t u = *reinterpret_cast<const uint32_t*>(p + c);
      v[e] = __uint_as_float(u << 16);
      v[e + 1] = __uint_as_float(u & 0xffff0000u);
    } else if constexpr (VE == 2) {
      const float2 a = *reinterpret_cast<const float2*>(p + c);
      v[e] = a.x, v[e + 1] = a.y;
    } else {
      v[e] = ld(p + c);
    }
  }
}
template <typename T, int VE, int N>
__device__ __forceinline__ void store(T* p, const float (&v)[N], int lane, int team, int width) {
#pragma unroll
  for (int e = 0; e < N; e += VE) {
    const int c = col_of<VE>(e, lane, team);
    if (c >= width) continue;
    if constexpr (VE >= 2 && sizeof(T) == 2) {
      uint32_t w[VE / 2];
#pragma unroll
      for (int i = 0; i < VE / 2; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[e + 2 * i], v[e + 2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
      if constexpr (VE == 8) *reinterpret_cast<uint4*>(p + c) = make_uint4(w[0], w[1], w[2], w[3]);
      else *reinterpret_cast<uint32_t*>(p + c) = w[0];
    } else if constexpr (VE == 8) {
      *reinterpret_cast<float4*>(p + c) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
      *reinterpret_cast<float4*>(p + c + 4) = make_float4(v[e + 4], v[e + 5], v[e + 6], v[e + 7]);
    } else if constexpr (VE == 2) {
      *reinterpret_cast<float2*>(p + c) = make_float2(v[e], v[e + 1]);
    } else {
      st(p + c, v[e]);
    }
  }
}

// CTA: threads of a CTA at most where it is one row's team, 0 where teams share warps.
// Sums of a team: by shuffles inside a warp, then (a team is the CTA) through shared memory, added in the warps' order.
template <bool BIG, int K>
__device__ __forceinline__ void team_sum(float (&s)[K], int team, float (*parts)[K]) {
#pragma unroll
  for (int o = 16; o; o >>= 1)
    if (BIG || o < team) {
#pragma unroll
      for (int i = 0; i < K; ++i) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    }
  if constexpr (BIG) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, n = blockDim.x >> 5;
    if (lane == 0)
#pragma unroll
      for (int i = 0; i < K; ++i) parts[warp][i] = s[i];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < K; ++i) {
      s[i] = lane < n ? parts[lane][i] : 0.f;
#pragma unroll
      for (int o = 16; o; o >>= 1) s[i] += __shfl_xor_sync(0xffffffffu, s[i], o);
    }
  }
}
__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }
template <typename T>
__device__ __forceinline__ const T* row_of(const pnn_rows& r, int64_t row) { return static_cast<const T*>(r.p) + row * r.stride; }
template <typename T>
__device__ __forceinline__ T* row_out(const pnn_rows& r, int64_t row) { return static_cast<T*>(r.p) + row * r.stride; }

// The columns' parameters (1 where absent)
template <int VE, int N>
__device__ __forceinline__ void params(float (&v)[N], const float* p, float otherwise, int lane, int team, int width) {
  if (p) {
    load<float, VE, N>(v, p, lane, team, width);
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e) v[e] = otherwise;
  }
}

template <typename T, typename R, int VE, int N, int CTA>
__global__ void __launch_bounds__(CTA ? CTA : 256) k_norm_fwd(const __grid_constant__ pnn_norm_args a, int team) {
  constexpr bool BIG = CTA > 0;
  __shared__ float parts[2][2][32][1];  // (a row's parts are read while the next row's are written)
  int par = 0;
  const int lane = BIG ? threadIdx.x : threadIdx.x % team, width = (int)a.width;
  const int teams = BIG ? 1 : 256 / team, mine = BIG ? 0 : threadIdx.x / team;
  const float inv = 1.f / (float)width;
  float w[N], sc[N], w2[N];
  params<VE, N>(w, a.weight, 1.f, lane, team, width);
  params<VE, N>(sc, a.scales, a.scale, lane, team, width);
  params<VE, N>(w2, a.next_weight, 1.f, lane, team, width);
  const int64_t step = (int64_t)gridDim.x * teams;
  for (int64_t r0 = (int64_t)blockIdx.x * teams; r0 < a.rows; r0 += step, par ^= 1) {  // (the warps of a CTA stay together)
    const int64_t row = r0 + mine < a.rows ? r0 + mine : a.rows - 1;
    const bool real = r0 + mine < a.rows;
    float x[N], g[N], h[N];
    load<T, VE, N>(x, row_of<T>(a.x, row), lane, team, width);
    if (a.gate.p) load<T, VE, N>(g, row_of<T>(a.gate, row), lane, team, width);
    if (a.res.p) load<R, VE, N>(h, row_of<R>(a.res, row), lane, team, width);
    float s[1] = {0.f}, rx = 1.f;
    if (a.weight) {
#pragma unroll
      for (int e = 0; e < N; ++e) s[0] = fmaf(x[e], x[e], s[0]);
      team_sum<BIG, 1>(s, team, parts[par][0]);
      rx = rsqrtf(fmaf(s[0], inv, a.eps));
    }
    s[0] = 0.f;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float y = x[e] * rx * w[e];
      if (a.gate.p) y *= g[e] * sigmoid(g[e]);
      h[e] = a.res.p ? fmaf(sc[e], y, h[e]) : sc[e] * y;
      s[0] = fmaf(h[e], h[e], s[0]);
    }
    if (real) store<R, VE, N>(row_out<R>(a.h, row), h, lane, team, width);
    if (a.next_weight) {
      // columns behind the width are zero in x and res
      team_sum<BIG, 1>(s, team, parts[par][1]);
      const float rh = rsqrtf(fmaf(s[0], inv, a.eps));
#pragma unroll
      for (int e = 0; e < N; ++e) h[e] *= rh * w2[e];
      if (real) store<T, VE, N>(row_out<T>(a.n, row), h, lane, team, width);
    }
  }
}

// Parts of the weight gradients: [CTA][weight, scale, next][width]
template <typename T, typename R, int VE, int N, int CTA>
__global__ void __launch_bounds__(CTA ? CTA : 256) k_norm_bwd(const __grid_constant__ pnn_norm_args a, int team, float* part) {
  constexpr bool BIG = CTA > 0;
  __shared__ float parts1[2][32][1], parts5[2][32][5];  // (a row's parts are read while the next row's are written)
  int par = 0;
  __shared__ float cols[BIG ? 1 : 256 * 8];
  const int lane = BIG ? threadIdx.x : threadIdx.x % team, width = (int)a.width;
  const int teams = BIG ? 1 : 256 / team, mine = BIG ? 0 : threadIdx.x / team;
  const float inv = 1.f / (float)width;
  float w[N], sc[N], w2[N], aw[N], as[N], an[N];
  params<VE, N>(w, a.weight, 1.f, lane, team, width);
  params<VE, N>(sc, a.scales, a.scale, lane, team, width);
  params<VE, N>(w2, a.next_weight, 1.f, lane, team, width);
#pragma unroll
  for (int e = 0; e < N; ++e) aw[e] = as[e] = an[e] = 0.f;
  const int64_t step = (int64_t)gridDim.x * teams;
  for (int64_t r0 = (int64_t)blockIdx.x * teams; r0 < a.rows; r0 += step, par ^= 1) {
    const bool real = r0 + mine < a.rows;
    const int64_t row = real ? r0 + mine : a.rows - 1;
    float x[N], g[N], h[N], dh[N], dn[N];
    load<T, VE, N>(x, row_of<T>(a.x, row), lane, team, width);
    if (a.gate.p) load<T, VE, N>(g, row_of<T>(a.gate, row), lane, team, width);
    if (a.dh.p) load<R, VE, N>(dh, row_of<R>(a.dh, row), lane, team, width);
    if (a.next_weight) {
      if (a.res.p) load<R, VE, N>(h, row_of<R>(a.res, row), lane, team, width);
      load<T, VE, N>(dn, row_of<T>(a.dn, row), lane, team, width);
    }
    float rx = 1.f;
    if (a.weight) {
      float s[1] = {0.f};
#pragma unroll
      for (int e = 0; e < N; ++e) s[0] = fmaf(x[e], x[e], s[0]);
      team_sum<BIG, 1>(s, team, parts1[par]);
      rx = rsqrtf(fmaf(s[0], inv, a.eps));
    }
    float s[5] = {0.f, 0.f, 0.f, 0.f, 0.f}, sg[N];
#pragma unroll
    for (int e = 0; e < N; ++e) {
      sg[e] = a.gate.p ? sigmoid(g[e]) : 1.f;
      const float act = a.gate.p ? g[e] * sg[e] : 1.f, t = x[e] * w[e] * act * sc[e];
      if (!a.dh.p) dh[e] = 0.f;
      s[2] = fmaf(t, dh[e], s[2]);
      if (a.next_weight) {
        h[e] = a.res.p ? fmaf(rx, t, h[e]) : rx * t;
        const float d = dn[e] * w2[e];
        s[0] = fmaf(h[e], h[e], s[0]);
        s[1] = fmaf(d, h[e], s[1]);
        s[3] = fmaf(t, d, s[3]);
        s[4] = fmaf(t, h[e], s[4]);
      }
    }
    if (a.weight || a.next_weight) team_sum<BIG, 5>(s, team, parts5[par]);
    float rh = 0.f, back = 0.f;  // D = dh + rh dn w2 - back h
    if (a.next_weight) {
      rh = rsqrtf(fmaf(s[0], inv, a.eps));
      back = rh * rh * rh * s[1] * inv;
    }
    const float st = a.weight ? s[2] + rh * s[3] - back * s[4] : 0.f;  // sum D t
    const float cx = rx * rx * st * inv;
#pragma unroll
    for (int e = 0; e < N; ++e) {
      float D = dh[e];
      if (a.next_weight) {
        if (real) an[e] = fmaf(dn[e] * rh, h[e], an[e]);
        D = fmaf(rh * dn[e], w2[e], fmaf(-back, h[e], D));
      }
      dh[e] = D;
      const float act = a.gate.p ? g[e] * sg[e] : 1.f, y = x[e] * rx, q = D * sc[e];
      if (real) {
        as[e] = fmaf(D * act, y * w[e], as[e]);
        aw[e] = fmaf(q * act, y, aw[e]);
      }
      if (a.gate.p) g[e] = q * y * w[e] * sg[e] * fmaf(g[e], 1.f - sg[e], 1.f);
      x[e] = rx * (q * act * w[e] - x[e] * cx);
    }
    if (real) {
      store<T, VE, N>(row_out<T>(a.dx, row), x, lane, team, width);
      if (a.dgate.p) store<T, VE, N>(row_out<T>(a.dgate, row), g, lane, team, width);
      if (a.dres.p) store<R, VE, N>(row_out<R>(a.dres, row), dh, lane, team, width);
    }
  }
  float* to = part + (int64_t)blockIdx.x * 3 * width;
  const bool want[3] = {a.dweight != nullptr, a.dscales != nullptr, a.dnext_weight != nullptr};
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    if (!want[i]) continue;
    const float(&v)[N] = i == 0 ? aw : i == 1 ? as : an;
    if constexpr (BIG) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int c = col_of<VE>(e, lane, team);
        if (c < width) to[i * width + c] = v[e];
      }
    } else {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < N; ++e) cols[mine * team * N + col_of<VE>(e, lane, team)] = v[e];
      __syncthreads();
      for (int c = threadIdx.x; c < width; c += 256) {
        float s = 0.f;
        for (int j = 0; j < teams; ++j) s += cols[j * team * N + c];
        to[i * width + c] = s;
      }
    }
  }
}

// The parts of all CTAs, in order: 32 columns by 32 groups of parts a CTA.
__global__ void __launch_bounds__(1024) k_norm_sum(const __grid_constant__ pnn_norm_args a, const float* part, int parts) {
  __shared__ float s[32][33];
  const int width = (int)a.width, c = blockIdx.x * 32 + threadIdx.x;
  float* out = blockIdx.y == 0 ? a.dweight : blockIdx.y == 1 ? a.dscales : a.dnext_weight;
  if (!out) return;
  const int each = (parts + 31) / 32, p0 = threadIdx.y * each, p1 = p0 + each < parts ? p0 + each : parts;
  float v = 0.f;
  if (c < width)
#pragma unroll 4
    for (int p = p0; p < p1; ++p) v += part[((int64_t)p * 3 + blockIdx.y) * width + c];
  s[threadIdx.y][threadIdx.x] = v;
  __syncthreads();
  if (threadIdx.y) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < 32; ++i) v += s[i][threadIdx.x];
  if (c < width) out[c] = v;
}

// Threads of a row's team, and CTAs of a launch.
struct Plan {
  int team, n;  // n: values of a thread
  bool big;
  unsigned grid;
};
Plan plan(const pnn_norm_args& a) {
  Plan p;
  p.n = a.width > 8192 ? 16 : 8;
  p.team = 8;
  while (p.team * p.n < a.width) p.team *= 2;
  p.big = p.team > 32;
  const int64_t teams = p.big ? 1 : 256 / p.team, need = (a.rows + teams - 1) / teams;
  const int64_t most = (int64_t)device_sm_count() * (p.big ? (p.team >= 512 ? 1 : p.team >= 256 ? 2 : 4) : 2);
  p.grid = (unsigned)(need < most ? need : most);
  return p;
}
bool vec(const pnn_rows& r, int64_t rows, int esz, int ve) {
  if (!r.p) return true;
  const int bytes = ve * esz < 16 ? ve * esz : 16;
  return (reinterpret_cast<uintptr_t>(r.p) % bytes) == 0 && (rows <= 1 || r.stride * esz % bytes == 0);
}
bool all_vec(const pnn_norm_args& a, bool back, int ve) {
  const int t = a.dtype == PNN_DT_BF16 ? 2 : 4, r = a.res_dtype == PNN_DT_BF16 ? 2 : 4;
  if (a.width % ve) return false;
  const pnn_rows none = {nullptr, 0};
  const pnn_rows weights[3] = {{(void*)a.weight, 0}, {(void*)a.scales, 0}, {(void*)a.next_weight, 0}};
  for (const pnn_rows& w : weights)
    if (!vec(w, 1, 4, ve)) return false;
  const pnn_rows ts[] = {a.x, a.gate, back ? a.dn : a.n, back ? a.dx : none, back ? a.dgate : none};
  for (const pnn_rows& x : ts)
    if (!vec(x, a.rows, t, ve)) return false;
  const pnn_rows rs[] = {a.res, back ? a.dh : a.h, back ? a.dres : none};
  for (const pnn_rows& x : rs)
    if (!vec(x, a.rows, r, ve)) return false;
  return true;
}
template <typename T, typename R, int VE, int N, int CTA>
cudaError_t run(const pnn_norm_args& a, bool back, const Plan& p, float* ws, cudaStream_t st) {
  const unsigned threads = CTA ? p.team : 256;
  if (!back) {
    k_norm_fwd<T, R, VE, N, CTA><<<p.grid, threads, 0, st>>>(a, p.team);
    return cudaGetLastError();
  }
  if (p.grid) k_norm_bwd<T, R, VE, N, CTA><<<p.grid, threads, 0, st>>>(a, p.team, ws);  // (no rows: the sums are zero)
  if (a.dweight || a.dscales || a.dnext_weight)
    k_norm_sum<<<dim3((unsigned)((a.width + 31) / 32), 3), dim3(32, 32), 0, st>>>(a, ws, (int)p.grid);
  return cudaGetLastError();
}
template <typename T, typename R, int VE>
cudaError_t sized(const pnn_norm_args& a, bool back, float* ws, cudaStream_t st) {
  const Plan p = plan(a);
  if (!p.big) return run<T, R, VE, 8, 0>(a, back, p, ws, st);
  if (p.team <= 256) return run<T, R, VE, 8, 256>(a, back, p, ws, st);
  return p.n == 8 ? run<T, R, VE, 8, 1024>(a, back, p, ws, st) : run<T, R, VE, 16, 1024>(a, back, p, ws, st);
}
template <typename T, typename R>
cudaError_t aligned(const pnn_norm_args& a, bool back, float* ws, cudaStream_t st) {
  if (all_vec(a, back, 8)) return sized<T, R, 8>(a, back, ws, st);
  if (all_vec(a, back, 2)) return sized<T, R, 2>(a, back, ws, st);
  return sized<T, R, 1>(a, back, ws, st);
}
}  // namespace

size_t norm_workspace(const pnn_norm_args& a) {
  if (!a.rows || !(a.weight || a.scales || a.next_weight)) return 0;
  return (size_t)plan(a).grid * 3 * a.width * 4;
}
cudaError_t launch_norm(const pnn_norm_args& a, bool back, void* ws, cudaStream_t st) {
  using seq::bf16;
  float* w = static_cast<float*>(ws);
  if (a.dtype == PNN_DT_BF16) return a.res_dtype == PNN_DT_BF16 ? aligned<bf16, bf16>(a, back, w, st) : aligned<bf16, float>(a, back, w, st);
  return a.res_dtype == PNN_DT_BF16 ? aligned<float, bf16>(a, back, w, st) : aligned<float, float>(a, back, w, st);
}

}  // namespace pnn
