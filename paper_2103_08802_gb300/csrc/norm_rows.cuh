// The norm after a block with its gate and residual scale, and the norm before
// the next block: forward, and backward with the gradients of the weights.
//
// A team of 8 to 1024 threads holds a row in its registers, 8 values a thread
// (16 in rows of more than 8192), the next row on its way behind it, and every
// tensor is read and written once.  The
// backward computes h again from the forward's inputs instead of reading what
// the forward stored, which is rounded.  With t = x w silu(g) scale,
//   D  = dh + rh (dn w2 - h rh^2 mean(dn w2 h))          (what reaches h)
//   dx = rx (q w - x rx^2 mean(q w x)),   q = D scale silu(g),   sum q w x = sum D t,
// so that after rx (one meeting of the team) all sums meet at once:
//   sum h^2, sum dn w2 h, sum t dh, sum t dn w2, sum t h.
// A thread keeps its columns' weight gradients over all its rows; the CTAs'
// parts are added in order by a second launch.
//
// Bound: HBM forwards (16384 x 2048 bf16 with an fp32 residual stream 74 us, 470 MB, 6.3
// TB/s; 524288 x 128 with its gate 78), backwards the instructions too (177 us for 738 MB, 130
// for 671): 60 to 70 % of the issue slots.  Without a row ahead 148 and 243 us; with
// it in registers, which spilled, 179 and 317 for rows of 128.
#pragma once
#include <math.h>

#include <atomic>

#include "norm_place.h"
#include "pnn_internal.h"
#include "pnn_seq.h"
#include "seq_common.cuh"
#include "tc_ptx.cuh"

namespace pnn {
namespace norm {
using namespace seq;

// Values e of a thread's N: places in vectors of VE (8: 16 bytes, where all is bf16; 4: 8 of bf16 and 16 of fp32; 1: any
// alignment).  A row that begins `off` values behind a vector's border has its column c at place c + off: the vectors are
// whole in memory, and a team's rows, a multiple of VE apart, all begin there.
template <int VE>
__device__ __forceinline__ int col_of(int e, int lane, int team) { return (e / VE) * team * VE + lane * VE + e % VE; }

// A row's values of a thread.  With ASYNC they are copied into the thread's own places of shared memory while the row before
// is computed (registers for that cost more in spills than they gained); 16-bit values at any address, which such copies
// cannot take, and rows for which there is no room, are loaded when they are wanted.
template <typename T, int VE, int N, bool ROOM, bool OFF>
struct Ahead {
  static constexpr int G = VE * (int)sizeof(T) < 16 ? VE * (int)sizeof(T) : 16, PER = G / (int)sizeof(T);  // bytes and values of a piece
  static constexpr bool ASYNC = ROOM && G >= 4;
  static constexpr int BYTES = ASYNC ? N * (int)sizeof(T) : 0;  // of a thread
  static __device__ __forceinline__ void fetch(uint32_t to, const T* p, int lane, int team, int width, int off, int threads) {
    if constexpr (ASYNC) {
#pragma unroll
      for (int e = 0; e < N; e += PER) {
        const int c = col_of<VE>(e, lane, team) - off, left = (width - c) * (int)sizeof(T);
        const uint32_t at = to + e / PER * threads * G;
        const int n = left <= 0 ? 0 : !OFF || left > G ? G : left;  // (what is not copied becomes zeros)
        const T* from = OFF ? reinterpret_cast<const T*>(piece_address(reinterpret_cast<uintptr_t>(p), reinterpret_cast<uintptr_t>(p + c), n == 0, G)) : n ? p + c : p;
        if constexpr (G == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(at), "l"(from), "r"(n) : "memory");
        else asm volatile("cp.async.ca.shared.global [%0], [%1], %3, %2;" ::"r"(at), "l"(from), "r"(n), "n"(G) : "memory");
      }
    }
  }
  static __device__ __forceinline__ void get(float (&v)[N], uint32_t from, const T* p, int lane, int team, int width, int off, int threads) {
#pragma unroll
    for (int e = 0; e < N; e += PER) {
      uint32_t w[G < 4 ? 1 : G / 4];
      const int c = col_of<VE>(e, lane, team) - off;
      const uint32_t at = from + e / PER * threads * G;
      if constexpr (ASYNC) {
        if constexpr (G == 16) asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at) : "memory");
        else if constexpr (G == 8) asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(at) : "memory");
        else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(w[0]) : "r"(at) : "memory");
      } else if constexpr (PER == 1) {
        w[0] = 0;
        if (c < width) {
          if constexpr (sizeof(T) == 4) w[0] = __ldcs(reinterpret_cast<const uint32_t*>(p + c));
          else w[0] = __ldcs(reinterpret_cast<const unsigned short*>(p + c));
        }
      } else if ((!OFF || c >= 0) && c + PER <= width) {
        if constexpr (G == 16) {
          const uint4 u = __ldcs(reinterpret_cast<const uint4*>(p + c));
          w[0] = u.x, w[1] = u.y, w[2] = u.z, w[3] = u.w;
        } else {
          const uint2 u = __ldcs(reinterpret_cast<const uint2*>(p + c));
          w[0] = u.x, w[1] = u.y;
        }
      } else {  // a row's ends
#pragma unroll
        for (int i = 0; i < G / 4; ++i) w[i] = 0;
#pragma unroll
        for (int i = 0; i < (OFF ? PER : 0); ++i)
          if (c + i >= 0 && c + i < width) {
            if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(p[c + i]);
            else w[i / 2] |= (uint32_t)*reinterpret_cast<const unsigned short*>(p + c + i) << i % 2 * 16;
          }
      }
#pragma unroll
      for (int i = 0; i < PER; ++i) {
        if constexpr (sizeof(T) == 4) v[e + i] = __uint_as_float(w[i]);
        else v[e + i] = __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
      }
      if (ASYNC && OFF && PER > 1 && c < 0) {  // (the end of the row before)
#pragma unroll
        for (int i = 0; i < PER; ++i)
          if (c + i < 0) v[e + i] = 0.f;
      }
    }
  }
};
// Rows of a CTA beside the sums of wide rows (3 x 8192 fp32): not where all of five tensors are fp32, nor above 8192
template <typename T, typename R, int N, int CTA> constexpr bool kRoom = CTA < 1024 || (N == 8 && sizeof(T) + sizeof(R) < 8);
template <typename T, int VE, int N, bool OFF>
__device__ __forceinline__ void store(T* p, const float (&v)[N], int lane, int team, int width, int off) {
#pragma unroll
  for (int e = 0; e < N; e += VE) {
    const int c = col_of<VE>(e, lane, team) - off;
    if (!OFF && c >= width) continue;
    if (VE == 1 || (OFF && (c < 0 || c + VE > width))) {
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (c + i >= 0 && c + i < width) st(p + c + i, v[e + i]);
      continue;
    }
    if constexpr (VE > 1 && sizeof(T) == 2) {
      uint32_t w[VE / 2];
#pragma unroll
      for (int i = 0; i < VE / 2; ++i) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(v[e + 2 * i], v[e + 2 * i + 1]);
        w[i] = *reinterpret_cast<const uint32_t*>(&h);
      }
      if constexpr (VE == 8) *reinterpret_cast<uint4*>(p + c) = make_uint4(w[0], w[1], w[2], w[3]);
      else *reinterpret_cast<uint2*>(p + c) = make_uint2(w[0], w[1]);
    } else if constexpr (VE == 4) {
      *reinterpret_cast<float4*>(p + c) = make_float4(v[e], v[e + 1], v[e + 2], v[e + 3]);
    }
  }
}

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
// Off by 4 + 1.16 |g| times 2^-23 of itself, which is 2e-6 at |g| = 10.  fp32 rows by expf and a rounded division: 4096 x 8192 of all
// parts forward 121 -> 135 us, 9000 x 4101 241 -> 289.
__device__ __forceinline__ float sigmoid(float g) { return __fdividef(1.f, 1.f + __expf(-g)); }
template <typename T>
__device__ __forceinline__ const T* row_of(const pnn_rows& r, int64_t row) { return static_cast<const T*>(r.p) + row * r.stride; }
template <typename T>
__device__ __forceinline__ T* row_out(const pnn_rows& r, int64_t row) { return static_cast<T*>(r.p) + row * r.stride; }

// The columns' parameters (`otherwise` where absent): in registers, or, of wide rows, read again for every row (from L1)
template <int VE, int N, bool OFF>
__device__ __forceinline__ void params(float (&v)[N], const float* p, float otherwise, int lane, int team, int width, int off) {
  const bool whole = !OFF && (reinterpret_cast<uintptr_t>(p) & 15) == 0;
#pragma unroll
  for (int e = 0; e < N; e += VE) {
    const int c = col_of<VE>(e, lane, team) - off;
#pragma unroll
    for (int i = 0; i < VE; ++i) v[e + i] = p ? 0.f : otherwise;
    if (!p) continue;
    if (VE >= 4 && whole && c + VE <= width) {
#pragma unroll
      for (int i = 0; i < VE / 4; ++i) {
        const float4 a = *reinterpret_cast<const float4*>(p + c + 4 * i);
        v[e + 4 * i] = a.x, v[e + 4 * i + 1] = a.y, v[e + 4 * i + 2] = a.z, v[e + 4 * i + 3] = a.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < VE; ++i)
        if (c + i >= 0 && c + i < width) v[e + i] = p[c + i];
    }
  }
}

// CTA: threads of a CTA at most where it is one row's team, 0 where teams of up to 32 share one of 256.
// WIDE: rows of more than 4096, whose teams of 1024 threads have 64 registers each.
template <typename T, typename R, int VE, bool OFF, int N, int CTA>
__global__ void __launch_bounds__(CTA ? CTA : 256, CTA == 0 || CTA == 256 ? 3 : 1) k_norm_fwd(const __grid_constant__ pnn_norm_args a, int team) {
  constexpr bool BIG = CTA > 0, WIDE = CTA == 1024, ROOM = kRoom<T, R, N, CTA>;
  __shared__ float parts[2][2][32][1];  // (a row's parts are read while the next row's are written)
  int par = 0;
  const int lane = BIG ? threadIdx.x : threadIdx.x % team, width = (int)a.width;
  const int teams = BIG ? 1 : 256 / team, mine = BIG ? 0 : threadIdx.x / team;
  const float inv = 1.f / (float)width;
  const int off = OFF ? (int)(((int64_t)blockIdx.x * teams + mine) * a.x.stride % VE) : 0;
  float w[N], sc[N], w2[N];
  auto fresh = [&]() {
    params<VE, N, OFF>(w, a.weight, 1.f, lane, team, width, off);
    params<VE, N, OFF>(sc, a.scales, a.scale, lane, team, width, off);
    params<VE, N, OFF>(w2, a.next_weight, 1.f, lane, team, width, off);
  };
  if (!WIDE) fresh();
  const int64_t step = (int64_t)gridDim.x * teams;
  using AT = Ahead<T, VE, N, ROOM, OFF>;
  using AR = Ahead<R, VE, N, ROOM, OFF>;
  extern __shared__ __align__(16) char stage[];  // a row: x, gate, res
  const int threads = blockDim.x;
  auto place = [&](int bytes, int g) { return tc::smem_u32(stage) + threads * bytes + threadIdx.x * g; };
  auto fetch = [&](int64_t r0) {
    const int64_t row = r0 + mine;
    if (row < a.rows) {  // (a team without a row computes with what it finds, and keeps nothing of it)
      AT::fetch(place(0, AT::G), row_of<T>(a.x, row), lane, team, width, off, threads);
      if (a.gate.p) AT::fetch(place(AT::BYTES, AT::G), row_of<T>(a.gate, row), lane, team, width, off, threads);
      if (a.res.p) AR::fetch(place(2 * AT::BYTES, AR::G), row_of<R>(a.res, row), lane, team, width, off, threads);
    }
  };
  fetch((int64_t)blockIdx.x * teams);
  for (int64_t r0 = (int64_t)blockIdx.x * teams; r0 < a.rows; r0 += step, par ^= 1) {  // (the warps of a CTA stay together)
    const int64_t row = r0 + mine;
    const bool real = row < a.rows;
    float x[N], g[N], h[N];
    tc::cp_async_wait_all();
    {
      const int64_t at = real ? row : 0;
      const int width = real ? (int)a.width : 0;
      AT::get(x, place(0, AT::G), row_of<T>(a.x, at), lane, team, width, off, threads);
      if (a.gate.p) AT::get(g, place(AT::BYTES, AT::G), row_of<T>(a.gate, at), lane, team, width, off, threads);
      if (a.res.p) AR::get(h, place(2 * AT::BYTES, AR::G), row_of<R>(a.res, at), lane, team, width, off, threads);
    }
    fetch(r0 + step);  // (into the places that this thread has just read)
    if (WIDE) fresh();
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
    if (real) store<R, VE, N, OFF>(row_out<R>(a.h, row), h, lane, team, width, off);
    if (a.next_weight) {
      // columns behind the width are zero in x and res
      team_sum<BIG, 1>(s, team, parts[par][1]);
      const float rh = rsqrtf(fmaf(s[0], inv, a.eps));
#pragma unroll
      for (int e = 0; e < N; ++e) h[e] *= rh * w2[e];
      if (real) store<T, VE, N, OFF>(row_out<T>(a.n, row), h, lane, team, width, off);
    }
  }
}

// Parts of the weight gradients: [CTA][weight, scale, next][width].  A thread's columns are summed over its rows in
// registers, or, of wide rows, in shared memory (each place its own thread's).
// NEXT: there is a next norm.
template <typename T, typename R, int VE, bool OFF, int N, int CTA, bool NEXT>
__global__ void __launch_bounds__(CTA ? CTA : 256, CTA == 0 || CTA == 256 ? 2 : 1) k_norm_bwd(const __grid_constant__ pnn_norm_args a, int team, float* part) {
  constexpr bool BIG = CTA > 0, WIDE = CTA == 1024, ROOM = kRoom<T, R, N, CTA>;
  __shared__ float parts1[4][32][1], parts5[2][32][5];  // (a row's parts are read while the next row's are written)
  __shared__ float cols[BIG ? 1 : 256 * 8];
  extern __shared__ __align__(16) char stage[];  // a row: x, gate, dn, dh, res; behind it wide rows' sums, [weight, scale, next][value][thread]
  int par = 0;
  const int lane = BIG ? threadIdx.x : threadIdx.x % team, width = (int)a.width;
  const int teams = BIG ? 1 : 256 / team, mine = BIG ? 0 : threadIdx.x / team;
  const float inv = 1.f / (float)width;
  const int off = OFF ? (int)(((int64_t)blockIdx.x * teams + mine) * a.x.stride % VE) : 0;
  using AT = Ahead<T, VE, N, ROOM, OFF>;
  using AR = Ahead<R, VE, N, ROOM, OFF>;
  float* wide = reinterpret_cast<float*>(stage + (size_t)blockDim.x * (3 * AT::BYTES + 2 * AR::BYTES));
  float w[N], sc[N], w2[N], aw[N], as[N], an[N];
  auto fresh = [&]() {
    params<VE, N, OFF>(w, a.weight, 1.f, lane, team, width, off);
    params<VE, N, OFF>(sc, a.scales, a.scale, lane, team, width, off);
    params<VE, N, OFF>(w2, a.next_weight, 1.f, lane, team, width, off);
  };
  if (!WIDE) fresh();
#pragma unroll
  for (int e = 0; e < N; ++e) {
    aw[e] = as[e] = an[e] = 0.f;
    if (WIDE)
      for (int i = 0; i < 3; ++i) wide[(i * N + e) * team + lane] = 0.f;
  }
  const int64_t step = (int64_t)gridDim.x * teams;
  const int threads = blockDim.x;
  auto place = [&](int bytes, int g) { return tc::smem_u32(stage) + threads * bytes + threadIdx.x * g; };
  auto fetch = [&](int64_t r0) {
    const int64_t row = r0 + mine;
    if (row < a.rows) {  // (a team without a row computes with what it finds, and keeps nothing of it)
      AT::fetch(place(0, AT::G), row_of<T>(a.x, row), lane, team, width, off, threads);
      if (a.gate.p) AT::fetch(place(AT::BYTES, AT::G), row_of<T>(a.gate, row), lane, team, width, off, threads);
      if (NEXT) AT::fetch(place(2 * AT::BYTES, AT::G), row_of<T>(a.dn, row), lane, team, width, off, threads);
      if (a.dh.p) AR::fetch(place(3 * AT::BYTES, AR::G), row_of<R>(a.dh, row), lane, team, width, off, threads);
      if (NEXT && a.res.p) AR::fetch(place(3 * AT::BYTES + AR::BYTES, AR::G), row_of<R>(a.res, row), lane, team, width, off, threads);
    }
  };
  fetch((int64_t)blockIdx.x * teams);
  for (int64_t r0 = (int64_t)blockIdx.x * teams; r0 < a.rows; r0 += step, par ^= 1) {
    const int64_t row = r0 + mine;
    const bool real = row < a.rows;
    float x[N], g[N], h[N], dh[N], dn[N];
    tc::cp_async_wait_all();
    {
      const int64_t at = real ? row : 0;
      const int width = real ? (int)a.width : 0;
      AT::get(x, place(0, AT::G), row_of<T>(a.x, at), lane, team, width, off, threads);
      if (a.gate.p) AT::get(g, place(AT::BYTES, AT::G), row_of<T>(a.gate, at), lane, team, width, off, threads);
      if (NEXT) AT::get(dn, place(2 * AT::BYTES, AT::G), row_of<T>(a.dn, at), lane, team, width, off, threads);
      if (a.dh.p) AR::get(dh, place(3 * AT::BYTES, AR::G), row_of<R>(a.dh, at), lane, team, width, off, threads);
      if (NEXT && a.res.p) AR::get(h, place(3 * AT::BYTES + AR::BYTES, AR::G), row_of<R>(a.res, at), lane, team, width, off, threads);
    }
    fetch(r0 + step);  // (into the places that this thread has just read)
    if (WIDE) fresh();
    float rx = 1.f;
    if (a.weight) {
      float s[1] = {0.f};
#pragma unroll
      for (int e = 0; e < N; ++e) s[0] = fmaf(x[e], x[e], s[0]);
      team_sum<BIG, 1>(s, team, parts1[par]);
      rx = rsqrtf(fmaf(s[0], inv, a.eps));
    }
    float sg[N], back = 0.f, rh = 0.f, dt = 0.f;  // D = dh + rh dn w2 - back h, dt = sum D t
    if (!a.dh.p) {
#pragma unroll
      for (int e = 0; e < N; ++e) dh[e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < N; ++e) sg[e] = a.gate.p ? sigmoid(g[e]) : 1.f;
    if constexpr (NEXT) {
      float s[5] = {0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float t = x[e] * w[e] * sc[e] * (a.gate.p ? g[e] * sg[e] : 1.f), d = dn[e] * w2[e];
        h[e] = a.res.p ? fmaf(rx, t, h[e]) : rx * t;
        s[0] = fmaf(h[e], h[e], s[0]);
        s[1] = fmaf(d, h[e], s[1]);
        s[2] = fmaf(t, dh[e], s[2]);
        s[3] = fmaf(t, d, s[3]);
        s[4] = fmaf(t, h[e], s[4]);
      }
      team_sum<BIG, 5>(s, team, parts5[par]);
      rh = rsqrtf(fmaf(s[0], inv, a.eps));
      back = rh * rh * rh * s[1] * inv;
      dt = s[2] + rh * s[3] - back * s[4];
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (WIDE) an[e] = wide[(2 * N + e) * team + lane];
        if (real) an[e] = fmaf(dn[e] * rh, h[e], an[e]);
        if (WIDE) wide[(2 * N + e) * team + lane] = an[e];
        dh[e] = fmaf(rh * dn[e], w2[e], fmaf(-back, h[e], dh[e]));
      }
    } else if (a.weight) {
      float s[1] = {0.f};
#pragma unroll
      for (int e = 0; e < N; ++e) s[0] = fmaf(x[e] * w[e] * sc[e] * (a.gate.p ? g[e] * sg[e] : 1.f), dh[e], s[0]);
      team_sum<BIG, 1>(s, team, parts1[2 + par]);
      dt = s[0];
    }
    if (real && a.dres.p) store<R, VE, N, OFF>(row_out<R>(a.dres, row), dh, lane, team, width, off);
    if (a.scales) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (WIDE) as[e] = wide[(N + e) * team + lane];
        if (real) as[e] = fmaf(dh[e] * (x[e] * rx), w[e] * (a.gate.p ? g[e] * sg[e] : 1.f), as[e]);
        if (WIDE) wide[(N + e) * team + lane] = as[e];
      }
    }
    if (a.gate.p) {
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const float q = dh[e] * sc[e], y = x[e] * rx, act = g[e] * sg[e];
        dh[e] = q * act;
        g[e] = q * (y * w[e]) * fmaf(act, 1.f - sg[e], sg[e]);  // silu' = sg (1 + g (1 - sg))
      }
      if (real && a.dgate.p) store<T, VE, N, OFF>(row_out<T>(a.dgate, row), g, lane, team, width, off);
    } else {
#pragma unroll
      for (int e = 0; e < N; ++e) dh[e] *= sc[e];
    }
    if (a.weight) {
      const float cx = rx * rx * rx * dt * inv;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        if (WIDE) aw[e] = wide[e * team + lane];
        if (real) aw[e] = fmaf(dh[e], x[e] * rx, aw[e]);
        if (WIDE) wide[e * team + lane] = aw[e];
        dh[e] = fmaf(dh[e], w[e] * rx, -cx * x[e]);
      }
    }
    if (real) store<T, VE, N, OFF>(row_out<T>(a.dx, row), dh, lane, team, width, off);
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
        const int c = col_of<VE>(e, lane, team) - off;
        if (c >= 0 && c < width) to[i * width + c] = WIDE ? wide[(i * N + e) * team + lane] : v[e];
      }
    } else {
      __syncthreads();
#pragma unroll
      for (int e = 0; e < N; ++e) cols[mine * team * N + col_of<VE>(e, lane, team)] = v[e];
      __syncthreads();
      for (int c = threadIdx.x; c < width; c += 256) {
        float s = 0.f;
        for (int j = 0; j < teams; ++j) s += cols[j * team * N + c + (OFF ? (int)(((int64_t)blockIdx.x * teams + j) * a.x.stride % VE) : 0)];
        to[i * width + c] = s;
      }
    }
  }
}

// The parts of all CTAs, in order: 32 columns by 32 groups of parts a CTA.
static __global__ void __launch_bounds__(1024) k_norm_sum(const __grid_constant__ pnn_norm_args a, const float* part, int parts) {
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
  int cta;      // see k_norm_fwd
  unsigned grid;
};
inline Plan plan(const pnn_norm_args& a, bool back, bool inside) {
  Plan p;
  const int64_t places = a.width + (inside ? 7 : 0);  // (rows that begin inside a vector)
  p.n = places > 8192 ? 16 : 8;
  p.team = 8;
  while (p.team * p.n < places) p.team *= 2;
  p.cta = p.team <= 32 ? 0 : p.team <= 256 ? 256 : p.team;
  const int64_t teams = p.cta ? 1 : 256 / p.team, need = (a.rows + teams - 1) / teams;
  const int threads = p.cta ? p.team : 256, fit = p.cta > 256 ? 1 : (back ? 512 : 768) / threads;  // CTAs of an SM
  const int64_t most = (int64_t)device_sm_count() * fit;
  p.grid = (unsigned)(need < most ? need : most > 8 ? most & ~7ll : most);  // (several rows of a team lie a multiple of 8 apart)
  return p;
}
// Whether all rows lie in vectors of ve values: their first ones on a vector's border, and all as far apart, but for whole vectors
inline bool vec(const pnn_rows& r, const pnn_norm_args& a, int esz, int ve) {
  if (!r.p) return true;
  const int bytes = ve * esz < 16 ? ve * esz : 16;
  return reinterpret_cast<uintptr_t>(r.p) % bytes == 0 && (a.rows <= 1 || r.stride % ve == a.x.stride % ve);
}
inline bool all_vec(const pnn_norm_args& a, bool back, int ve) {
  const int t = a.dtype == PNN_DT_BF16 ? 2 : 4, r = a.res_dtype == PNN_DT_BF16 ? 2 : 4;
  const pnn_rows none = {nullptr, 0};
  const pnn_rows ts[] = {a.x, a.gate, back ? a.dn : a.n, back ? a.dx : none, back ? a.dgate : none};
  for (const pnn_rows& x : ts)
    if (!vec(x, a, t, ve)) return false;
  const pnn_rows rs[] = {a.res, back ? a.dh : a.h, back ? a.dres : none};
  for (const pnn_rows& x : rs)
    if (!vec(x, a, r, ve)) return false;
  return true;
}
template <typename T, typename R, int VE, bool OFF, int N, int CTA>
cudaError_t run(const pnn_norm_args& a, bool back, const Plan& p, float* ws, cudaStream_t st) {
  const unsigned threads = CTA ? p.team : 256;
  using AT = Ahead<T, VE, N, kRoom<T, R, N, CTA>, OFF>;
  using AR = Ahead<R, VE, N, kRoom<T, R, N, CTA>, OFF>;
  constexpr int most = CTA ? CTA : 256, fwd = 2 * AT::BYTES + AR::BYTES, bwd = 3 * AT::BYTES + 2 * AR::BYTES + (CTA == 1024 ? 3 * N * 4 : 0);  // bytes a thread
  static std::atomic<uint64_t> ready{0};  // one bit a device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(k_norm_fwd<T, R, VE, OFF, N, CTA>, cudaFuncAttributeMaxDynamicSharedMemorySize, fwd * most);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_norm_bwd<T, R, VE, OFF, N, CTA, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, bwd * most);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_norm_bwd<T, R, VE, OFF, N, CTA, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, bwd * most);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  if (!back) {
    k_norm_fwd<T, R, VE, OFF, N, CTA><<<p.grid, threads, fwd * threads, st>>>(a, p.team);
    return cudaGetLastError();
  }
  if (p.grid) {  // (no rows: the sums are zero)
    if (a.next_weight) k_norm_bwd<T, R, VE, OFF, N, CTA, true><<<p.grid, threads, bwd * threads, st>>>(a, p.team, ws);
    else k_norm_bwd<T, R, VE, OFF, N, CTA, false><<<p.grid, threads, bwd * threads, st>>>(a, p.team, ws);
  }
  if (a.dweight || a.dscales || a.dnext_weight)
    k_norm_sum<<<dim3((unsigned)((a.width + 31) / 32), 3), dim3(32, 32), 0, st>>>(a, ws, (int)p.grid);
  return cudaGetLastError();
}
template <typename T, typename R, int VE, bool OFF>
cudaError_t sized(const pnn_norm_args& a, bool back, float* ws, cudaStream_t st) {
  const Plan p = plan(a, back, OFF);
  if (p.cta == 0) return run<T, R, VE, OFF, 8, 0>(a, back, p, ws, st);
  if (p.cta == 256) return run<T, R, VE, OFF, 8, 256>(a, back, p, ws, st);
  if (p.cta == 512) return run<T, R, VE, OFF, 8, 512>(a, back, p, ws, st);
  return p.n == 8 ? run<T, R, VE, OFF, 8, 1024>(a, back, p, ws, st) : run<T, R, VE, OFF, 16, 1024>(a, back, p, ws, st);
}
template <typename T, typename R>
cudaError_t aligned(const pnn_norm_args& a, bool back, float* ws, cudaStream_t st) {
  constexpr int VE = sizeof(T) + sizeof(R) == 4 ? 8 : 4;
  if (all_vec(a, back, VE)) {
    if (a.width % VE == 0 && (a.rows <= 1 || a.x.stride % VE == 0)) return sized<T, R, VE, false>(a, back, ws, st);
    if (a.width <= 16384 - 7) return sized<T, R, VE, true>(a, back, ws, st);
  }
  return sized<T, R, 1, false>(a, back, ws, st);
}
// x, gate, n in bf16 or fp32, the residual stream in either
cudaError_t run_bf16(const pnn_norm_args& a, bool back, float* ws, cudaStream_t st);
cudaError_t run_f32(const pnn_norm_args& a, bool back, float* ws, cudaStream_t st);

}  // namespace norm
}  // namespace pnn
