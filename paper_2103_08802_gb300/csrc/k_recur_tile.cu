// Gated linear recurrence on TMA-fed tiles: the scan and its backward pass for
// rows that a tensor map can describe (16-byte aligned base and strides).
//
// h_t = f_t h_{t-1} + u_t, u_t = (1 - f_t) x_t, is affine in the state: a run
// of steps is a pair (A, B) = (product of f, its result from zero), and runs
// compose, (A2, B2) after (A1, B1) = (A2 A1, A2 B1 + B2).
//
// A CTA owns 64 channels and walks along time in pieces of 8 S steps.  A
// producer warp keeps a ring of stages filled by TMA (z, x and, backward, dh);
// each of eight warps takes 8 channels of the piece, alone: 4 lanes are its
// channel pairs, 8 groups of lanes its consecutive runs of S steps.  A thread
// solves its run from zero (f and u stay in registers), the 8 runs are
// composed by warp shuffles, and the thread runs its steps again from its true
// first state, writing h over x in the stage, from where TMA stores it.  No
// barrier joins the warps.  The backward pass is the same recurrence along
// decreasing time, R_t = f_t (dh_t + R_{t+1}); it recomputes the states in
// fp32 from each piece's first state, which the forward saved.
//
// Too few (sequence, channel tile) pairs to fill the GPU: a cluster of CTAs
// takes one pair and works on consecutive pieces at once; a warp sends the
// (A, B) of its 8 channels to the same warp of its peers (st.async, counted by
// an mbarrier) and composes theirs.
//
// Bank conflicts: for a step i the 8 groups read rows g S + i of one 16-byte
// (bf16) or 32-byte (fp32) column.  The 128-byte swizzle moves a row's 16-byte
// chunks by row mod 8; S odd (bf16) makes those eight distinct, S = 2 mod 4
// (fp32, half a warp at a time) the four pairs of chunks.
#include <cuda.h>

#include <atomic>

#include "pnn_internal.h"
#include "pnn_seq.h"
#include "recur_common.cuh"
#include "seq_common.cuh"
#include "tc_ptx.cuh"

namespace pnn {
namespace {
using namespace seq;
using namespace tc;

__device__ int g_gave_up;  // set when a bounded wait expired; read and cleared by recur_tile_status

constexpr int kWarps = 8, kThreads = 32 * (kWarps + 1), kTile = 64;
constexpr int kFwdCluster = 16, kBwdCluster = 8;  // CTAs of a cluster at most: what their pairs take of shared memory

struct alignas(64) TMap {
  uint8_t b[128];
};
struct FwdMaps { TMap z, x, h; };
struct BwdMaps { TMap z, x, dh, dz, dx; };

template <typename T>
struct Geo {
  static constexpr int S = kRunSteps<T>;       // steps of a thread
  static constexpr int L = 8 * S;              // steps of a piece
  static constexpr int NB = sizeof(T) / 2;     // boxes of 128-byte rows across the tile
  static constexpr int BOX = L * 128, SLOT = BOX * NB;
  static_assert(BOX % 1024 == 0, "boxes start on the swizzle's period");
};

// ---------------------------------------------------------------- pairs of fp32
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
constexpr f2 kOne2 = 0x3f8000003f800000ull, kNegOne2 = 0xbf800000bf800000ull;

// Both gates of a pair: e = exp(-z), r = 1 / (1 + e), f = r, 1 - f = e r, each
// with its own relative accuracy.  The exponent is cut off at 2^126, where r =
// 2^-126 is still a normal number; taking that off r makes z = -inf give f = 0
// and changes no r above 2^-101.
__device__ __forceinline__ float exp_neg(float y) {  // 2^min(y, 126), NaN kept
  float r;
  asm("{\n\t.reg .f32 c;\n\tmin.NaN.f32 c, %1, 0f42FC0000;\n\tex2.approx.ftz.f32 %0, c;\n\t}" : "=f"(r) : "f"(y));
  return r;
}
__device__ __forceinline__ float rcp(float y) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}
__device__ __forceinline__ void gate2(f2 z, f2& f, f2& g) {
  constexpr float kL = -1.4426950408889634f;
  float a, b;
  upk(mul2(z, pk(kL, kL)), a, b);
  const f2 e = pk(exp_neg(a), exp_neg(b));
  upk(add2(e, kOne2), a, b);
  const f2 r = pk(rcp(a), rcp(b));
  g = mul2(e, r);
  f = add2(r, pk(-1.17549435e-38f, -1.17549435e-38f));
}
__device__ __forceinline__ void gate1(float z, f2& f, f2& g) {
  const float e = exp_neg(z * -1.4426950408889634f), r = rcp(1.f + e), q = e * r, p = r - 1.17549435e-38f;
  f = pk(p, p);
  g = pk(q, q);
}

template <typename T> __device__ __forceinline__ f2 lds2(const char* p);
template <> __device__ __forceinline__ f2 lds2<bf16>(const char* p) {
  const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
  return pk(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <> __device__ __forceinline__ f2 lds2<float>(const char* p) { return *reinterpret_cast<const f2*>(p); }
template <typename T> __device__ __forceinline__ void sts2(char* p, f2 v);
template <> __device__ __forceinline__ void sts2<bf16>(char* p, f2 v) {
  float a, b;
  upk(v, a, b);
  *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(a, b);
}
template <> __device__ __forceinline__ void sts2<float>(char* p, f2 v) { *reinterpret_cast<f2*>(p) = v; }

// ---------------------------------------------------------------- TMA, cluster
__device__ __forceinline__ void tma_load_3d(uint32_t dst, const void* map, int x, int y, int z, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];" ::
          "r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_store_3d(const void* map, int x, int y, int z, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.3d.global.shared::cta.bulk_group [%0, {%1, %2, %3}], [%4];" ::"l"(map), "r"(x),
               "r"(y), "r"(z), "r"(src)
               : "memory");
}
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_peer(uint32_t addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
  return r;
}
// (a, b) to a peer's shared memory; its mbarrier counts the 16 bytes
__device__ __forceinline__ void send(uint32_t to, f2 a, f2 b, uint32_t bar) {
  asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];" ::"r"(to), "l"(a),
               "l"(b), "r"(bar)
               : "memory");
}

// The barriers of a CTA and the pairs its cluster's CTAs send.
template <int NST, int MAXC>
struct Shared {
  uint64_t full[NST], done[NST], arrived[2][kWarps];
  int abort_;
  ulonglong2 peer[MAXC > 1 ? 2 : 1][MAXC > 1 ? kWarps : 1][MAXC][4];
};

template <int NST, int MAXC>
__device__ __forceinline__ void init_shared(Shared<NST, MAXC>& s) {
  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(smem_u32(&s.full[i]), 1);
      mbar_init(smem_u32(&s.done[i]), kWarps);
    }
    for (int i = 0; i < 2 * kWarps; ++i) mbar_init(smem_u32(&s.arrived[0][0] + i), 1);
    s.abort_ = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (MAXC > 1) cluster_sync();  // every CTA of the cluster runs and waits before anything is sent to it
}

__device__ __forceinline__ bool wait_or_abort(uint64_t* bar, uint32_t parity, int* abort_) {
  if (mbar_wait(smem_u32(bar), parity, abort_)) return true;
  *reinterpret_cast<volatile int*>(abort_) = 1;
  g_gave_up = 1;
  return false;
}

// (A, B) of the runs before (UP) or after (down) a lane's run, and of the
// whole piece, from every lane's own.
template <bool UP>
__device__ __forceinline__ void join(f2 A, f2 B, int lane, f2& eA, f2& eB, f2& tA, f2& tB) {
  constexpr uint32_t M = 0xffffffffu;
#pragma unroll
  for (int o = 4; o < 32; o *= 2) {
    const f2 a = UP ? __shfl_up_sync(M, A, o) : __shfl_down_sync(M, A, o);
    const f2 b = UP ? __shfl_up_sync(M, B, o) : __shfl_down_sync(M, B, o);
    if (UP ? lane >= o : lane < 32 - o) {
      B = fma2(A, b, B);
      A = mul2(A, a);
    }
  }
  eA = UP ? __shfl_up_sync(M, A, 4) : __shfl_down_sync(M, A, 4);
  eB = UP ? __shfl_up_sync(M, B, 4) : __shfl_down_sync(M, B, 4);
  if (UP ? lane < 4 : lane >= 28) {
    eA = kOne2;
    eB = 0;
  }
  tA = __shfl_sync(M, A, UP ? 28 + (lane & 3) : lane & 3);
  tB = __shfl_sync(M, B, UP ? 28 + (lane & 3) : lane & 3);
}

// Exchange of one round: the piece's (A, B) goes to every CTA of the cluster;
// s (the value before the round's first piece in scan order) becomes the one
// after its last, the result is the one before this CTA's piece.
template <bool UP, int NST, int MAXC>
__device__ __forceinline__ bool exchange(Shared<NST, MAXC>& sh, int warp, int lane, int rank, int C, int r, f2 tA, f2 tB,
                                         f2& s, f2& mine) {
  const int par = r & 1;
  if (lane == 0) mbar_expect_tx(smem_u32(&sh.arrived[par][warp]), C * 64);
  __syncwarp();
  for (int q = lane >> 2; q < C; q += 8)
    send(in_peer(smem_u32(&sh.peer[par][warp][rank][lane & 3]), q), tA, tB, in_peer(smem_u32(&sh.arrived[par][warp]), q));
  if (!wait_or_abort(&sh.arrived[par][warp], (r >> 1) & 1, &sh.abort_)) return false;
  for (int i = 0; i < C; ++i) {
    const int q = UP ? i : C - 1 - i;
    if (q == rank) mine = s;
    const ulonglong2 v = sh.peer[par][warp][q][lane & 3];
    s = fma2(v.x, s, v.y);
  }
  return true;
}

__device__ __forceinline__ f2 load_pair(const float* p, int64_t c, int64_t D) {
  return p ? pk(c < D ? p[c] : 0.f, c + 1 < D ? p[c + 1] : 0.f) : 0;
}
__device__ __forceinline__ void store_pair(float* p, int64_t c, int64_t D, f2 v) {
  float a, b;
  upk(v, a, b);
  if (c < D) p[c] = a;
  if (c + 1 < D) p[c + 1] = b;
}

// ---------------------------------------------------------------- forward
template <typename T, bool SH, bool CL>  // two CTAs an SM, beside the cluster's pairs
constexpr int kFwdStages = SH ? 6 : sizeof(T) == 4 && CL ? 3 : 4;

template <typename T, bool SH, bool CL>
__global__ void __launch_bounds__(kThreads, 2)
    k_recur_fwd_tile(const __grid_constant__ FwdMaps maps, const __grid_constant__ pnn_recur_args a, int C) {
  using G = Geo<T>;
  constexpr int S = G::S, L = G::L, NST = kFwdStages<T, SH, CL>, SB = (SH ? 1 : 2) * G::SLOT, XO = SH ? 0 : G::SLOT;
  extern __shared__ char raw[];
  __shared__ Shared<NST, CL ? kFwdCluster : 1> sh;
  char* ring = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
  init_shared(sh);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = CL ? (int)cluster_rank() : 0;
  const int b = blockIdx.y, n = recur_len(a, b);
  const int64_t c0 = (int64_t)(CL ? blockIdx.x / C : blockIdx.x) * kTile, D = a.heads * a.width;
  const int pieces = (int)((a.time + L - 1) / L), rounds = (pieces + C - 1) / C;
  bool ok = true;
  if (warp == kWarps) {
    if (lane == 0) {
      const int nb = c0 + kTile / 2 < D ? G::NB : 1;  // boxes that hold channels
      auto issue = [&](int r) {
        const int64_t t0 = (int64_t)(r * C + rank) * L;
        const uint32_t bar = smem_u32(&sh.full[r % NST]), at = smem_u32(ring) + (r % NST) * SB;
        if (t0 >= n) {  // behind the end: nothing is read
          mbar_arrive(bar);
          return;
        }
        mbar_expect_tx(bar, nb * G::BOX * (SH ? 1 : 2));
        for (int i = 0; i < nb; ++i) {
          if (!SH) tma_load_3d(at + i * G::BOX, &maps.z, (int)c0 + i * 32, (int)t0, b, bar);
          tma_load_3d(at + XO + i * G::BOX, &maps.x, (int)c0 + i * 32, (int)t0, b, bar);
        }
      };
      for (int r = 0; r < NST && r < rounds; ++r) issue(r);
      int filled = NST < rounds ? NST : rounds, r = 0;
      for (; r < rounds; ++r) {
        if (!wait_or_abort(&sh.done[r % NST], (r / NST) & 1, &sh.abort_)) break;
        const int64_t t0 = (int64_t)(r * C + rank) * L;
        if (t0 < a.time)
          for (int i = 0; i < nb; ++i)
            tma_store_3d(&maps.h, (int)c0 + i * 32, (int)t0, b, smem_u32(ring) + (r % NST) * SB + XO + i * G::BOX);
        bulk_commit();
        if (r >= 1 && r - 1 + NST < rounds) {
          bulk_wait_read<1>();  // the stage before this one is stored: refill it
          issue(r - 1 + NST);
          filled = r + NST;
        }
      }
      bulk_wait_all();
      if (r < rounds)  // gave up: leave no copy in flight
        for (int q = r; q < filled; ++q) mbar_wait_drain(smem_u32(&sh.full[q % NST]), (q / NST) & 1);
    }
    __syncwarp();
  } else {
    const int grp = lane >> 2, pr = lane & 3, row0 = grp * S;
    const int64_t c = c0 + warp * 8 + pr * 2;
    // this thread's column in a row of a slot, by row mod 8
    const int ch = sizeof(T) == 2 ? warp : 2 * (warp & 3) + (pr >> 1);
    const int in = sizeof(T) == 2 ? pr * 4 : (warp >> 2) * G::BOX + (pr & 1) * 8;
    int off[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) off[j] = row0 * 128 + ((ch ^ ((row0 + j) & 7)) << 4) + in;
    f2 s = a.h0 ? load_pair(a.h0 + b * D, c, D) : 0;
    const T* zp = nullptr;
    T zr[SH ? S : 1];
    auto load_z = [&](int r) {
      const int64_t t = (int64_t)(r * C + rank) * L + row0;
      const T* q = zp + t * a.z_stride_t;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        if (t + i < n && c < D) zr[SH ? i : 0] = *q;
        q += a.z_stride_t;
      }
    };
    if (SH) {
      zp = static_cast<const T*>(a.z) + b * a.z_stride_b + c / a.width;
      load_z(0);
    }
    for (int r = 0; r < rounds; ++r) {
      char* st = ring + (r % NST) * SB;
      const int64_t t0 = (int64_t)(r * C + rank) * L;
      ok = wait_or_abort(&sh.full[r % NST], (r / NST) & 1, &sh.abort_);
      if (!ok) break;
      const bool edge = t0 + L > n;
      const int left = (int)(n - t0) - row0;  // steps of this run before the end
      f2 f[S], u[S], A = kOne2, B = 0;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        f2 g;
        if (SH) gate1(ld(&zr[SH ? i : 0]), f[i], g);
        else gate2(lds2<T>(st + off[i & 7] + i * 128), f[i], g);
        u[i] = mul2(g, lds2<T>(st + XO + off[i & 7] + i * 128));
        if (edge && i >= left) {  // keeps the state
          f[i] = kOne2;
          u[i] = 0;
        }
        A = mul2(A, f[i]);
        B = fma2(f[i], B, u[i]);
      }
      if (SH && r + 1 < rounds) load_z(r + 1);
      f2 eA, eB, tA, tB, h;
      join<true>(A, B, lane, eA, eB, tA, tB);
      f2 mine = s;
      if constexpr (CL) {
        ok = exchange<true>(sh, warp, lane, rank, C, r, tA, tB, s, mine);
        if (!ok) break;
      } else {
        s = fma2(tA, s, tB);
      }
      if (a.saved && grp == 0 && t0 < a.time) store_pair(a.saved + ((int64_t)b * pieces + t0 / L) * D, c, D, mine);
      h = fma2(eA, mine, eB);
#pragma unroll
      for (int i = 0; i < S; ++i) {
        h = fma2(f[i], h, u[i]);
        sts2<T>(st + XO + off[i & 7] + i * 128, edge && i >= left ? 0 : h);
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sh.done[r % NST]));
    }
    if (ok && a.h_last && rank == 0 && grp == 0) store_pair(a.h_last + b * D, c, D, s);
  }
  if (CL) cluster_sync();  // peers may still send to this CTA
}

// ---------------------------------------------------------------- backward
template <typename T, bool SH, bool CL>
constexpr int kBwdStages = SH ? 3 : sizeof(T) == 4 && CL ? 2 : 3;

// SH: dz of a head is the sum over its channels.  Each warp sums its 8; the
// producer warp adds them up to pw channels (8, 16, 32 or 64): the head's dz
// if pw = width, else one of its parts, [batch][time][channels / pw] in part.
template <typename T, bool SH, bool CL>
__global__ void __launch_bounds__(kThreads, 2)
    k_recur_bwd_tile(const __grid_constant__ BwdMaps maps, const __grid_constant__ pnn_recur_args a, int C, float* part,
                     int pw) {
  using G = Geo<T>;
  constexpr int S = G::S, L = G::L, NST = kBwdStages<T, SH, CL>, SB = (SH ? 2 : 3) * G::SLOT;
  constexpr int XO = SH ? 0 : G::SLOT, DO = XO + G::SLOT;
  extern __shared__ char raw[];
  __shared__ Shared<NST, CL ? kBwdCluster : 1> sh;
  __shared__ float zsum[SH ? NST : 1][SH ? L : 1][kWarps];
  char* ring = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
  init_shared(sh);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = CL ? (int)cluster_rank() : 0;
  const int b = blockIdx.y, n = recur_len(a, b);
  const int64_t c0 = (int64_t)(CL ? blockIdx.x / C : blockIdx.x) * kTile, D = a.heads * a.width;
  const int pieces = (int)((a.time + L - 1) / L), rounds = (pieces + C - 1) / C;
  auto first_step = [&](int r) { return (int64_t)((rounds - 1 - r) * C + rank) * L; };
  bool ok = true;
  if (warp == kWarps) {
    const int nb = c0 + kTile / 2 < D ? G::NB : 1;
    auto issue = [&](int r) {
      const int64_t t0 = first_step(r);
      const uint32_t bar = smem_u32(&sh.full[r % NST]), at = smem_u32(ring) + (r % NST) * SB;
      if (t0 >= n) {
        mbar_arrive(bar);
        return;
      }
      mbar_expect_tx(bar, nb * G::BOX * (SH ? 2 : 3));
      for (int i = 0; i < nb; ++i) {
        if (!SH) tma_load_3d(at + i * G::BOX, &maps.z, (int)c0 + i * 32, (int)t0, b, bar);
        tma_load_3d(at + XO + i * G::BOX, &maps.x, (int)c0 + i * 32, (int)t0, b, bar);
        tma_load_3d(at + DO + i * G::BOX, &maps.dh, (int)c0 + i * 32, (int)t0, b, bar);
      }
    };
    int filled = NST < rounds ? NST : rounds, r = 0;
    if (lane == 0)
      for (int q = 0; q < filled; ++q) issue(q);
    for (; r < rounds; ++r) {
      ok = wait_or_abort(&sh.done[r % NST], (r / NST) & 1, &sh.abort_);
      if (!ok) break;
      const int64_t t0 = first_step(r);
      if (lane == 0) {
        if (t0 < a.time)
          for (int i = 0; i < nb; ++i) {
            const uint32_t at = smem_u32(ring) + (r % NST) * SB + i * G::BOX;
            if (!SH) tma_store_3d(&maps.dz, (int)c0 + i * 32, (int)t0, b, at);
            tma_store_3d(&maps.dx, (int)c0 + i * 32, (int)t0, b, at + XO);
          }
        bulk_commit();
      }
      if (SH) {
        const int per = kTile / pw, w8 = pw / 8;
        for (int i = lane; i < L * per; i += 32) {
          const int row = i / per, k = i - row * per;
          const int64_t t = t0 + row, cc = c0 + k * pw;
          if (t < a.time && cc < D) {
            float q = 0.f;
            for (int j = 0; j < w8; ++j) q += zsum[r % NST][row][k * w8 + j];
            if (part) part[(b * a.time + t) * (D / pw) + cc / pw] = q;
            else ::pnn::seq::st(static_cast<T*>(a.dz) + b * a.dz_stride_b + t * a.dz_stride_t + cc / pw, q);
          }
        }
        __syncwarp();
      }
      if (r >= 1 && r - 1 + NST < rounds) {
        if (lane == 0) {
          bulk_wait_read<1>();
          issue(r - 1 + NST);
        }
        filled = r + NST;
      }
    }
    if (lane == 0) {
      bulk_wait_all();
      if (r < rounds)
        for (int q = r; q < filled; ++q) mbar_wait_drain(smem_u32(&sh.full[q % NST]), (q / NST) & 1);
    }
    __syncwarp();
  } else {
    const int grp = lane >> 2, pr = lane & 3, row0 = grp * S;
    const int64_t c = c0 + warp * 8 + pr * 2;
    const int ch = sizeof(T) == 2 ? warp : 2 * (warp & 3) + (pr >> 1);
    const int in = sizeof(T) == 2 ? pr * 4 : (warp >> 2) * G::BOX + (pr & 1) * 8;
    int off[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) off[j] = row0 * 128 + ((ch ^ ((row0 + j) & 7)) << 4) + in;
    f2 R = a.dh_last ? load_pair(a.dh_last + b * D, c, D) : 0;
    const T* zp = nullptr;
    T zr[SH ? S : 1];
    auto load_z = [&](int r) {
      const int64_t t = first_step(r) + row0;
      const T* q = zp + t * a.z_stride_t;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        if (t + i < n && c < D) zr[SH ? i : 0] = *q;
        q += a.z_stride_t;
      }
    };
    if (SH) {
      zp = static_cast<const T*>(a.z) + b * a.z_stride_b + c / a.width;
      load_z(0);
    }
    auto load_state = [&](int r) {
      const int64_t t0 = first_step(r);
      return t0 < n ? load_pair(a.saved + ((int64_t)b * pieces + t0 / L) * D, c, D) : 0;
    };
    f2 before = load_state(0);
    for (int r = 0; r < rounds; ++r) {
      char* st = ring + (r % NST) * SB;
      const int64_t t0 = first_step(r);
      ok = wait_or_abort(&sh.full[r % NST], (r / NST) & 1, &sh.abort_);
      if (!ok) break;
      const bool edge = t0 + L > n;
      const int left = (int)(n - t0) - row0;
      f2 f[S], g[S], A = kOne2, Bf = 0, Bb = 0;
#pragma unroll
      for (int i = 0; i < S; ++i) {
        if (SH) gate1(ld(&zr[SH ? i : 0]), f[i], g[i]);
        else gate2(lds2<T>(st + off[i & 7] + i * 128), f[i], g[i]);
        f2 u = mul2(g[i], lds2<T>(st + XO + off[i & 7] + i * 128));
        if (edge && i >= left) {
          f[i] = kOne2;
          g[i] = u = 0;
        }
        A = mul2(A, f[i]);
        Bf = fma2(f[i], Bf, u);
      }
#pragma unroll
      for (int i = S - 1; i >= 0; --i) {
        f2 d = lds2<T>(st + DO + off[i & 7] + i * 128);
        if (edge && i >= left) d = 0;
        Bb = mul2(f[i], add2(d, Bb));
      }
      if (SH && r + 1 < rounds) load_z(r + 1);
      f2 eA, eB, tA, tB, h, w, mine = R;
      join<true>(A, Bf, lane, eA, eB, tA, tB);
      h = fma2(eA, before, eB);
      if (r + 1 < rounds) before = load_state(r + 1);
      join<false>(A, Bb, lane, eA, eB, tA, tB);
      if constexpr (CL) {
        ok = exchange<false>(sh, warp, lane, rank, C, r, tA, tB, R, mine);
        if (!ok) break;
      } else {
        R = fma2(tA, R, tB);
      }
      w = fma2(eA, mine, eB);
      f2 q[S];  // h_{t-1} - x_t
#pragma unroll
      for (int i = 0; i < S; ++i) {
        const f2 x = lds2<T>(st + XO + off[i & 7] + i * 128);
        q[i] = fma2(x, kNegOne2, h);
        f2 u = mul2(g[i], x);
        if (edge && i >= left) u = 0;
        h = fma2(f[i], h, u);
      }
#pragma unroll
      for (int i = S - 1; i >= 0; --i) {
        const bool past = edge && i >= left;
        f2 d = lds2<T>(st + DO + off[i & 7] + i * 128);
        if (past) d = 0;
        const f2 Gt = add2(d, w);
        w = mul2(f[i], Gt);
        sts2<T>(st + XO + off[i & 7] + i * 128, past ? 0 : mul2(g[i], Gt));
        const f2 dz = past ? 0 : mul2(mul2(g[i], w), q[i]);
        if (!SH) {
          sts2<T>(st + off[i & 7] + i * 128, dz);
        } else {
          float v0, v1;
          upk(dz, v0, v1);
          v0 += v1;
          v0 += __shfl_xor_sync(0xffffffffu, v0, 1);
          v0 += __shfl_xor_sync(0xffffffffu, v0, 2);
          if (pr == 0) zsum[SH ? r % NST : 0][SH ? row0 + i : 0][warp] = v0;
        }
      }
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&sh.done[r % NST]));
    }
    if (ok && a.dh0 && rank == 0 && grp == 0) store_pair(a.dh0 + b * D, c, D, R);
  }
  if (CL) cluster_sync();
}

// ---------------------------------------------------------------- host
// What a tensor map can describe: 16-byte aligned base and positive strides of
// 16-byte multiples (the stride of a single sequence or step does not matter).
bool map_ok(const void* p, int64_t sb, int64_t st, const pnn_recur_args& a, size_t esz) {
  const int64_t per = 16 / esz;
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (a.time == 1 || (st > 0 && st % per == 0 && st * (int64_t)esz < (1LL << 40))) &&
         (a.batch == 1 || (sb > 0 && sb % per == 0 && sb * (int64_t)esz < (1LL << 40)));
}
template <typename T>
int encode(TMap& m, const void* p, int64_t sb, int64_t st, const pnn_recur_args& a) {
  const char* why = nullptr;
  const int64_t D = a.heads * a.width, row = (D * (int64_t)sizeof(T) + 15) / 16 * 16 / (int64_t)sizeof(T);
  if (a.time == 1) st = row;
  if (a.batch == 1) sb = st;
  return encode_tensor_map_3d(&m, p, sizeof(T) == 2, D, a.time, a.batch, st, sb, 128 / (int)sizeof(T), Geo<T>::L, &why);
}

// CTAs that run at once with clusters of 2^i CTAs (i = 0 .. 4; 0: no such
// cluster), asked of the runtime once for each kernel.
struct Slots {
  std::atomic<int> ready{0}, n[5];
};
template <typename K>
cudaError_t slots_of(K kernel, int smem, int most, Slots& s) {
  if (s.ready.load(std::memory_order_acquire)) return cudaSuccess;
  cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e == cudaSuccess && most > 8) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return e;
  for (int i = 0; i < 5; ++i) {
    int n = 0;
    if (1 << i <= most) {
      cudaLaunchConfig_t cfg = {};
      cfg.gridDim = dim3(1 << i);
      cfg.blockDim = dim3(kThreads);
      cfg.dynamicSmemBytes = smem;
      cudaLaunchAttribute at[1];
      at[0].id = cudaLaunchAttributeClusterDimension;
      at[0].val.clusterDim.x = 1 << i;
      at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
      cfg.attrs = at;
      cfg.numAttrs = 1;
      e = cudaOccupancyMaxActiveClusters(&n, kernel, &cfg);
      if (e != cudaSuccess) return e;
    }
    s.n[i].store(n << i, std::memory_order_relaxed);
  }
  s.ready.store(1, std::memory_order_release);
  return cudaSuccess;
}

// CTAs of a cluster: the launch takes about (waves of CTAs over the slots) x
// (pieces of a CTA); a cluster's exchange costs a little at every piece.
int cluster_of(int64_t tiles, int64_t pieces, const Slots& one, const Slots& many) {
  int best = 1;
  double least = 0;
  for (int i = 0; i <= 4; ++i) {
    const int64_t c = 1 << i, n = (i ? many : one).n[i].load(std::memory_order_relaxed);
    if (n < c || (i && c / 2 >= pieces)) break;
    const double cost = (double)((tiles * c + n - 1) / n) * (double)((pieces + c - 1) / c) * (i ? 1.06 + 0.02 * i : 1.0);
    if (i == 0 || cost < least) best = (int)c, least = cost;
  }
  return best;
}

template <typename K, typename... A>
cudaError_t launch(K kernel, int smem, int C, int64_t tiles, int64_t batch, cudaStream_t st, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * C), (unsigned)batch);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = C > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

template <typename T, bool SH>
cudaError_t fwd(const pnn_recur_args& a, cudaStream_t st) {
  constexpr int bytes = (SH ? 1 : 2) * Geo<T>::SLOT;
  constexpr int smem1 = kFwdStages<T, SH, false> * bytes + 1024, smemC = kFwdStages<T, SH, true> * bytes + 1024;
  static Slots one, many;
  cudaError_t e = slots_of(k_recur_fwd_tile<T, SH, false>, smem1, 1, one);
  if (e == cudaSuccess) e = slots_of(k_recur_fwd_tile<T, SH, true>, smemC, kFwdCluster, many);
  if (e != cudaSuccess) return e;
  FwdMaps m;
  if ((!SH && encode<T>(m.z, a.z, a.z_stride_b, a.z_stride_t, a)) || encode<T>(m.x, a.x, a.x_stride_b, a.x_stride_t, a) ||
      encode<T>(m.h, a.h, a.h_stride_b, a.h_stride_t, a))
    return cudaErrorInvalidValue;
  const int64_t tiles = (a.heads * a.width + kTile - 1) / kTile;
  const int C = cluster_of(tiles * a.batch, (a.time + Geo<T>::L - 1) / Geo<T>::L, one, many);
  return C > 1 ? launch(k_recur_fwd_tile<T, SH, true>, smemC, C, tiles, a.batch, st, m, a, C)
               : launch(k_recur_fwd_tile<T, SH, false>, smem1, 1, tiles, a.batch, st, m, a, 1);
}

template <typename T, bool SH>
cudaError_t bwd(const pnn_recur_args& a, float* part, int pw, cudaStream_t st) {
  constexpr int bytes = (SH ? 2 : 3) * Geo<T>::SLOT;
  constexpr int smem1 = kBwdStages<T, SH, false> * bytes + 1024, smemC = kBwdStages<T, SH, true> * bytes + 1024;
  static Slots one, many;
  cudaError_t e = slots_of(k_recur_bwd_tile<T, SH, false>, smem1, 1, one);
  if (e == cudaSuccess) e = slots_of(k_recur_bwd_tile<T, SH, true>, smemC, kBwdCluster, many);
  if (e != cudaSuccess) return e;
  BwdMaps m;
  if ((!SH && (encode<T>(m.z, a.z, a.z_stride_b, a.z_stride_t, a) || encode<T>(m.dz, a.dz, a.dz_stride_b, a.dz_stride_t, a))) ||
      encode<T>(m.x, a.x, a.x_stride_b, a.x_stride_t, a) || encode<T>(m.dh, a.dh, a.dh_stride_b, a.dh_stride_t, a) ||
      encode<T>(m.dx, a.dx, a.dx_stride_b, a.dx_stride_t, a))
    return cudaErrorInvalidValue;
  const int64_t tiles = (a.heads * a.width + kTile - 1) / kTile;
  const int C = cluster_of(tiles * a.batch, (a.time + Geo<T>::L - 1) / Geo<T>::L, one, many);
  return C > 1 ? launch(k_recur_bwd_tile<T, SH, true>, smemC, C, tiles, a.batch, st, m, a, C, part, pw)
               : launch(k_recur_bwd_tile<T, SH, false>, smem1, 1, tiles, a.batch, st, m, a, 1, part, pw);
}
}  // namespace

bool recur_tile_fwd_ok(const pnn_recur_args& a) {
  const size_t e = a.dtype == PNN_DT_BF16 ? 2 : 4;
  const bool z = a.width == 1 ? map_ok(a.z, a.z_stride_b, a.z_stride_t, a, e) : a.width % 8 == 0;
  return z && map_ok(a.x, a.x_stride_b, a.x_stride_t, a, e) && map_ok(a.h, a.h_stride_b, a.h_stride_t, a, e);
}
bool recur_tile_bwd_ok(const pnn_recur_args& a) {
  const size_t e = a.dtype == PNN_DT_BF16 ? 2 : 4;
  const bool z = a.width == 1 ? map_ok(a.z, a.z_stride_b, a.z_stride_t, a, e) && map_ok(a.dz, a.dz_stride_b, a.dz_stride_t, a, e)
                              : a.width % 8 == 0;
  return z && map_ok(a.x, a.x_stride_b, a.x_stride_t, a, e) && map_ok(a.dh, a.dh_stride_b, a.dh_stride_t, a, e) &&
         map_ok(a.dx, a.dx_stride_b, a.dx_stride_t, a, e);
}

cudaError_t launch_recur_tile_fwd(const pnn_recur_args& a, cudaStream_t st) {
  if (a.dtype == PNN_DT_BF16) return a.width > 1 ? fwd<bf16, true>(a, st) : fwd<bf16, false>(a, st);
  return a.width > 1 ? fwd<float, true>(a, st) : fwd<float, false>(a, st);
}
cudaError_t launch_recur_tile_bwd(const pnn_recur_args& a, float* part, int pw, cudaStream_t st) {
  if (a.dtype == PNN_DT_BF16) return a.width > 1 ? bwd<bf16, true>(a, part, pw, st) : bwd<bf16, false>(a, part, pw, st);
  return a.width > 1 ? bwd<float, true>(a, part, pw, st) : bwd<float, false>(a, part, pw, st);
}

cudaError_t recur_tile_status(int* gave_up, cudaStream_t st) {
  const int zero = 0;
  cudaError_t e = cudaMemcpyFromSymbolAsync(gave_up, g_gave_up, sizeof(int), 0, cudaMemcpyDeviceToHost, st);
  if (e == cudaSuccess) e = cudaStreamSynchronize(st);
  if (e == cudaSuccess && *gave_up) e = cudaMemcpyToSymbolAsync(g_gave_up, &zero, sizeof(int), 0, cudaMemcpyHostToDevice, st);
  if (e == cudaSuccess && *gave_up) e = cudaStreamSynchronize(st);
  return e;
}

}  // namespace pnn
