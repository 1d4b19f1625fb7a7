// Gated linear recurrence on tiles: the scan, its backward pass, and the sums
// that let several CTAs share one long sequence.
//
// h_t = f_t h_{t-1} + u_t, u_t = (1 - f_t) x_t, is affine in the state: a run
// of steps is a pair (A, B) = (product of f, its result from zero), and runs
// compose, (A2, B2) after (A1, B1) = (A2 A1, A2 B1 + B2).  This is the parareal
// structure with an exact coarse propagator: the pieces of the time axis are
// solved at once, and the composed pairs give each its true first state.
//
// A CTA owns 64 channels and walks along time in pieces of 8 S steps, held in
// a ring of stages in shared memory.  Each of eight warps takes 8 channels of
// the piece, alone: 4 lanes are its channel pairs, 8 groups of lanes its
// consecutive runs of S steps.  A thread solves its run from zero, the 8 runs
// are composed by warp shuffles, and the thread finishes its steps from its
// true first state, writing h over x in the stage.  No barrier joins the
// warps.  The backward pass is the same recurrence along decreasing time, R_t =
// f_t (dh_t + R_{t+1}); it recomputes the states in fp32 from each piece's
// first state, which the forward saved.
//
// The stages are filled and emptied by one warp through TMA where a tensor map
// can describe the rows (16-byte aligned base and strides), else by two warps
// with cp.async and plain accesses.
//
// With too few (sequence, channel tile) pairs to fill the GPU the pieces of a
// pair are split into segments, one CTA each: a first launch forms every
// segment's (A, B) (it reads z and x, or z and dh, and keeps nothing), the
// second composes those before its own and proceeds as above.  The first
// launch walks away from the end at which the second begins, which then finds
// the latest 100 MB or so in L2.
//
// Bank conflicts: for a step i the 8 groups read rows g S + i of one 16-byte
// (bf16) or 32-byte (fp32) column.  The 128-byte swizzle moves a row's 16-byte
// chunks by row mod 8; S odd (bf16) makes those eight distinct, S = 2 mod 4
// (fp32, half a warp at a time) the four pairs of chunks.
#pragma once
#include <cuda.h>
#include <cuda_bf16.h>

#include <atomic>
#include <type_traits>

#include "pnn_internal.h"
#include "pnn_seq.h"
#include "seq_common.cuh"
#include "tc_ptx.cuh"

namespace pnn {
namespace recur {
using namespace seq;
using namespace tc;

enum Op { FWD, BWD, SUM_FWD, SUM_BWD };
// OWN: a gate for each channel.  HEAD: one for a head of a multiple of 8
// channels; each warp forms its gates once a step.  SPREAD: one for a head of
// any other width; z is spread over the channels when a stage is filled.
enum Gate { OWN, HEAD, SPREAD };

constexpr int kWarps = 8, kTile = 64, kLoaders = 2;

struct alignas(64) TMap {
  uint8_t b[128];
};
struct Maps {
  TMap z, x, dh, h, dz, dx;
};
// What a launch needs beside the caller's arguments.
struct Plan {
  int segments, per;     // CTAs along time, pieces of each
  ulonglong2* sums;      // [batch][segment][tile][32 channel pairs] (A, B), with several segments
  float* part;           // heads wider than pw: fp32 parts of dz, [batch][time][channels / pw]
  int pw;                // channels whose dz one CTA sums (HEAD: 8, 16, 32 or 64; SPREAD: 1)
};

template <typename T, int GATE, int OP>
struct Geo {
  // steps of a thread: what its registers hold of gates and partial results
  static constexpr int S = sizeof(T) == 2 ? (GATE == HEAD ? 11 : 9) : 6;
  static constexpr int L = 8 * S;                   // steps of a piece
  static constexpr int NB = sizeof(T) / 2;          // boxes of 128-byte rows across the tile
  static constexpr int BOX = L * 128, SLOT = BOX * NB;
  static constexpr bool Z = GATE != HEAD, X = OP != SUM_BWD, D = OP == BWD || OP == SUM_BWD;
  // z's slot is there too where the backward keeps partial results in it
  static constexpr bool ZS = Z || (OP == BWD && sizeof(T) == 2);
  static constexpr int ARRAYS = Z + X + D, STAGE = (ZS + X + D) * SLOT;
  static constexpr int XO = ZS ? SLOT : 0, DO = XO + (X ? SLOT : 0);  // offsets of x and dh in a stage
  // stages: what two CTAs of an SM have room for (beside the gates' tables), at most 6
  static constexpr int FIT = (111 * 1024 - (GATE == HEAD ? kWarps * L * 8 : 0)) / STAGE, NST = FIT > 6 ? 6 : FIT;
  static constexpr bool SUM = OP == SUM_FWD || OP == SUM_BWD;
  static_assert(BOX % 1024 == 0, "boxes start on the swizzle's period");
  static_assert(NST >= 2, "a ring");
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

// Gates: e = exp(-z), r = 1 / (1 + e), f = r, 1 - f = e r, each with its own
// relative accuracy.  The exponent is cut off at 2^126, where r = 2^-126 is
// still a normal number; taking that off r makes z = -inf give f = 0 and
// changes no r above 2^-101.
__device__ __forceinline__ float exp2_cut(float y) {  // 2^min(y, 126), NaN kept
  float r;
  asm("{\n\t.reg .f32 c;\n\tmin.NaN.f32 c, %1, 0f42FC0000;\n\tex2.approx.ftz.f32 %0, c;\n\t}" : "=f"(r) : "f"(y));
  return r;
}
__device__ __forceinline__ float rcp(float y) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}
constexpr float kNegLog2e = -1.4426950408889634f, kLeast = 1.17549435e-38f;
__device__ __forceinline__ void gate2(f2 z, f2& f, f2& g) {
  float a, b;
  upk(mul2(z, pk(kNegLog2e, kNegLog2e)), a, b);
  const f2 e = pk(exp2_cut(a), exp2_cut(b));
  upk(add2(e, kOne2), a, b);
  const f2 r = pk(rcp(a), rcp(b));
  g = mul2(e, r);
  f = add2(r, pk(-kLeast, -kLeast));
}
__device__ __forceinline__ float2 gate1(float z) {
  const float e = exp2_cut(z * kNegLog2e), r = rcp(1.f + e);
  return make_float2(r - kLeast, e * r);
}

template <typename T> __device__ __forceinline__ f2 lds2(const char* p) {
  if constexpr (sizeof(T) == 2) {
    const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
    return pk(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  } else {
    return *reinterpret_cast<const f2*>(p);
  }
}
template <typename T> __device__ __forceinline__ void sts2(char* p, f2 v) {
  if constexpr (sizeof(T) == 2) {
    float a, b;
    upk(v, a, b);
    *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(a, b);
  } else {
    *reinterpret_cast<f2*>(p) = v;
  }
}
__device__ __forceinline__ float lds1(const char* p) { return *reinterpret_cast<const float*>(p); }
__device__ __forceinline__ void sts1(char* p, float v) { *reinterpret_cast<float*>(p) = v; }

// ---------------------------------------------------------------- copies
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
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>  // all but this thread's latest N groups have landed
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <int NST>
struct Bars {
  uint64_t full[NST], done[NST];
  int abort_;
};

__device__ __forceinline__ int seq_len(const pnn_recur_args& a, int64_t b) {
  if (!a.lengths) return (int)a.time;
  const int64_t n = a.lengths[b];
  return (int)(n < 0 ? 0 : n > a.time ? a.time : n);
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

// A gate shared by the 8 channels of a warp: its lanes form the L gates of a
// piece once, for one row each (every fourth lane's run would otherwise form
// the same ones), into a table of the warp's own.
template <typename T, int L>
struct GateTable {
  static constexpr int N = (L + 31) / 32;
  const T* p;             // this lane's first row of the next piece
  int64_t stride, piece;  // elements from row to row + 32, from piece to piece
  T z[N];                 // the next piece's, as loaded
  __device__ __forceinline__ void load(int left, int lane) {  // left: rows of that piece before the end
    const T* q = p;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (lane + 32 * i < (left < L ? left : L)) z[i] = *q;
      q += stride;
    }
    p += piece;
  }
  __device__ __forceinline__ void form(float2* table, int lane) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (lane + 32 * i < L) table[lane + 32 * i] = gate1(ld(&z[i]));
    __syncwarp();
  }
};

// ---------------------------------------------------------------- filling and emptying stages
// Byte offset of the swizzled word `word` (0 .. 31) of a row in a box.
__device__ __forceinline__ int word_at(int row, int word) { return row * 128 + (((word >> 2) ^ (row & 7)) << 4) + (word & 3) * 4; }

// The rows of one loader warp, and its lane's word in each (by row mod 8).  A
// lane has channels 2 l and 2 l + 1 (bf16) or l and l + 32 (fp32).
template <typename T, int R, int BOX>
struct Rows {
  int row0, ca, off[8];
  bool one, two;  // the lane's channels exist
  int64_t D;
  __device__ __forceinline__ Rows(int row0_, int lane, int64_t c0, int64_t D_) : row0(row0_), D(D_) {
    ca = sizeof(T) == 2 ? 2 * lane : lane;
    one = c0 + ca < D;
    two = c0 + ca + (sizeof(T) == 2 ? 1 : 32) < D;
#pragma unroll
    for (int j = 0; j < 8; ++j) off[j] = word_at(row0 + j, lane);
  }
  // f(o) for this warp's rows that exist, o the lane's offset; eight rows at a
  // time, without a test where all eight exist
  template <typename F>
  __device__ __forceinline__ void each(int rows, F f) const {
    const int m = rows - row0 < R ? rows - row0 : R;
#pragma unroll 1
    for (int h = 0; h < m; h += 8) {
      if (h + 8 <= m) {
#pragma unroll
        for (int i = 0; i < 8; ++i) f(off[i] + h * 128);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (h + i < m) f(off[i] + h * 128);
      }
    }
  }
  // p: row 0 and channel 0 of the piece.  One cp.async of 4 bytes for each
  // word that lies on one, else value by value.
  __device__ __forceinline__ void fill(char* slot, const T* p, int64_t stride, int rows) const {
    const uint32_t to = smem_u32(slot);
    const T* q = p + row0 * stride + ca;
    if constexpr (sizeof(T) == 4) {
      each(rows, [&](int o) {
        if (one) cp_async4(to + o, q);
        if (two) cp_async4(to + o + BOX, q + 32);
        q += stride;
      });
    } else if (((reinterpret_cast<uintptr_t>(p) | (uintptr_t)stride * 2) & 3) == 0) {
      each(rows, [&](int o) {
        if (two) cp_async4(to + o, q);
        else if (one) *reinterpret_cast<T*>(slot + o) = *q;
        q += stride;
      });
    } else {
      const int m = rows - row0 < R ? rows - row0 : R;
      const uint16_t* v = reinterpret_cast<const uint16_t*>(q);
#pragma unroll 1
      for (int h = 0; h < m; h += 8) {
        uint16_t lo[8], hi[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          if (h + i < m && one) lo[i] = v[0];
          if (h + i < m && two) hi[i] = v[1];
          v += stride;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (h + i < R) *reinterpret_cast<uint32_t*>(slot + off[i] + h * 128) = lo[i] | (uint32_t)hi[i] << 16;
      }
    }
  }
  // z of each channel's head (p: row 0, head 0)
  __device__ __forceinline__ void fill_spread(char* slot, const T* p, int64_t stride, int rows, int64_t ha, int64_t hb) const {
    const int m = rows - row0 < R ? rows - row0 : R;
    const T* v = p + row0 * stride;
#pragma unroll 1
    for (int h = 0; h < m; h += 8) {
      T va[8], vb[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (h + i < m && one) va[i] = v[ha];
        if (h + i < m && two) vb[i] = v[hb];
        v += stride;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        char* w = slot + off[i] + h * 128;
        if (h + i >= R) continue;
        if constexpr (sizeof(T) == 2) {
          *reinterpret_cast<__nv_bfloat162*>(w) = __halves2bfloat162(va[i], vb[i]);
        } else {
          *reinterpret_cast<float*>(w) = va[i];
          *reinterpret_cast<float*>(w + BOX) = vb[i];
        }
      }
    }
  }
  // the rows of a finished slot to global memory
  __device__ __forceinline__ void empty(const char* slot, T* p, int64_t stride, int rows) const {
    T* q = p + row0 * stride + ca;
    if constexpr (sizeof(T) == 4) {
      each(rows, [&](int o) {
        if (one) q[0] = lds1(slot + o);
        if (two) q[32] = lds1(slot + o + BOX);
        q += stride;
      });
    } else if (((reinterpret_cast<uintptr_t>(p) | (uintptr_t)stride * 2) & 3) == 0) {
      each(rows, [&](int o) {
        const __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162*>(slot + o);
        if (two) *reinterpret_cast<__nv_bfloat162*>(q) = v;
        else if (one) *q = v.x;
        q += stride;
      });
    } else {
      each(rows, [&](int o) {
        const __nv_bfloat162 v = *reinterpret_cast<const __nv_bfloat162*>(slot + o);
        if (one) q[0] = v.x;
        if (two) q[1] = v.y;
        q += stride;
      });
    }
  }
  // dz of every channel in fp32 (heads of any width; p: row 0, channel 0 of
  // the tile): bf16 pairs left theirs where z and dh were, fp32 ones where z was
  __device__ __forceinline__ void empty_spread(const char* zslot, const char* dslot, float* p, int rows) const {
    float* q = p + row0 * D + ca;
    each(rows, [&](int o) {
      if (one) q[0] = lds1(zslot + o);
      if (two) q[sizeof(T) == 2 ? 1 : 32] = lds1(sizeof(T) == 2 ? dslot + o : zslot + BOX + o);
      q += D;
    });
  }
};

// dz of the rows row0 .. row1 of a piece, one gate for a head.  Each channel
// pair left the sum of its two shares where its dh was: the 4 lanes of a warp
// one swizzled 16-byte chunk (bf16), or two with every other word (fp32).
template <typename T, typename G>
__device__ __forceinline__ void sum_heads(const char* slot, const pnn_recur_args& a, const Plan& pl, int64_t b, int64_t t0,
                                          int row0, int row1, int64_t c0, int64_t D, int lane) {
  const int w8 = pl.pw / 8, sh = 31 - __clz(kTile / pl.pw);  // 64 / pw parts in a row
  for (int i = lane; i < (row1 - row0) << sh; i += 32) {
    const int row = row0 + (i >> sh), k = i & ((1 << sh) - 1);
    const int64_t t = t0 + row, c = c0 + k * pl.pw;
    if (t >= a.time || c >= D) continue;
    float q = 0.f;
#pragma unroll 4
    for (int w = k * w8; w < (k + 1) * w8; ++w) {
      if constexpr (sizeof(T) == 2) {
        const float4 v = *reinterpret_cast<const float4*>(slot + row * 128 + ((w ^ (row & 7)) << 4));
        q += (v.x + v.y) + (v.z + v.w);
      } else {
        const char* p = slot + (w >> 2) * G::BOX + row * 128;
        const float4 v = *reinterpret_cast<const float4*>(p + (((2 * (w & 3)) ^ (row & 7)) << 4));
        const float4 u = *reinterpret_cast<const float4*>(p + (((2 * (w & 3) + 1) ^ (row & 7)) << 4));
        q += (v.x + v.z) + (u.x + u.z);
      }
    }
    if (pl.part) pl.part[(b * a.time + t) * (D / pl.pw) + c / pl.pw] = q;
    else st(static_cast<T*>(a.dz) + b * a.dz_stride_b + t * a.dz_stride_t + c / pl.pw, q);
  }
}
// ---------------------------------------------------------------- the kernel
template <typename T, int GATE, bool TMA, int OP>
__global__ void __launch_bounds__(32 * (kWarps + (TMA ? 1 : kLoaders)), 2)
    k_recur_tile(const __grid_constant__ Maps maps, const __grid_constant__ pnn_recur_args a, const __grid_constant__ Plan pl,
                 int* gave_up) {
  using G = Geo<T, GATE, OP>;
  constexpr int S = G::S, L = G::L, NST = G::NST, SB = G::STAGE, XO = G::XO, DO = G::DO;
  constexpr bool UP = OP == FWD || OP == SUM_BWD;  // the pieces of a segment in increasing time
  extern __shared__ char raw[];
  __shared__ Bars<NST> bars;
  __shared__ float2 table[GATE == HEAD ? kWarps : 1][GATE == HEAD ? L : 1];
  char* ring = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(smem_u32(&bars.full[i]), TMA ? 1 : kLoaders);
      mbar_init(smem_u32(&bars.done[i]), kWarps);
    }
    bars.abort_ = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int64_t D = a.heads * a.width;
  const int tiles = (int)((D + kTile - 1) / kTile), tile = blockIdx.x % tiles;
  const int seg = blockIdx.x / tiles + (OP == SUM_BWD ? 1 : 0);  // the outermost segment's sum is not needed
  const int b = blockIdx.y, n = seq_len(a, b);
  const int64_t c0 = (int64_t)tile * kTile;
  const int pieces = (int)((a.time + L - 1) / L), p0 = seg * pl.per;
  const int rounds = p0 + pl.per < pieces ? pl.per : pieces - p0;
  auto first_step = [&](int r) { return (UP ? p0 + r : p0 + rounds - 1 - r) * L; };  // below time, which fits an int
  auto wait = [&](uint64_t* bar, int r) {
    if (mbar_wait(smem_u32(bar), (r / NST) & 1, &bars.abort_)) return true;
    *reinterpret_cast<volatile int*>(&bars.abort_) = 1;
    *reinterpret_cast<volatile int*>(gave_up) = 1;
    return false;
  };

  if (TMA && warp == kWarps) {
    // -------------------------------------------------------------- TMA: one lane fills and stores
    const int nb = c0 + kTile / 2 < D ? G::NB : 1;  // boxes that hold channels
    auto issue = [&](int r) {
      const int t0 = (int)first_step(r);
      const uint32_t bar = smem_u32(&bars.full[r % NST]), at = smem_u32(ring) + (r % NST) * SB;
      if (t0 >= n) {  // behind the end: nothing is read
        mbar_arrive(bar);
        return;
      }
      mbar_expect_tx(bar, nb * G::BOX * G::ARRAYS);
      for (int i = 0; i < nb; ++i) {
        const int x = (int)c0 + i * 32;
        if (G::Z) tma_load_3d(at + i * G::BOX, &maps.z, x, t0, b, bar);
        if (G::X) tma_load_3d(at + XO + i * G::BOX, &maps.x, x, t0, b, bar);
        if (G::D) tma_load_3d(at + DO + i * G::BOX, &maps.dh, x, t0, b, bar);
      }
    };
    int filled = NST < rounds ? NST : rounds, r = 0;
    if (lane == 0)
      for (int q = 0; q < filled; ++q) issue(q);
    for (; r < rounds; ++r) {
      if (!wait(&bars.done[r % NST], r)) break;
      const int t0 = first_step(r);
      if (!G::SUM && lane == 0) {
        for (int i = 0; i < nb; ++i) {
          const uint32_t at = smem_u32(ring) + (r % NST) * SB + i * G::BOX;
          const int x = (int)c0 + i * 32;
          if (OP == FWD) tma_store_3d(&maps.h, x, t0, b, at + XO);
          if (OP == BWD) tma_store_3d(&maps.dx, x, t0, b, at + XO);
          if (OP == BWD && GATE == OWN) tma_store_3d(&maps.dz, x, t0, b, at);
        }
        bulk_commit();
      }
      if (OP == BWD && GATE == HEAD) {
        sum_heads<T, G>(ring + (r % NST) * SB + DO, a, pl, b, t0, 0, L, c0, D, lane);
        __syncwarp();
      }
      if (r + NST < rounds) {
        if (lane == 0) {
          if (!G::SUM) bulk_wait_read<0>();  // the store has left the stage: refill it
          issue(r + NST);
        }
        filled = r + NST + 1;
      }
    }
    if (lane == 0) {
      bulk_wait_all();
      if (r < rounds)  // gave up: leave no copy in flight
        for (int q = r; q < filled; ++q) mbar_wait_drain(smem_u32(&bars.full[q % NST]), (q / NST) & 1);
    }
    __syncwarp();
  } else if (!TMA && warp >= kWarps) {
    // -------------------------------------------------------------- two warps, half of a piece's rows each
    constexpr int R = L / kLoaders;
    static_assert(L % kLoaders == 0, "rows of a loader");
    const Rows<T, R, G::BOX> rw((warp - kWarps) * R, lane, c0, D);
    const int64_t ha = GATE == SPREAD ? (c0 + rw.ca) / a.width : 0;
    const int64_t hb = GATE == SPREAD ? (c0 + rw.ca + (sizeof(T) == 2 ? 1 : 32)) / a.width : 0;
    auto src = [&](const void* p, int64_t sb, int64_t st, int64_t t0) { return static_cast<const T*>(p) + b * sb + t0 * st; };
    auto dst = [&](void* p, int64_t sb, int64_t st, int64_t t0) { return static_cast<T*>(p) + b * sb + t0 * st + c0; };
    // a stage is handed over when the K stages after it are under way
    constexpr int K = NST - 2;
    for (int r = 0; r < rounds + NST; ++r) {
      char* at = ring + (r % NST) * SB;
      if (r >= NST) {
        const int q = r - NST;
        if (q >= rounds || !wait(&bars.done[r % NST], q)) break;
        if (!G::SUM) {
          const int t0 = first_step(q);
          const int rows = a.time - t0 < L ? (int)(a.time - t0) : L;
          if (OP == FWD) rw.empty(at + XO, dst(a.h, a.h_stride_b, a.h_stride_t, t0), a.h_stride_t, rows);
          if (OP == BWD) rw.empty(at + XO, dst(a.dx, a.dx_stride_b, a.dx_stride_t, t0), a.dx_stride_t, rows);
          if (OP == BWD && GATE == OWN) rw.empty(at, dst(a.dz, a.dz_stride_b, a.dz_stride_t, t0), a.dz_stride_t, rows);
          if (OP == BWD && GATE == HEAD) sum_heads<T, G>(at + DO, a, pl, b, t0, rw.row0, rw.row0 + R, c0, D, lane);
          if (OP == BWD && GATE == SPREAD) rw.empty_spread(at, at + DO, pl.part + (b * a.time + t0) * D + c0, rows);
          __syncwarp();
        }
      }
      if (r < rounds) {
        const int t0 = first_step(r);
        const int rows = n - t0 < L ? n - t0 : L;  // rows that are there (none behind the end)
        if (rows > 0) {
          if (G::X) rw.fill(at + XO, src(a.x, a.x_stride_b, a.x_stride_t, t0) + c0, a.x_stride_t, rows);
          if (G::D) rw.fill(at + DO, src(a.dh, a.dh_stride_b, a.dh_stride_t, t0) + c0, a.dh_stride_t, rows);
          if (GATE == OWN) rw.fill(at, src(a.z, a.z_stride_b, a.z_stride_t, t0) + c0, a.z_stride_t, rows);
          if (GATE == SPREAD) rw.fill_spread(at, src(a.z, a.z_stride_b, a.z_stride_t, t0), a.z_stride_t, rows, ha, hb);
        }
      }
      cp_async_commit();
      if (r >= K && r - K < rounds) {
        cp_async_wait<K>();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&bars.full[(r - K) % NST]));
      }
    }
    cp_async_wait_all();
  } else {
    // -------------------------------------------------------------- eight warps compute
    const int grp = lane >> 2, pr = lane & 3, row0 = grp * S;
    const int64_t c = c0 + warp * 8 + pr * 2;
    // this thread's column in a row of a slot, by row mod 8
    const int ch = sizeof(T) == 2 ? warp : 2 * (warp & 3) + (pr >> 1);
    const int in = sizeof(T) == 2 ? pr * 4 : (warp >> 2) * G::BOX + (pr & 1) * 8;
    int off[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) off[j] = row0 * 128 + ((ch ^ ((row0 + j) & 7)) << 4) + in;
    GateTable<T, L> gates;
    if (GATE == HEAD) {
      gates.p = static_cast<const T*>(a.z) + b * a.z_stride_b + (c0 + warp * 8 < D ? c0 + warp * 8 : 0) / a.width +
                (int64_t)(first_step(0) + lane) * a.z_stride_t;
      gates.stride = 32 * a.z_stride_t;
      gates.piece = (UP ? L : -L) * a.z_stride_t;
      gates.load(n - first_step(0), lane);
    }
    // the value carried along the pieces: the state, or R; composed over the segments before
    ulonglong2* sums = pl.sums + ((int64_t)b * pl.segments * tiles + tile) * 32 + warp * 4 + pr;
    f2 s = 0, tot = kOne2;  // SUM: (tot, s) of the pieces so far
    if (OP == FWD) {
      s = a.h0 ? load_pair(a.h0 + b * D, c, D) : 0;
      for (int q = 0; q < seg; ++q) {
        const ulonglong2 v = sums[(int64_t)q * tiles * 32];
        s = fma2(v.x, s, v.y);
      }
    }
    if (OP == BWD) {
      s = a.dh_last ? load_pair(a.dh_last + b * D, c, D) : 0;
      for (int q = pl.segments - 1; q > seg; --q) {
        const ulonglong2 v = sums[(int64_t)q * tiles * 32];
        s = fma2(v.x, s, v.y);
      }
    }
    float* saved = a.saved + ((int64_t)b * pieces + (UP ? p0 : p0 + rounds - 1)) * D;  // the piece's first state
    f2 before = OP == BWD && first_step(0) < n ? load_pair(saved, c, D) : 0;
    bool ok = true;
    for (int r = 0; r < rounds; ++r) {
      char* at = ring + (r % NST) * SB;
      const int t0 = first_step(r);
      ok = wait(&bars.full[r % NST], r);
      if (!ok) break;
      if (GATE == HEAD) {
        gates.form(table[GATE == HEAD ? warp : 0], lane);
        if (r + 1 < rounds) gates.load(n - first_step(r + 1), lane);
      }
      const int left = t0 < n ? n - t0 - row0 : 0;
      // EDGE: the piece reaches behind the end, where steps keep the state
      auto piece = [&](auto edge) {
        constexpr bool EDGE = decltype(edge)::value;
        auto gate_at = [&](int i, f2& f, f2& g) {
          if (GATE == HEAD) {
            const float2 q = table[GATE == HEAD ? warp : 0][row0 + i];
            f = pk(q.x, q.x);
            g = pk(q.y, q.y);
          } else {
            gate2(lds2<T>(at + off[i & 7] + i * 128), f, g);
          }
          if (EDGE && i >= left) {
            f = kOne2;
            g = 0;
          }
        };
        auto x_at = [&](int i) {
          const f2 x = lds2<T>(at + XO + off[i & 7] + i * 128);
          return EDGE && i >= left ? 0 : x;
        };
        auto d_at = [&](int i) {
          const f2 d = lds2<T>(at + DO + off[i & 7] + i * 128);
          return EDGE && i >= left ? 0 : d;
        };
        f2 eA, eB, tA, tB;
        if constexpr (G::SUM) {
          f2 A = kOne2, B = 0;
#pragma unroll
          for (int j = 0; j < S; ++j) {
            const int i = OP == SUM_FWD ? j : S - 1 - j;
            f2 f, g;
            gate_at(i, f, g);
            A = mul2(A, f);
            B = OP == SUM_FWD ? fma2(f, B, mul2(g, x_at(i))) : mul2(f, add2(d_at(i), B));
          }
          join<OP == SUM_FWD>(A, B, lane, eA, eB, tA, tB);
          s = fma2(tot, tB, s);  // this piece comes before those so far
          tot = mul2(tot, tA);
        } else if constexpr (OP == FWD) {
          // of the run's first i + 1 steps; both channels of a shared gate have the same A
          std::conditional_t<GATE == HEAD, float, f2> A[S];
          f2 B[S], P = kOne2;
#pragma unroll
          for (int i = 0; i < S; ++i) {
            f2 f, g;
            gate_at(i, f, g);
            const f2 u = mul2(g, x_at(i));
            P = i ? mul2(P, f) : f;
            B[i] = i ? fma2(f, B[i - 1], u) : u;
            if constexpr (GATE == HEAD) A[i] = __uint_as_float((uint32_t)P);
            else A[i] = P;
          }
          auto A_at = [&](int i) {
            if constexpr (GATE == HEAD) return pk(A[i], A[i]);
            else return A[i];
          };
          join<true>(P, B[S - 1], lane, eA, eB, tA, tB);
          if (a.saved && grp == 0) store_pair(saved, c, D, s);
          saved += D;
          const f2 h = fma2(eA, s, eB);
          s = fma2(tA, s, tB);
#pragma unroll
          for (int i = 0; i < S; ++i) sts2<T>(at + XO + off[i & 7] + i * 128, EDGE && i >= left ? 0 : fma2(A_at(i), h, B[i]));
        } else {
          // what a thread keeps for its second walk: the gates (a shared one is read again from the table), and
          // h_{t-1} - x_t (bf16: as two fp32 words where z and x were)
          constexpr bool KEEP = GATE != HEAD, SPILL = sizeof(T) == 2;
          [[maybe_unused]] f2 f[KEEP ? S : 1] = {}, g[KEEP ? S : 1] = {}, q[SPILL ? 1 : S] = {};
          f2 A = kOne2, Bf = 0, Bb = 0;
          auto gate_kept = [&](int i, f2& fi, f2& gi) {
            if constexpr (KEEP) fi = f[i], gi = g[i];
            else gate_at(i, fi, gi);
          };
#pragma unroll
          for (int i = 0; i < S; ++i) {
            f2 fi, gi;
            gate_at(i, fi, gi);
            if constexpr (KEEP) f[i] = fi, g[i] = gi;
            A = mul2(A, fi);
            Bf = fma2(fi, Bf, mul2(gi, x_at(i)));
          }
#pragma unroll
          for (int i = S - 1; i >= 0; --i) {
            f2 fi, gi;
            gate_kept(i, fi, gi);
            Bb = mul2(fi, add2(d_at(i), Bb));
          }
          join<false>(A, Bb, lane, eA, eB, tA, tB);
          f2 w = fma2(eA, s, eB);
          s = fma2(tA, s, tB);
          join<true>(A, Bf, lane, eA, eB, tA, tB);
          f2 h = fma2(eA, before, eB);
          saved -= D;
          before = r + 1 < rounds && first_step(r + 1) < n ? load_pair(saved, c, D) : 0;
#pragma unroll
          for (int i = 0; i < S; ++i) {
            f2 fi, gi;
            gate_kept(i, fi, gi);
            const f2 x = x_at(i), d = fma2(x, kNegOne2, h);
            if constexpr (SPILL) {
              float lo, hi;
              upk(d, lo, hi);
              sts1(at + off[i & 7] + i * 128, lo);
              sts1(at + XO + off[i & 7] + i * 128, hi);
            } else {
              q[i] = d;
            }
            h = fma2(fi, h, mul2(gi, x));
          }
#pragma unroll
          for (int i = S - 1; i >= 0; --i) {
            f2 fi, gi, d;
            gate_kept(i, fi, gi);
            if constexpr (SPILL) d = pk(lds1(at + off[i & 7] + i * 128), lds1(at + XO + off[i & 7] + i * 128));
            else d = q[i];
            const f2 Gt = add2(d_at(i), w);
            w = mul2(fi, Gt);
            f2 dx = mul2(gi, Gt), dz = mul2(mul2(gi, w), d);
            if (EDGE && i >= left) dx = dz = 0;
            sts2<T>(at + XO + off[i & 7] + i * 128, dx);
            float lo, hi;
            upk(dz, lo, hi);
            if constexpr (GATE == HEAD) {
              sts1(at + DO + off[i & 7] + i * 128, lo + hi);
            } else if constexpr (GATE == SPREAD && sizeof(T) == 2) {
              sts1(at + off[i & 7] + i * 128, lo);
              sts1(at + DO + off[i & 7] + i * 128, hi);
            } else {
              sts2<T>(at + off[i & 7] + i * 128, dz);
            }
          }
        }
      };
      if (n - t0 < L) piece(std::true_type());
      else piece(std::false_type());
      if (TMA && !G::SUM) fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.done[r % NST]));
    }
    if (ok && grp == 0) {
      if (G::SUM) sums[(int64_t)seg * tiles * 32] = make_ulonglong2(tot, s);
      if (OP == FWD && a.h_last && seg == pl.segments - 1) store_pair(a.h_last + b * D, c, D, s);
      if (OP == BWD && a.dh0 && seg == 0) store_pair(a.dh0 + b * D, c, D, s);
    }
  }
}

// ---------------------------------------------------------------- host
// What a tensor map can describe: 16-byte aligned base and positive strides of
// 16-byte multiples (the stride of a single sequence or step does not matter).
inline bool map_ok(const void* p, int64_t sb, int64_t st, const pnn_recur_args& a, size_t esz) {
  const int64_t per = 16 / esz;
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (a.time == 1 || (st > 0 && st % per == 0 && st * (int64_t)esz < (1LL << 40))) &&
         (a.batch == 1 || (sb > 0 && sb % per == 0 && sb * (int64_t)esz < (1LL << 40)));
}

template <typename T, int L>
bool encode(TMap& m, const void* p, int64_t sb, int64_t st, const pnn_recur_args& a) {
  const char* why = nullptr;
  const int64_t D = a.heads * a.width, row = (D * (int64_t)sizeof(T) + 15) / 16 * 16 / (int64_t)sizeof(T);
  if (a.time == 1) st = row;
  if (a.batch == 1) sb = st;
  return encode_tensor_map_3d(&m, p, sizeof(T) == 2, D, a.time, a.batch, st, sb, 128 / (int)sizeof(T), L, &why) == 0;
}

template <typename T, int GATE, bool TMA, int OP>
cudaError_t launch_one(const Maps& m, const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st) {
  constexpr int smem = Geo<T, GATE, OP>::NST * Geo<T, GATE, OP>::STAGE + 1024;
  const auto kernel = k_recur_tile<T, GATE, TMA, OP>;
  static std::atomic<uint64_t> ready{0};  // one bit a device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  const int64_t tiles = (a.heads * a.width + kTile - 1) / kTile;
  const int segs = pl.segments - (OP == SUM_FWD || OP == SUM_BWD ? 1 : 0);
  kernel<<<dim3((unsigned)(tiles * segs), (unsigned)a.batch), 32 * (kWarps + (TMA ? 1 : kLoaders)), smem, st>>>(m, a, pl, gave_up);
  return cudaGetLastError();
}

template <typename T, int GATE, bool TMA>
cudaError_t run(bool backward, const Maps& m, const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  if (pl.segments > 1)
    e = backward ? launch_one<T, GATE, TMA, SUM_BWD>(m, a, pl, gave_up, st) : launch_one<T, GATE, TMA, SUM_FWD>(m, a, pl, gave_up, st);
  if (e != cudaSuccess) return e;
  return backward ? launch_one<T, GATE, TMA, BWD>(m, a, pl, gave_up, st) : launch_one<T, GATE, TMA, FWD>(m, a, pl, gave_up, st);
}

// Which form takes these arguments, and its launches.
template <typename T>
cudaError_t dispatch(bool backward, const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st) {
  const int gate = a.width == 1 ? OWN : a.width % 8 == 0 ? HEAD : SPREAD;
  constexpr size_t e = sizeof(T);
  bool tma = gate != SPREAD && map_ok(a.x, a.x_stride_b, a.x_stride_t, a, e);
  if (gate == OWN) tma = tma && map_ok(a.z, a.z_stride_b, a.z_stride_t, a, e);
  if (!backward) tma = tma && map_ok(a.h, a.h_stride_b, a.h_stride_t, a, e);
  if (backward) tma = tma && map_ok(a.dh, a.dh_stride_b, a.dh_stride_t, a, e) && map_ok(a.dx, a.dx_stride_b, a.dx_stride_t, a, e);
  if (backward && gate == OWN) tma = tma && map_ok(a.dz, a.dz_stride_b, a.dz_stride_t, a, e);
  Maps m;
  if (tma) {
    const auto enc = gate == OWN ? encode<T, Geo<T, OWN, FWD>::L> : encode<T, Geo<T, HEAD, FWD>::L>;
    bool ok = enc(m.x, a.x, a.x_stride_b, a.x_stride_t, a);
    if (gate == OWN) ok = ok && enc(m.z, a.z, a.z_stride_b, a.z_stride_t, a);
    if (!backward) ok = ok && enc(m.h, a.h, a.h_stride_b, a.h_stride_t, a);
    if (backward) ok = ok && enc(m.dh, a.dh, a.dh_stride_b, a.dh_stride_t, a) && enc(m.dx, a.dx, a.dx_stride_b, a.dx_stride_t, a);
    if (backward && gate == OWN) ok = ok && enc(m.dz, a.dz, a.dz_stride_b, a.dz_stride_t, a);
    if (!ok) return cudaErrorInvalidValue;
    return gate == OWN ? run<T, OWN, true>(backward, m, a, pl, gave_up, st) : run<T, HEAD, true>(backward, m, a, pl, gave_up, st);
  }
  if (gate == OWN) return run<T, OWN, false>(backward, m, a, pl, gave_up, st);
  if (gate == HEAD) return run<T, HEAD, false>(backward, m, a, pl, gave_up, st);
  return run<T, SPREAD, false>(backward, m, a, pl, gave_up, st);
}

cudaError_t run_bf16(bool backward, const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st);
cudaError_t run_f32(bool backward, const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st);

}  // namespace recur
}  // namespace pnn
