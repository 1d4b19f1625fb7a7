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
// true first state, writing h over x in the stage.  The backward pass is the
// same recurrence along decreasing time, R_t = f_t (dh_t + R_{t+1}); it
// recomputes the states in fp32 from each piece's first state, which the
// forward saved.
//
// One warp fills the stages through TMA.  Where a tensor map can describe the
// rows (16-byte aligned base and strides) it stores the results from there too
// and no barrier joins the other warps.  Other rows come through one map for
// every 16-byte phase a row can start in and lie in the stage as they do in
// memory, and the computing warps write them out row by row a round later (from
// their registers, 8 channels a row, they took 200 us instead of 147 for the
// odd bf16 rows below; by warps of their own, 172).
//
// Bound: HBM where rows are aligned; 8 x 4096 x 2048 bf16 takes 67 us (6.0
// TB/s), backward 113 (5.9), fp32 134 and 225 (6.0).  Rows of 2046 take 117 and
// 232, of 2047 146 and 329 (single values through shared memory), 1023 fp32 90
// and 171; 32 heads of 64 63 and 119 (dz of a head is summed over its
// channels), 400 of 5 88 and 270 (every walk reads both channels' gates from the
// table again, the backward has four), 399 of them, in rows of 1995, 289 and
// 514 (each place found anew for every access, a bf16 pair in two of them; 84
// and 32 bytes of registers spilled).
//
// With too few (sequence, channel tile) pairs to fill the GPU the pieces of a
// pair are split into segments, one CTA each: a first launch forms every
// segment's (A, B) (it reads z and x, or z and dh, and keeps nothing), the
// second composes those before its own and proceeds as above.  The first
// launch walks towards the end at which the second begins, so that short
// sequences come from L2 the second time (hints on what L2 should keep changed
// nothing for long ones).
//
// Bank conflicts: for a step i the 8 groups read rows g S + i of one 16-byte
// (bf16) or 32-byte (fp32) column.  TMA's 128-byte swizzle moves a row's
// 16-byte chunks by row mod 8; S odd (bf16) makes those eight distinct, S = 2
// mod 4 (fp32, half a warp at a time) the four pairs of chunks.  Other rows lie
// 144 (bf16, the 8 groups apart but for one) or 288 bytes apart.
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
// channels.  SPREAD: one for a head of any other width, so that a warp's 8
// channels lie in up to 4 heads.  Shared gates each warp forms once a step.
enum Gate { OWN, HEAD, SPREAD };

// SWZ: rows as TMA swizzles them.  PAIR, ELEM: rows as they lie in memory,
// channel pairs on whole words (PAIR) or anywhere (ELEM).
enum Layout { SWZ, PAIR, ELEM };

constexpr int kWarps = 8, kTile = 64;

struct alignas(64) TMap {
  uint8_t b[128];
};
struct Maps {
  TMap z, x, dh, h, dz, dx;
};
enum Array { AX, AZ, ADH, AH, ADX, ADZ };
// Rows of any alignment: every P-th row (P = 16 bytes / a value) starts alike,
// so map i has the rows i, i + P, ... of a sequence (of all, where they follow
// one another), seen from the 16-byte boundary at or below row i.
struct Offs {
  TMap m[3][8];  // of x, z, dh
};
// What a launch needs beside the caller's arguments.
struct Plan {
  int segments, per;     // CTAs along time, pieces of each
  int same;              // bit per array (order of Array): laid out as x is, so that its rows start in 16 bytes where x's do
  int mapped, flat;      // bit per array: those that Offs describes; of them, those whose sequences follow one another
  ulonglong2* sums;      // [batch][segment][tile][32 channel pairs] (A, B), with several segments
  float* part;           // fp32 parts of dz: heads wider than pw, [batch][time][channels / pw]; SPREAD, [batch][time][tile][2]
  int pw;                // HEAD: channels whose dz one CTA sums (8, 16, 32 or 64)
};

template <typename T, int GATE, int OP, int LAY = SWZ>
struct Geo {
  // steps of a thread: what its registers hold of gates and partial results
  static constexpr int S = sizeof(T) == 2 ? (GATE == HEAD ? 11 : 9) : 6;
  static constexpr int L = 8 * S;                   // steps of a piece
  static constexpr int NB = sizeof(T) / 2;          // boxes of 128-byte rows across the tile
  static constexpr int BOX = L * 128;
  // rows that start anywhere: their pitch (72 values), the RB rows of a box and their place in a slot
  static constexpr int PITCH = 72 * sizeof(T);
  static constexpr int P = 16 / sizeof(T), RB = L / P, BOXP = (RB * PITCH + 127) / 128 * 128;
  static constexpr int SLOT = LAY == SWZ ? BOX * NB : P * BOXP;
  static __host__ __device__ constexpr int place(int row) { return row % P * BOXP + row / P * PITCH; }
  static constexpr int NH = GATE == OWN ? 0 : GATE == HEAD ? 1 : 4;  // heads of a warp's channels
  static constexpr bool Z = GATE == OWN, X = OP != SUM_BWD, D = OP == BWD || OP == SUM_BWD;
  // z's slot is there too where the backward keeps partial results in it
  static constexpr bool ZS = Z || (OP == BWD && sizeof(T) == 2);
  static constexpr int ARRAYS = Z + X + D, STAGE = (ZS + X + D) * SLOT;
  static constexpr int XO = ZS ? SLOT : 0, DO = XO + (X ? SLOT : 0);  // offsets of x and dh in a stage
  // stages: what two CTAs of an SM have room for (beside the gates' tables), at most 4: more
  // only keep more of DRAM's pages open at once (the 8 x 4096 x 2048 bf16 scan: 67 us with 4, 69 with 3, 75 with 6)
  static constexpr int FIT = (111 * 1024 - kWarps * L * NH * 8) / STAGE, NST = FIT > 4 ? 4 : FIT;
  static constexpr bool SUM = OP == SUM_FWD || OP == SUM_BWD;
  static_assert(BOX % 1024 == 0, "boxes start on the swizzle's period");
  // the computing warps write out rows that TMA does not, and sum dz of shared gates; of swizzled heads the TMA warp
  // does (8 x 4096 x 32 x 64 bf16: 120 us, 131 by the computing warps), for fp32 with another one to help it (5 x 1531 x
  // 25 x 48: 44 us, 50 alone; bf16 has more steps a piece and gains nothing)
  static constexpr bool SHARE = OP == BWD && (GATE == SPREAD || (GATE == HEAD && LAY != SWZ)), OUT = SHARE || (LAY != SWZ && !SUM);
  static constexpr bool TMASUM = OP == BWD && GATE == HEAD && LAY == SWZ, HELP = TMASUM && sizeof(T) == 4;
  static constexpr int THREADS = 32 * (kWarps + 1 + HELP);
  static constexpr int LATE = NST > 2 ? 1 : 0;  // rounds by which they do so later: a ring of two has none to spare
  static_assert(L % P == 0, "boxes of as many rows");
  static_assert(NST >= 2, "a ring");
};

constexpr f2 kOne2 = 0x3f8000003f800000ull, kNegOne2 = 0xbf800000bf800000ull;

// Gates: e = exp(-z), r = 1 / (1 + e), f = r, 1 - f = e r, each with its own
// relative accuracy: (8 + 1.2 |z|) 2^-24, f from z = -70 on (2^-101), 1 - f up to
// z = 87.  The exponent is cut off at 2^126, where r = 2^-126 is still a normal
// number; taking that off r makes z = -inf give f = 0, changes no r above 2^-101
// and is an absolute error of 2^-126 below.
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

template <typename T, int LAY> __device__ __forceinline__ f2 lds2(const char* p) {
  if constexpr (LAY == ELEM) {
    return pk(ld(reinterpret_cast<const T*>(p)), ld(reinterpret_cast<const T*>(p) + 1));
  } else if constexpr (sizeof(T) == 2) {
    const uint32_t v = *reinterpret_cast<const uint32_t*>(p);
    return pk(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
  } else {
    return *reinterpret_cast<const f2*>(p);
  }
}
template <typename T, int LAY> __device__ __forceinline__ void sts2(char* p, f2 v) {
  float a, b;
  upk(v, a, b);
  if constexpr (LAY == ELEM) {
    st(reinterpret_cast<T*>(p), a);
    st(reinterpret_cast<T*>(p) + 1, b);
  } else if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<__nv_bfloat162*>(p) = __floats2bfloat162_rn(a, b);
  } else {
    *reinterpret_cast<f2*>(p) = v;
  }
}
// an fp32 word where a pair lies (bf16 pairs of any alignment: in two halves)
template <typename T, int LAY> __device__ __forceinline__ float lds1(const char* p) {
  if constexpr (LAY == ELEM && sizeof(T) == 2) {
    const uint16_t* q = reinterpret_cast<const uint16_t*>(p);
    return __uint_as_float(q[0] | (uint32_t)q[1] << 16);
  } else {
    return *reinterpret_cast<const float*>(p);
  }
}
template <typename T, int LAY> __device__ __forceinline__ void sts1(char* p, float v) {
  if constexpr (LAY == ELEM && sizeof(T) == 2) {
    const uint32_t u = __float_as_uint(v);
    reinterpret_cast<uint16_t*>(p)[0] = (uint16_t)u;
    reinterpret_cast<uint16_t*>(p)[1] = (uint16_t)(u >> 16);
  } else {
    *reinterpret_cast<float*>(p) = v;
  }
}

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
template <int NST>
struct Bars {
  uint64_t full[NST], done[NST], out[NST];
  int abort_;
  int64_t first;  // of the sequence's channels in h0, h_last, dh_last and dh0
};

__device__ __forceinline__ int seq_len(const pnn_recur_args& a, int64_t b) {
  if (!a.lengths) return (int)a.time;
  const int64_t n = a.lengths[b];
  return (int)(n < 0 ? 0 : n > a.time ? a.time : n);
}
__device__ __forceinline__ f2 load_pair(const float* p, int c, int D) {
  return p ? pk(c < D ? p[c] : 0.f, c + 1 < D ? p[c + 1] : 0.f) : 0;
}
__device__ __forceinline__ void store_pair(float* p, int c, int D, f2 v) {
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

// Gates shared by channels of a warp: its lanes form them once a step (a
// head's lanes would otherwise form the same ones), into a table of the warp's
// own, NH a row.  Lanes l take head l mod NH of rows l / NH, l / NH + 32 / NH, ...
template <typename T, int L, int NH>
struct GateTable {
  static constexpr int BY = 32 / NH, N = (L + BY - 1) / BY;
  const T* p;             // this lane's first row of the next piece
  int64_t stride, piece;  // elements from row to row + BY, from piece to piece
  uint32_t z[N];          // the next piece's, as loaded: in time, not where the compiler would move it
  __device__ __forceinline__ void load(int left, int lane) {  // left: rows of that piece before the end
    const T* q = p;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      if (lane / NH + BY * i < (left < L ? left : L)) {
        if constexpr (sizeof(T) == 2) asm volatile("{\n\t.reg .u16 h;\n\tld.global.u16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(z[i]) : "l"(q));
        else asm volatile("ld.global.u32 %0, [%1];" : "=r"(z[i]) : "l"(q));
      }
      q += stride;
    }
    p += piece;
  }
  __device__ __forceinline__ void form(float2* table, int lane) const {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (lane / NH + BY * i < L) table[lane + 32 * i] = gate1(__uint_as_float(sizeof(T) == 2 ? z[i] << 16 : z[i]));
    __syncwarp();
  }
};

// ---------------------------------------------------------------- filling and emptying stages
// Rows of any alignment.  Row `row` of a piece lies at place(row), its first
// channel `shift` bytes further, where shift = (address of x's row) mod 16; a
// piece is a multiple of 16 bytes long in every row stride, so the shifts are
// those of any piece.
template <typename T, typename G>
struct Rows {
  int lane;
  int base, step, bytes;     // x's first address and row stride mod 16; bytes of a row in the tile
  __device__ __forceinline__ int shift(int row) const { return (base + row * step) & 15; }
  __device__ __forceinline__ Rows(int lane_, const T* x, int64_t stride, int c0, int D)
      : lane(lane_), base((int)(reinterpret_cast<uintptr_t>(x) & 15)), step((int)(stride * sizeof(T) & 15)),
        bytes((D - c0 < kTile ? D - c0 : kTile) * (int)sizeof(T)) {}
  // Arrays that no map describes or that are laid out in another way, value by
  // value: lane l takes values l and l + 32.
  __device__ __forceinline__ void fill_each(char* slot, const T* p, int64_t by, int rows) const {
    const int m = rows < G::L ? rows : G::L;
    const bool one = lane * (int)sizeof(T) < bytes, two = (lane + 32) * (int)sizeof(T) < bytes;
    const T* v = p;
#pragma unroll 1
    for (int h = 0; h < m; h += 8) {
      T va[8], vb[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (h + i < m && one) va[i] = v[lane];
        if (h + i < m && two) vb[i] = v[lane + 32];
        v += by;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (h + i < m) {
          const int row = h + i;
          T* w = reinterpret_cast<T*>(slot + G::place(row) + shift(row));
          if (one) w[lane] = va[i];
          if (two) w[lane + 32] = vb[i];
        }
    }
  }
};

// dz of `rows` rows of a piece, one gate for a head.  Each channel
// pair left the sum of its two shares where its dh was: the 4 lanes of a warp
// one swizzled 16-byte chunk (bf16), or two with every other word (fp32); in
// the other layouts pair by pair (shift(row): where the row starts).
template <typename T, int LAY, typename G, typename F>
__device__ __forceinline__ void sum_heads(const char* slot, const pnn_recur_args& a, const Plan& pl, int64_t b, int64_t t0,
                                          int row0, int rows, int c0, int D, int lane, F shift) {
  const int w8 = pl.pw / 8, sh = 31 - __clz(kTile / pl.pw);  // 64 / pw parts in a row
  for (int i = lane; i < rows << sh; i += 32) {
    const int row = row0 + (i >> sh), k = i & ((1 << sh) - 1);
    const int64_t t = t0 + row;
    const int c = c0 + k * pl.pw;
    if (c >= D) continue;
    float q = 0.f;
    if constexpr (LAY != SWZ) {
      const char* p = slot + G::place(row) + shift(row);
      for (int j = k * pl.pw / 2; j < (k + 1) * pl.pw / 2; ++j) q += lds1<T, LAY>(p + j * 2 * sizeof(T));
    } else {
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
    }
    if (pl.part) pl.part[(b * a.time + t) * (D / pl.pw) + c / pl.pw] = q;
    else st(static_cast<T*>(a.dz) + b * a.dz_stride_b + t * a.dz_stride_t + c / pl.pw, q);
  }
}

// The same for heads of any width: dz of every channel in fp32, bf16 pairs
// where z and dh were, fp32 where dh was.  A head that lies in the tile is
// summed here; one that goes on leaves its part of the row, at 1 in the tile
// where it begins and at 0 in the others.
template <typename T, int LAY, typename G, typename F>
__device__ __forceinline__ void sum_spread(const char* zslot, const char* dslot, const pnn_recur_args& a, const Plan& pl, int64_t b,
                                           int64_t t0, int row0, int rows, int tile, int tiles, int lane, F shift) {
  const int W = (int)a.width, D = (int)a.heads * W, c0 = tile * kTile, c1 = c0 + kTile < D ? c0 + kTile : D;
  const int k0 = c0 / W, n = (c1 - 1) / W - k0 + 1;
  const float by = 1.f / (float)n;
  for (int i = lane; i < rows * n; i += 32) {
    const int j = (int)(((float)i + 0.5f) * by), row = row0 + j, k = k0 + i - j * n;  // (i < 2048: exact)
    const int lo = k * W < c0 ? c0 : k * W, hi = k * W + W > c1 ? c1 : k * W + W;
    const int at = LAY == SWZ ? row * 128 : G::place(row) + shift(row);
    float q = 0.f;
#pragma unroll 4
    for (int c = lo - c0; c < hi - c0; ++c) {
      if constexpr (sizeof(T) == 2)
        q += lds1<T, LAY>((c & 1 ? dslot : zslot) + at + (LAY == SWZ ? ((c >> 3) ^ (row & 7)) << 4 | (c >> 1 & 3) << 2 : c >> 1 << 2));
      else
        q += lds1<T, LAY>(dslot + at + (LAY == SWZ ? (c >> 5) * G::BOX + (((c >> 2 & 7) ^ (row & 7)) << 4 | (c & 3) << 2) : c << 2));
    }
    const int64_t t = t0 + row;
    if (hi - lo == W) st(static_cast<T*>(a.dz) + b * a.dz_stride_b + t * a.dz_stride_t + k, q);
    else pl.part[((b * a.time + t) * tiles + tile) * 2 + (k * W >= c0)] = q;
  }
}

// ---------------------------------------------------------------- the kernel
template <typename T, int GATE, int LAY, int OP>
__global__ void __launch_bounds__(Geo<T, GATE, OP, LAY>::THREADS, 2)
    k_recur_tile(const __grid_constant__ std::conditional_t<LAY == SWZ, Maps, Offs> maps, const __grid_constant__ pnn_recur_args a, const __grid_constant__ Plan pl,
                 int* gave_up) {
  using G = Geo<T, GATE, OP, LAY>;
  constexpr bool TMA = LAY == SWZ;
  constexpr int S = G::S, L = G::L, NST = G::NST, SB = G::STAGE, XO = G::XO, DO = G::DO;
  constexpr bool UP = OP == FWD || OP == SUM_BWD;  // the pieces of a segment in increasing time
  if (G::SUM) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ char raw[];
  __shared__ Bars<NST> bars;
  __shared__ float2 table[GATE == OWN ? 1 : kWarps][GATE == OWN ? 1 : L * G::NH];
  char* ring = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(smem_u32(&bars.full[i]), TMA ? 1 : 2);
      mbar_init(smem_u32(&bars.done[i]), kWarps);
      mbar_init(smem_u32(&bars.out[i]), G::HELP ? 1 : kWarps);
    }
    bars.abort_ = 0;
    // A sequence's place among the states, in 64 bits, waits in shared memory for its two uses: in registers, or from its first
    // channel on in the backward, odd heads spill (8 x 4096 x 400 heads of 5 284 us instead of 268, 399 of them 567 instead of 511)
    bars.first = (int64_t)blockIdx.y * (a.heads * a.width);
    if (OP == BWD) bars.first += blockIdx.x % ((a.heads * a.width + kTile - 1) / kTile) * kTile;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int D = (int)(a.heads * a.width);
  const int tiles = (D + kTile - 1) / kTile, tile = blockIdx.x % tiles;
  const int seg = blockIdx.x / tiles + (OP == SUM_BWD ? 1 : 0);  // the outermost segment's sum is not needed
  const int b = blockIdx.y, n = seq_len(a, b);
  const int c0 = tile * kTile;
  const int cs = OP == BWD ? c0 : 0;
  const int pieces = (int)((a.time + L - 1) / L), p0 = seg * pl.per;
  const int rounds = p0 + pl.per < pieces ? pl.per : pieces - p0;
  const int64_t x_stride_b = OP == SUM_BWD ? a.dh_stride_b : a.x_stride_b, x_stride_t = OP == SUM_BWD ? a.dh_stride_t : a.x_stride_t;
  auto first_step = [&](int r) { return (UP ? p0 + r : p0 + rounds - 1 - r) * L; };  // below time, which fits an int
  auto first = [&] { return *static_cast<volatile int64_t*>(&bars.first); };
  auto wait = [&](uint64_t* bar, int r) {
    if (mbar_wait(smem_u32(bar), (r / NST) & 1, &bars.abort_)) return true;
    *reinterpret_cast<volatile int*>(&bars.abort_) = 1;
    count_give_up(gave_up);
    return false;
  };
  const Rows<T, G> rw(lane,
                      static_cast<const T*>(OP == SUM_BWD ? a.dh : a.x) + b * x_stride_b + c0, x_stride_t, c0, D);
  __syncthreads();

  constexpr int N = G::HELP ? L / 2 : L;  // rows of a warp that sums
  auto sum_rows = [&](int r, int row0) {
    const int t0 = first_step(r), left = (int)(a.time - t0 - row0), m = left < 0 ? 0 : left < N ? left : N;
    sum_heads<T, LAY, G>(ring + (r % NST) * SB + DO, a, pl, b, t0, row0, m, c0, D, lane, [](int) { return 0; });
    __syncwarp();
  };
  if constexpr (TMA) if (warp == kWarps) {
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
        const int x = c0 + i * 32;
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
          const int x = c0 + i * 32;
          if (OP == FWD) tma_store_3d(&maps.h, x, t0, b, at + XO);
          if (OP == BWD) tma_store_3d(&maps.dx, x, t0, b, at + XO);
          if (OP == BWD && GATE == OWN) tma_store_3d(&maps.dz, x, t0, b, at);
        }
        bulk_commit();
      }
      if constexpr (G::TMASUM) sum_rows(r, 0);
      if ((G::SHARE || G::HELP) && !wait(&bars.out[r % NST], r)) break;
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
  }
  if constexpr (G::HELP) if (warp == kWarps + 1) {
    for (int r = 0; r < rounds && wait(&bars.done[r % NST], r); ++r) {
      sum_rows(r, N);
      if (lane == 0) mbar_arrive(smem_u32(&bars.out[r % NST]));
    }
  }
  if constexpr (!TMA) if (warp == kWarps) {
    // -------------------------------------------------------------- one warp fills
    auto src = [&](const void* p, int64_t sb, int64_t st, int t0) { return static_cast<const T*>(p) + b * sb + t0 * st; };
    const int mapped = pl.same & pl.mapped & (G::X << AX | (GATE == OWN) << AZ | G::D << ADH);
    const bool issuer = lane == 0;
    auto box = [&](char* slot, int which, int t0, uint32_t bar) {
      if (!issuer) return;
      const bool flat = pl.flat >> which & 1;
      const int64_t row = flat ? b * a.time + t0 : t0;
#pragma unroll 1
      for (int i = 0; i < G::P; ++i)
        tma_load_3d(smem_u32(slot) + i * G::BOXP, &maps.m[which][(row + i) % G::P], c0, (int)((row + i) / G::P), flat ? 0 : b, bar);
    };
    auto fill = [&](char* slot, int which, const void* p, int64_t sb, int64_t st, int t0, int rows, uint32_t bar) {
      if (mapped >> which & 1) box(slot, which, t0, bar);
      else rw.fill_each(slot, src(p, sb, st, t0) + c0, st, rows);
    };
    int filled = 0;
    for (int r = 0; r < rounds; ++r) {
      char* at = ring + (r % NST) * SB;
      if (r >= NST && !wait(G::SUM ? &bars.done[r % NST] : &bars.out[r % NST], r - NST)) break;
      const int t0 = first_step(r);
      const int rows = n - t0 < L ? n - t0 : L;  // rows that are there (none behind the end)
      const uint32_t bar = smem_u32(&bars.full[r % NST]);
      if (issuer) mbar_expect_tx(bar, rows > 0 ? __popc(mapped) * (G::L * G::PITCH) : 0);
      if (rows > 0) {
        if (G::X) fill(at + XO, AX, a.x, a.x_stride_b, a.x_stride_t, t0, rows, bar);
        if (G::D) fill(at + DO, ADH, a.dh, a.dh_stride_b, a.dh_stride_t, t0, rows, bar);
        if (GATE == OWN) fill(at, AZ, a.z, a.z_stride_b, a.z_stride_t, t0, rows, bar);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(bar);
      filled = r + 1;
    }
    if (issuer)  // gave up: leave no copy in flight
      for (int q = filled > NST ? filled - NST : 0; q < filled; ++q) mbar_wait_drain(smem_u32(&bars.full[q % NST]), (q / NST) & 1);
  }
  if (warp < kWarps) {
    // -------------------------------------------------------------- eight warps compute
    const int grp = lane >> 2, pr = lane & 3, row0 = grp * S;
    const int c = c0 + warp * 8 + pr * 2;
    // this thread's pair in the rows of its run: the swizzle repeats every 8 rows
    int off[TMA ? 8 : S];
    if (TMA) {
      const int ch = sizeof(T) == 2 ? warp : 2 * (warp & 3) + (pr >> 1);
      const int in = sizeof(T) == 2 ? pr * 4 : (warp >> 2) * G::BOX + (pr & 1) * 8;
#pragma unroll
      for (int j = 0; j < 8; ++j) off[j < (TMA ? 8 : S) ? j : 0] = row0 * 128 + ((ch ^ ((row0 + j) & 7)) << 4) + in;
    } else {
      const T* x = static_cast<const T*>(OP == SUM_BWD ? a.dh : a.x) + b * x_stride_b + c0;
#pragma unroll
      for (int j = 0; j < S; ++j) {
        const int row = row0 + j;
        off[j < (TMA ? 8 : S) ? j : 0] = G::place(row) + (warp * 8 + pr * 2) * (int)sizeof(T) +
                                         (int)((reinterpret_cast<uintptr_t>(x) + row * (x_stride_t * sizeof(T))) & 15);
      }
    }
    auto pos = [&](int i) {
      if (!TMA && GATE == SPREAD)  // (found each time: kept, they would spill)
        return G::place(row0 + i) + rw.shift(row0 + i) + (warp * 8 + pr * 2) * (int)sizeof(T);
      return TMA ? off[i & 7] + i * 128 : off[i < (TMA ? 8 : S) ? i : 0];
    };
    // Rows that no tensor map describes go out (a round later) when all warps have written theirs: S rows a warp, by
    // words.  bf16 rows at odd places have single values at the ends, the first two lanes'.
    auto rows_out = [&](const char* slot, int which, void* out, int64_t sb, int64_t stride, int t0) {
      const int first = warp * S, m = a.time - t0 - first < S ? (int)(a.time - t0 - first) : S, valid = rw.bytes / (int)sizeof(T);
      if (m <= 0) return;
      T* p = static_cast<T*>(out) + b * sb + (t0 + first) * stride + c0;
      const uint32_t from = smem_u32(slot);
      if (!(pl.same >> which & 1)) {
        for (int j = 0; j < m; ++j, p += stride) {
          const T* q = reinterpret_cast<const T*>(slot + G::place(first + j) + rw.shift(first + j));
          if (lane < valid) p[lane] = q[lane];
          if (lane + 32 < valid) p[lane + 32] = q[lane + 32];
        }
        return;
      }
      uint32_t v[S], u[S];
#pragma unroll
      for (int j = 0; j < S; ++j) {
        const int row = first + (j < m ? j : 0), s = rw.shift(row);
        const uint32_t at = from + G::place(row) + s;
        asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v[j]) : "r"((at & ~3u) + 4 * lane));
        if constexpr (sizeof(T) == 4) {
          asm volatile("ld.shared.u32 %0, [%1];" : "=r"(u[j]) : "r"(at + 128 + 4 * lane));
        } else {
          if (lane < 2) asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(u[j]) : "r"(at + (lane ? 2 * valid - 2 : 0)));
        }
      }
#pragma unroll
      for (int j = 0; j < S; ++j) {
        if (j < m) {
          if constexpr (sizeof(T) == 4) {
            if (lane < valid) reinterpret_cast<uint32_t*>(p)[lane] = v[j];
            if (lane + 32 < valid) reinterpret_cast<uint32_t*>(p)[lane + 32] = u[j];
          } else {
            const int odd = LAY == ELEM ? rw.shift(first + j) >> 1 & 1 : 0, k = 2 * lane - odd;
            if (k >= 0 && k + 1 < valid) *reinterpret_cast<uint32_t*>(p + k) = v[j];
            if (odd | (valid & 1)) {
              if (lane == 0 && odd) *reinterpret_cast<uint16_t*>(p) = (uint16_t)u[j];
              if (lane == 1 && ((valid ^ odd) & 1) && valid > odd) *reinterpret_cast<uint16_t*>(p + valid - 1) = (uint16_t)u[j];
            }
          }
        }
        p += stride;
      }
    };
    auto stage_out = [&](int r) {
      if (!wait(&bars.done[r % NST], r)) return false;
      const int t0 = first_step(r);
      const char* at = ring + (r % NST) * SB;
      if constexpr (G::SHARE) {
        const int first = warp * S, left = (int)(a.time - t0 - first), m = left < 0 ? 0 : left < S ? left : S;
        const auto shift = [&](int row) { return TMA ? 0 : rw.shift(row); };
        if constexpr (GATE == HEAD) sum_heads<T, LAY, G>(at + DO, a, pl, b, t0, first, m, c0, D, lane, shift);
        else sum_spread<T, LAY, G>(at, at + DO, a, pl, b, t0, first, m, tile, tiles, lane, shift);
      }
      if constexpr (!TMA) {
        if (OP == FWD) rows_out(at + XO, AH, a.h, a.h_stride_b, a.h_stride_t, t0);
        if (OP == BWD) rows_out(at + XO, ADX, a.dx, a.dx_stride_b, a.dx_stride_t, t0);
        if (OP == BWD && GATE == OWN) rows_out(at, ADZ, a.dz, a.dz_stride_b, a.dz_stride_t, t0);
      }
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.out[r % NST]));
      return true;
    };
    constexpr int NH = GATE == OWN ? 1 : G::NH;
    GateTable<T, L, NH> gates;
    const int heads = (int)a.heads, W = (int)a.width;
    auto head_of = [&](int ch) { return ch < D ? ch / W : heads - 1; };
    const int head0 = GATE == OWN ? 0 : head_of(c0 + warp * 8);  // of the warp's first channel; of this thread's, from there:
    const int ka = GATE == SPREAD ? head_of(c) - head0 : 0, kb = GATE == SPREAD ? head_of(c + 1) - head0 : 0;
    if (GATE != OWN) {
      const int k = head0 + lane % NH;
      gates.p = static_cast<const T*>(a.z) + b * a.z_stride_b + (k < heads ? k : heads - 1) + (int64_t)(first_step(0) + lane / NH) * a.z_stride_t;
      gates.stride = gates.BY * a.z_stride_t;
      gates.piece = (UP ? L : -L) * a.z_stride_t;
      gates.load(n - first_step(0), lane);
    }
    // the value carried along the pieces: the state, or R; composed over the segments before
    ulonglong2* sums = pl.sums + ((int64_t)b * pl.segments * tiles + tile) * 32 + warp * 4 + pr;
    f2 s = 0, tot = kOne2;  // SUM: (tot, s) of the pieces so far
    if (!G::SUM && pl.segments > 1) asm volatile("griddepcontrol.wait;" ::: "memory");  // the sums are there
    if (OP == FWD) {
      s = a.h0 ? load_pair(a.h0 + first(), c - cs, D - cs) : 0;
      for (int q = 0; q < seg; ++q) {
        const ulonglong2 v = sums[(int64_t)q * tiles * 32];
        s = fma2(v.x, s, v.y);
      }
    }
    if (OP == BWD) {
      s = a.dh_last ? load_pair(a.dh_last + first(), c - cs, D - cs) : 0;
      for (int q = pl.segments - 1; q > seg; --q) {
        const ulonglong2 v = sums[(int64_t)q * tiles * 32];
        s = fma2(v.x, s, v.y);
      }
    }
    float* saved = a.saved + ((int64_t)b * pieces + (UP ? p0 : p0 + rounds - 1)) * D;  // the piece's first state
    f2 before = OP == BWD && first_step(0) < n ? load_pair(saved, c, D) : 0;
    bool ok = true;
    for (int r = 0; ok && r < rounds; ++r) {
      char* at = ring + (r % NST) * SB;
      const int t0 = first_step(r);
      ok = wait(&bars.full[r % NST], r);
      if (!ok) break;
      if (GATE != OWN) {
        gates.form(table[GATE == OWN ? 0 : warp], lane);
        if (TMA && r + 1 < rounds) gates.load(n - first_step(r + 1), lane);
      }
      const int left = t0 < n ? n - t0 - row0 : 0;
      // EDGE: the piece reaches behind the end, where steps keep the state
      auto piece = [&](auto edge) {
        constexpr bool EDGE = decltype(edge)::value;
        auto gate_at = [&](int i, f2& f, f2& g) {
          if constexpr (GATE == HEAD) {
            const float2 q = table[warp][row0 + i];
            f = pk(q.x, q.x);
            g = pk(q.y, q.y);
          } else if constexpr (GATE == SPREAD) {
            const float2 q = table[warp][(row0 + i) * NH + ka], u = table[warp][(row0 + i) * NH + kb];
            f = pk(q.x, u.x);
            g = pk(q.y, u.y);
          } else {
            gate2(lds2<T, LAY>(at + pos(i)), f, g);
          }
          if (EDGE && i >= left) {
            f = kOne2;
            g = 0;
          }
        };
        auto x_at = [&](int i) {
          const f2 x = lds2<T, LAY>(at + XO + pos(i));
          return EDGE && i >= left ? 0 : x;
        };
        auto d_at = [&](int i) {
          const f2 d = lds2<T, LAY>(at + DO + pos(i));
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
          for (int i = 0; i < S; ++i) sts2<T, LAY>(at + XO + pos(i), EDGE && i >= left ? 0 : fma2(A_at(i), h, B[i]));
        } else {
          // what a thread keeps for its second walk: the gates (a shared one is read again from the table), and
          // h_{t-1} - x_t (bf16: as two fp32 words where z and x were)
          constexpr bool KEEP = GATE != SPREAD, SPILL = sizeof(T) == 2;
          [[maybe_unused]] std::conditional_t<GATE == HEAD, float, f2> f[KEEP ? S : 1] = {}, g[KEEP ? S : 1] = {};
          [[maybe_unused]] f2 q[SPILL ? 1 : S] = {};
          f2 A = kOne2, Bf = 0, Bb = 0;
          auto gate_kept = [&](int i, f2& fi, f2& gi) {
            if constexpr (GATE == HEAD) fi = pk(f[i], f[i]), gi = pk(g[i], g[i]);
            else if constexpr (KEEP) fi = f[i], gi = g[i];
            else gate_at(i, fi, gi);
          };
#pragma unroll
          for (int i = 0; i < S; ++i) {
            f2 fi, gi;
            gate_at(i, fi, gi);
            if constexpr (GATE == HEAD) f[i] = __uint_as_float((uint32_t)fi), g[i] = __uint_as_float((uint32_t)gi);
            else if constexpr (KEEP) f[i] = fi, g[i] = gi;
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
              sts1<T, LAY>(at + pos(i), lo);
              sts1<T, LAY>(at + XO + pos(i), hi);
            } else {
              q[i] = d;
            }
            h = fma2(fi, h, mul2(gi, x));
          }
#pragma unroll
          for (int i = S - 1; i >= 0; --i) {
            f2 fi, gi, d;
            gate_kept(i, fi, gi);
            if constexpr (SPILL) d = pk(lds1<T, LAY>(at + pos(i)), lds1<T, LAY>(at + XO + pos(i)));
            else d = q[i];
            const f2 Gt = add2(d_at(i), w);
            w = mul2(fi, Gt);
            f2 dx = mul2(gi, Gt), dz = mul2(mul2(gi, w), d);
            if (EDGE && i >= left) dx = dz = 0;
            sts2<T, LAY>(at + XO + pos(i), dx);
            float lo, hi;
            upk(dz, lo, hi);
            if constexpr (GATE == HEAD) {
              sts1<T, LAY>(at + DO + pos(i), lo + hi);
            } else if constexpr (GATE == SPREAD && sizeof(T) == 2) {
              sts1<T, LAY>(at + pos(i), lo);
              sts1<T, LAY>(at + DO + pos(i), hi);
            } else {
              sts2<T, LAY>(at + (GATE == SPREAD ? DO : 0) + pos(i), dz);
            }
          }
        }
      };
      if (n - t0 < L) piece(std::true_type());
      else piece(std::false_type());
      if (!G::SUM) fence_proxy_async();
      __syncwarp();
      if (lane == 0) mbar_arrive(smem_u32(&bars.done[r % NST]));
      if constexpr (G::OUT) {
        if (r >= G::LATE) ok = stage_out(r - G::LATE);
      }
      // (where registers are short the next gates are loaded last: earlier they would be spilled, each after its whole
      // latency; 8 x 4096 x 399 x 5 took 402 and 625 us so)
      if (!TMA && GATE != OWN && r + 1 < rounds) gates.load(n - first_step(r + 1), lane);
    }
    if constexpr (G::OUT && G::LATE) {
      if (ok && rounds > 0) ok = stage_out(rounds - 1);
    }
    if (ok && grp == 0) {
      if (G::SUM) sums[(int64_t)seg * tiles * 32] = make_ulonglong2(tot, s);
      if (OP == FWD && a.h_last && seg == pl.segments - 1) store_pair(a.h_last + first(), c - cs, D - cs, s);
      if (OP == BWD && a.dh0 && seg == 0) store_pair(a.dh0 + first(), c - cs, D - cs, s);
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
  return encode_tensor_map_3d(&m, p, sizeof(T) == 2, D, a.time, a.batch, st, sb, 128 / (int)sizeof(T), L, true, &why) == 0;
}

// Rows of any alignment: the P maps of an array whose sequences follow one
// another (flat) or lie multiples of 16 bytes apart.
template <typename T>
bool offs_ok(int64_t sb, int64_t st, const pnn_recur_args& a, bool& flat) {
  constexpr int64_t P = 16 / sizeof(T);
  flat = a.batch == 1 || sb == a.time * st;
  const int64_t rows = flat ? a.batch * a.time : a.time;
  return rows >= P && rows / P < (1LL << 31) - 128 && st >= a.heads * a.width && st < (1LL << 35) &&
         (flat || (sb > 0 && sb % P == 0 && sb < (1LL << 37)));
}
template <typename T>
bool encode_offs(TMap* m, const void* p, int64_t sb, int64_t st, bool flat, int box_rows, const pnn_recur_args& a) {
  const char* why = nullptr;
  constexpr int64_t P = 16 / sizeof(T);
  const int64_t rows = flat ? a.batch * a.time : a.time, D = a.heads * a.width;
  for (int64_t i = 0; i < P; ++i) {
    const uintptr_t at = reinterpret_cast<uintptr_t>(static_cast<const T*>(p) + i * st);
    if (encode_tensor_map_3d(&m[i], reinterpret_cast<const void*>(at & ~(uintptr_t)15), sizeof(T) == 2, (int64_t)(at & 15) / (int64_t)sizeof(T) + D,
                             (rows - i + P - 1) / P, flat ? 1 : a.batch, P * st, flat ? P * st : sb, 72, box_rows, false, &why))
      return false;
  }
  return true;
}

template <typename T, int GATE, int LAY, int OP, typename M>
cudaError_t launch_one(const M& m, const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st) {
  constexpr int smem = Geo<T, GATE, OP, LAY>::NST * Geo<T, GATE, OP, LAY>::STAGE + 1024;
  const auto kernel = k_recur_tile<T, GATE, LAY, OP>;
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
  // the launch after the sums begins beside them: it fills its stages, and waits before it reads the sums
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(tiles * segs), (unsigned)a.batch);
  cfg.blockDim = dim3(Geo<T, GATE, OP, LAY>::THREADS);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = pl.segments > 1 && segs == pl.segments ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, m, a, pl, gave_up);
}

template <typename T, int GATE, int LAY, bool BACK, typename M>
cudaError_t run(const M& m, const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st) {
  cudaError_t e = cudaSuccess;
  if (pl.segments > 1)
    e = launch_one<T, GATE, LAY, BACK ? SUM_BWD : SUM_FWD>(m, a, pl, gave_up, st);
  if (e != cudaSuccess) return e;
  return launch_one<T, GATE, LAY, BACK ? BWD : FWD>(m, a, pl, gave_up, st);
}

// Which form takes these arguments, and its launches.
template <typename T, bool BACK>
cudaError_t dispatch(const pnn_recur_args& a, Plan pl, int* gave_up, cudaStream_t st) {
  const int gate = a.width == 1 ? OWN : a.width % 8 == 0 ? HEAD : SPREAD;
  constexpr int64_t e = sizeof(T);
  struct { const void* p; int64_t sb, st; TMap Maps::*map; bool used; } const all[6] = {
      {a.x, a.x_stride_b, a.x_stride_t, &Maps::x, true},
      {a.z, a.z_stride_b, a.z_stride_t, &Maps::z, gate == OWN},
      {a.dh, a.dh_stride_b, a.dh_stride_t, &Maps::dh, BACK},
      {a.h, a.h_stride_b, a.h_stride_t, &Maps::h, !BACK},
      {a.dx, a.dx_stride_b, a.dx_stride_t, &Maps::dx, BACK},
      {a.dz, a.dz_stride_b, a.dz_stride_t, &Maps::dz, BACK && gate == OWN}};
  bool tma = true, two = true;
  pl.same = 0;
  for (int i = 0; i < 6; ++i) {
    if (!all[i].used) continue;
    tma = tma && map_ok(all[i].p, all[i].sb, all[i].st, a, e);
    // rows that start in 16 bytes where x's do
    const uintptr_t d = reinterpret_cast<uintptr_t>(all[i].p) - reinterpret_cast<uintptr_t>(a.x);
    if (d % 16 == 0 && all[i].st == a.x_stride_t && (all[i].sb - a.x_stride_b) * e % 16 == 0)
      pl.same |= 1 << i;
    // the sums of the backward read dh alone: it sets the layout there
    if (i == AX || i == ADH) two = two && reinterpret_cast<uintptr_t>(all[i].p) % (2 * e) == 0 && all[i].st % 2 == 0 && all[i].sb % 2 == 0;
  }
  if (BACK && !(pl.same >> ADH & 1)) {
    two = false;
    pl.same &= ~(1 << AZ);
  }
  Maps m;
  if (tma) {
    const auto enc = gate == HEAD ? encode<T, Geo<T, HEAD, FWD>::L> : encode<T, Geo<T, OWN, FWD>::L>;
    for (int i = 0; i < 6; ++i)
      if (all[i].used && !enc(m.*all[i].map, all[i].p, all[i].sb, all[i].st, a)) return cudaErrorInvalidValue;
    return gate == OWN    ? run<T, OWN, SWZ, BACK>(m, a, pl, gave_up, st)
           : gate == HEAD ? run<T, HEAD, SWZ, BACK>(m, a, pl, gave_up, st)
                          : run<T, SPREAD, SWZ, BACK>(m, a, pl, gave_up, st);
  }
  Offs o;
  pl.mapped = pl.flat = 0;
  const int box = gate == HEAD ? Geo<T, HEAD, FWD>::RB : Geo<T, OWN, FWD>::RB;
  for (int i : {AX, AZ, ADH}) {
    bool flat;
    if (all[i].used && offs_ok<T>(all[i].sb, all[i].st, a, flat)) {
      if (!encode_offs<T>(o.m[i], all[i].p, all[i].sb, all[i].st, flat, box, a)) return cudaErrorInvalidValue;
      pl.flat |= flat << i;
      pl.mapped |= 1 << i;
    }
  }
  if (gate == HEAD) return run<T, HEAD, ELEM, BACK>(o, a, pl, gave_up, st);
  if (gate == SPREAD) return run<T, SPREAD, ELEM, BACK>(o, a, pl, gave_up, st);
  return two ? run<T, OWN, PAIR, BACK>(o, a, pl, gave_up, st) : run<T, OWN, ELEM, BACK>(o, a, pl, gave_up, st);
}

cudaError_t run_fwd_bf16(const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st);
cudaError_t run_fwd_f32(const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st);
cudaError_t run_bwd_bf16(const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st);
cudaError_t run_bwd_f32(const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st);

}  // namespace recur
}  // namespace pnn
