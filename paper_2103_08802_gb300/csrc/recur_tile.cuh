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
// that copy the 16-byte chunks a row of 64 channels touches, wherever it
// starts in the first one.
//
// With too few (sequence, channel tile) pairs to fill the GPU the pieces of a
// pair are split into segments, one CTA each: a first launch forms every
// segment's (A, B) (it reads z and x, or z and dh, and keeps nothing), the
// second composes those before its own and proceeds as above.  The first
// launch walks away from the end at which the second begins, which then finds
// the latest 100 MB or so in L2.
//
// Bank conflicts: for a step i the 8 groups read rows g S + i of one 16-byte
// (bf16) or 32-byte (fp32) column.  TMA's 128-byte swizzle moves a row's
// 16-byte chunks by row mod 8; S odd (bf16) makes those eight distinct, S = 2
// mod 4 (fp32, half a warp at a time) the four pairs of chunks.  Rows copied in
// chunks lie 144 (bf16) or 272 bytes apart, which does the same.
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

// SWZ: rows as TMA swizzles them.  PAIR, ELEM: rows as their chunks lie in
// memory, channel pairs on whole (PAIR) or any (ELEM) words.
enum Layout { SWZ, PAIR, ELEM };

constexpr int kWarps = 8, kTile = 64, kLoaders = 2;

struct alignas(64) TMap {
  uint8_t b[128];
};
struct Maps {
  TMap z, x, dh, h, dz, dx;
};
enum Array { AX, AZ, ADH, AH, ADX, ADZ };
// What a launch needs beside the caller's arguments.
struct Plan {
  int segments, per;     // CTAs along time, pieces of each
  int same;              // bit per array (order of Array): laid out as x is, so that its rows start in their chunks where x's do
  ulonglong2* sums;      // [batch][segment][tile][32 channel pairs] (A, B), with several segments
  float* part;           // heads wider than pw: fp32 parts of dz, [batch][time][channels / pw]
  int pw;                // channels whose dz one CTA sums (HEAD: 8, 16, 32 or 64; SPREAD: 1)
};

template <typename T, int GATE, int OP, int LAY = SWZ>
struct Geo {
  // steps of a thread: what its registers hold of gates and partial results
  static constexpr int S = sizeof(T) == 2 ? (GATE == HEAD ? 11 : 9) : 6;
  static constexpr int L = 8 * S;                   // steps of a piece
  static constexpr int NB = sizeof(T) / 2;          // boxes of 128-byte rows across the tile
  static constexpr int BOX = L * 128;
  static constexpr int CHUNKS = kTile * sizeof(T) / 16 + 1, PITCH = CHUNKS * 16;  // of a row that starts anywhere
  static constexpr int SLOT = LAY == SWZ ? BOX * NB : (L * PITCH + 127) / 128 * 128;
  static constexpr bool Z = GATE != HEAD, X = OP != SUM_BWD, D = OP == BWD || OP == SUM_BWD;
  // z's slot is there too where the backward keeps partial results in it
  static constexpr bool ZS = Z || (OP == BWD && sizeof(T) == 2);
  static constexpr int ARRAYS = Z + X + D, STAGE = (ZS + X + D) * SLOT;
  static constexpr int XO = ZS ? SLOT : 0, DO = XO + (X ? SLOT : 0);  // offsets of x and dh in a stage
  // stages: what two CTAs of an SM have room for (beside the gates' tables and the chunks'), at most 4: more
  // only keep more of DRAM's pages open at once (the 8 x 4096 x 2048 bf16 scan: 67 us with 4, 69 with 3, 75 with 6)
  // the chunk table, in whole batches of the loaders
  static constexpr int PER = 32 * kLoaders * 4, TABLE_ROWS = (L * CHUNKS + PER - 1) / PER * PER;
  static constexpr int TABLE = LAY == SWZ ? 0 : TABLE_ROWS * 8;
  static constexpr int FIT = (111 * 1024 - (GATE == HEAD ? kWarps * L * 8 : 0) - TABLE) / STAGE, NST = FIT > 4 ? 4 : FIT;
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
// 16 bytes, of which the first n are read and the rest zeroed; none if n is 0
__device__ __forceinline__ void cp_async16_if(uint32_t dst, const void* src, int n) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.s32 p, %2, 0;\n\t@p cp.async.cg.shared.global [%0], [%1], 16, %2;\n\t}" ::"r"(dst),
               "l"(src), "r"(n)
               : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>  // all but this thread's latest N groups have landed
__device__ __forceinline__ void cp_async_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

template <int NST>
struct Bars {
  uint64_t full[NST], done[NST], emptied;
  int abort_;
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
// The chunk layout.  Row `row` of a piece lies at row * PITCH, its first channel
// `shift` bytes further, where shift = (address of x's row) mod 16; a piece is
// a multiple of 16 bytes long in every row stride, so the shifts are those of
// any piece.  A chunk: where from the piece's first value; and packed, its
// place in the slot (16 bits), end and begin of the row's bytes in it (5, 4),
// row (7).
struct Chunk {
  int from;
  uint32_t what;
};
// Shared memory answers a loader warp only after the computing warps' queued
// accesses (about 100 cycles each way), so its loops have a batch under way.
constexpr int kBatch = 4;
template <int ROWS>
__device__ __forceinline__ void fill_chunks(uint32_t table, uint32_t slot, const char* p, int rows) {
#pragma unroll 1
  for (int h = 0; h < ROWS; h += kBatch * 32 * kLoaders, table += kBatch * 32 * kLoaders * 8) {
    int from[kBatch];
    uint32_t what[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(from[i]), "=r"(what[i]) : "r"(table + i * 32 * kLoaders * 8));
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      cp_async16_if(slot + (what[i] & 0xffff), p + from[i], (int)(what[i] >> 25) < rows ? (int)(what[i] >> 16 & 31) : 0);
  }
}
template <int ROWS>
__device__ __forceinline__ void empty_chunks(uint32_t table, uint32_t slot, char* p, int rows) {
#pragma unroll 1
  for (int h = 0; h < ROWS; h += kBatch * 32 * kLoaders, table += kBatch * 32 * kLoaders * 8) {
    int from[kBatch];
    uint32_t what[kBatch];
    uint4 v[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(from[i]), "=r"(what[i]) : "r"(table + i * 32 * kLoaders * 8));
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(v[i].x), "=r"(v[i].y), "=r"(v[i].z), "=r"(v[i].w)
                   : "r"(slot + (what[i] & 0xffff)));
#pragma unroll
    for (int i = 0; i < kBatch; ++i)
      if ((what[i] >> 16 & 511) == 16 && (int)(what[i] >> 25) < rows) *reinterpret_cast<uint4*>(p + from[i]) = v[i];
  }
}
// The chunks that rows share with their neighbours, value by value: 16 /
// sizeof(T) lanes for a row's first, as many for its last, without branches (a
// lane's share differs from row to row).
template <typename T, int PITCH>
__device__ __forceinline__ void empty_edges(uint32_t slot, char* p, int64_t stride, int base, int step, int bytes, int rows, int lane) {
  constexpr int E = 16 / sizeof(T), PER = 16 / E, N = 6;
  const int in = (lane & (E - 1)) * (int)sizeof(T), sub = lane / (2 * E);
  const bool last = lane & E;
  p += sub * stride + in;
  slot += sub * PITCH + in;
  base += sub * step;
#pragma unroll 1
  for (int r = sub; r < rows; r += N * PER) {
    uint32_t v[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int s = (base + i * PER * step) & 15, at = last ? (bytes + s) & ~15 : 0;
      const uint32_t from = slot + (r + i * PER < rows ? i * PER * PITCH : 0) + at;
      if (sizeof(T) == 2) asm volatile("{\n\t.reg .u16 h;\n\tld.shared.u16 h, [%1];\n\tcvt.u32.u16 %0, h;\n\t}" : "=r"(v[i]) : "r"(from));
      else asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v[i]) : "r"(from));
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int s = base & 15, total = bytes + s;
      const int at = last ? total & ~15 : 0, lo = last ? at : s, hi = last ? total : total < 16 ? total : 16;
      const int some = (last ? (int)(total > 16) : (int)(s > 0) | (int)(total < 16)) & (int)(r + i * PER < rows);
      if (some & (int)(at + in >= lo) & (int)(at + in < hi)) {
        if (sizeof(T) == 2) *reinterpret_cast<uint16_t*>(p - s + at) = (uint16_t)v[i];
        else *reinterpret_cast<uint32_t*>(p - s + at) = v[i];
      }
      p += PER * stride;
      base += PER * step;
    }
    slot += N * PER * PITCH;
  }
}
template <typename T, typename G>
struct Rows {
  static constexpr int L = G::L, PITCH = G::PITCH, CHUNKS = G::CHUNKS, R = L / kLoaders;
  const Chunk* chunks;
  int row0, lane, first;     // value by value: half of the rows a warp; chunks: every other 32
  int base, step, bytes;     // x's first address and row stride mod 16; bytes of a row in the tile
  int64_t stride;            // of x, in bytes
  __device__ __forceinline__ int shift(int row) const { return (base + row * step) & 15; }
  __device__ __forceinline__ Rows(const Chunk* chunks_, int loader, int lane_, const T* x, int64_t stride_, int c0, int D)
      : chunks(chunks_), row0(loader * R), lane(lane_), first(loader * 32 + lane_),
        base((int)(reinterpret_cast<uintptr_t>(x) & 15)), step((int)(stride_ * sizeof(T) & 15)),
        bytes((D - c0 < kTile ? D - c0 : kTile) * (int)sizeof(T)), stride(stride_ * sizeof(T)) {}
  // the table, by all threads of the CTA
  __device__ __forceinline__ void describe(Chunk* to) const {
    for (int i = threadIdx.x; i < G::TABLE_ROWS; i += blockDim.x) {
      const int row = i / CHUNKS, ch = i % CHUNKS, s = shift(row), begin = ch ? 0 : s;
      int end = bytes + s - ch * 16;
      end = end > 16 ? 16 : end;
      if (end <= begin) end = 0;
      // (what fills up the last batch: no bytes, at the slot's beginning)
      to[i] = row < L ? Chunk{(int)(row * stride) - s + ch * 16, (uint32_t)(row * PITCH + ch * 16) | (uint32_t)end << 16 |
                                                                     (uint32_t)begin << 21 | (uint32_t)row << 25}
                      : Chunk{0, 127u << 25};
    }
  }
  // p: the piece's first value in this tile.  Arrays laid out as x is, chunk by
  // chunk (a chunk's bytes outside the row are read only where they share its
  // 16 bytes, and used by nobody).
  __device__ __forceinline__ void fill(char* slot, const T* p, int rows) const {
    fill_chunks<G::TABLE_ROWS>(smem_u32(chunks + first), smem_u32(slot), reinterpret_cast<const char*>(p), rows < L ? rows : 128);
  }
  __device__ __forceinline__ void empty(const char* slot, T* p, int rows) const {
    const int m = rows - row0 < R ? rows - row0 : R;
    empty_chunks<G::TABLE_ROWS>(smem_u32(chunks + first), smem_u32(slot), reinterpret_cast<char*>(p), rows < L ? rows : 128);
    empty_edges<T, PITCH>(smem_u32(slot) + row0 * PITCH, reinterpret_cast<char*>(p) + row0 * stride, stride, base + row0 * step, step,
                          bytes, m, lane);
  }
  // Arrays laid out in another way, value by value: lane l takes values l and
  // l + 32, read at a and b (the channels themselves, or their heads).
  __device__ __forceinline__ void fill_each(char* slot, const T* p, int64_t by, int rows, int a, int b) const {
    const int m = rows - row0 < R ? rows - row0 : R;
    const bool one = lane * (int)sizeof(T) < bytes, two = (lane + 32) * (int)sizeof(T) < bytes;
    const T* v = p + row0 * by;
#pragma unroll 1
    for (int h = 0; h < m; h += 8) {
      T va[8], vb[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (h + i < m && one) va[i] = v[a];
        if (h + i < m && two) vb[i] = v[b];
        v += by;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i)
        if (h + i < m) {
          const int row = row0 + h + i;
          T* w = reinterpret_cast<T*>(slot + row * PITCH + shift(row));
          if (one) w[lane] = va[i];
          if (two) w[lane + 32] = vb[i];
        }
    }
  }
  __device__ __forceinline__ void empty_each(const char* slot, T* p, int64_t by, int rows) const {
    const int m = rows - row0 < R ? rows - row0 : R;
    const bool one = lane * (int)sizeof(T) < bytes, two = (lane + 32) * (int)sizeof(T) < bytes;
    for (int i = 0; i < m; ++i) {
      const int row = row0 + i;
      const T* w = reinterpret_cast<const T*>(slot + row * PITCH + shift(row));
      if (one) p[row * by + lane] = w[lane];
      if (two) p[row * by + lane + 32] = w[lane + 32];
    }
  }
  // dz of every channel in fp32 (heads of any width; p: the piece's first row
  // and the tile's first channel, D channels a row): bf16 pairs left theirs
  // where z and dh were, fp32 ones where z was
  template <int LAY>
  __device__ __forceinline__ void empty_spread(const char* zslot, const char* dslot, float* p, int D, int rows) const {
    const int m = rows - row0 < R ? rows - row0 : R;
    for (int i = 0; i < m; ++i) {
      const int row = row0 + i, at = row * PITCH + shift(row);
      const int one = sizeof(T) == 2 ? 2 * lane : lane, two = one + (sizeof(T) == 2 ? 1 : 32);
      if (one * (int)sizeof(T) < bytes) p[(int64_t)row * D + one] = lds1<T, LAY>(zslot + at + 4 * lane);
      if (two * (int)sizeof(T) < bytes) p[(int64_t)row * D + two] = lds1<T, LAY>((sizeof(T) == 2 ? dslot + at : zslot + at + 128) + 4 * lane);
    }
  }
};

// dz of the rows row0 .. row1 of a piece, one gate for a head.  Each channel
// pair left the sum of its two shares where its dh was: the 4 lanes of a warp
// one swizzled 16-byte chunk (bf16), or two with every other word (fp32); in
// the chunk layout pair by pair (shift(row): where the row starts).
template <typename T, int LAY, typename G, typename F>
__device__ __forceinline__ void sum_heads(const char* slot, const pnn_recur_args& a, const Plan& pl, int64_t b, int64_t t0,
                                          int row0, int row1, int c0, int D, int lane, F shift) {
  const int w8 = pl.pw / 8, sh = 31 - __clz(kTile / pl.pw);  // 64 / pw parts in a row
  for (int i = lane; i < (row1 - row0) << sh; i += 32) {
    const int row = row0 + (i >> sh), k = i & ((1 << sh) - 1);
    const int64_t t = t0 + row;
    const int c = c0 + k * pl.pw;
    if (t >= a.time || c >= D) continue;
    float q = 0.f;
    if constexpr (LAY != SWZ) {
      const char* p = slot + row * G::PITCH + shift(row);
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

// ---------------------------------------------------------------- the kernel
template <typename T, int GATE, int LAY, int OP>
__global__ void __launch_bounds__(32 * (kWarps + (LAY == SWZ ? 1 : kLoaders)), 2)
    k_recur_tile(const __grid_constant__ Maps maps, const __grid_constant__ pnn_recur_args a, const __grid_constant__ Plan pl,
                 int* gave_up) {
  using G = Geo<T, GATE, OP, LAY>;
  constexpr bool TMA = LAY == SWZ;
  constexpr int S = G::S, L = G::L, NST = G::NST, SB = G::STAGE, XO = G::XO, DO = G::DO;
  constexpr bool UP = OP == FWD || OP == SUM_BWD;  // the pieces of a segment in increasing time
  if (G::SUM) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ char raw[];
  __shared__ Bars<NST> bars;
  __shared__ float2 table[GATE == HEAD ? kWarps : 1][GATE == HEAD ? L : 1];
  __shared__ Chunk chunks[TMA ? 1 : G::TABLE_ROWS];
  char* ring = raw + ((1024 - (smem_u32(raw) & 1023)) & 1023);
  if (threadIdx.x == 0) {
    for (int i = 0; i < NST; ++i) {
      mbar_init(smem_u32(&bars.full[i]), TMA ? 1 : kLoaders);
      mbar_init(smem_u32(&bars.done[i]), kWarps);
    }
    mbar_init(smem_u32(&bars.emptied), kLoaders);
    bars.abort_ = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int D = (int)(a.heads * a.width);
  const int tiles = (D + kTile - 1) / kTile, tile = blockIdx.x % tiles;
  const int seg = blockIdx.x / tiles + (OP == SUM_BWD ? 1 : 0);  // the outermost segment's sum is not needed
  const int b = blockIdx.y, n = seq_len(a, b);
  const int c0 = tile * kTile;
  const int pieces = (int)((a.time + L - 1) / L), p0 = seg * pl.per;
  const int rounds = p0 + pl.per < pieces ? pl.per : pieces - p0;
  const int64_t x_stride_b = OP == SUM_BWD ? a.dh_stride_b : a.x_stride_b, x_stride_t = OP == SUM_BWD ? a.dh_stride_t : a.x_stride_t;
  auto first_step = [&](int r) { return (UP ? p0 + r : p0 + rounds - 1 - r) * L; };  // below time, which fits an int
  auto wait = [&](uint64_t* bar, int r) {
    if (mbar_wait(smem_u32(bar), (r / NST) & 1, &bars.abort_)) return true;
    *reinterpret_cast<volatile int*>(&bars.abort_) = 1;
    *reinterpret_cast<volatile int*>(gave_up) = 1;
    return false;
  };
  const Rows<T, G> rw(chunks, warp - kWarps, lane,
                      static_cast<const T*>(OP == SUM_BWD ? a.dh : a.x) + b * x_stride_b + c0, x_stride_t, c0, D);
  if (!TMA) rw.describe(chunks);
  __syncthreads();

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
      if (OP == BWD && GATE == HEAD) {
        sum_heads<T, LAY, G>(ring + (r % NST) * SB + DO, a, pl, b, t0, 0, L, c0, D, lane, [](int) { return 0; });
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
    // -------------------------------------------------------------- two warps fill and empty
    static_assert(L % kLoaders == 0, "rows of a loader");
    auto src = [&](const void* p, int64_t sb, int64_t st, int t0) { return static_cast<const T*>(p) + b * sb + t0 * st; };
    auto dst = [&](void* p, int64_t sb, int64_t st, int t0) { return static_cast<T*>(p) + b * sb + t0 * st + c0; };
    const int ha = (c0 + lane) / (int)a.width, hb = (c0 + lane + 32) / (int)a.width;  // SPREAD: heads of lane's channels
    auto fill = [&](char* slot, int which, const void* p, int64_t sb, int64_t st, int t0, int rows) {
      if (pl.same >> which & 1) rw.fill(slot, src(p, sb, st, t0) + c0, rows);
      else rw.fill_each(slot, src(p, sb, st, t0) + c0, st, rows, lane, lane + 32);
    };
    auto empty = [&](const char* slot, int which, void* p, int64_t sb, int64_t st, int t0, int rows) {
      if (pl.same >> which & 1) rw.empty(slot, dst(p, sb, st, t0), rows);
      else rw.empty_each(slot, dst(p, sb, st, t0), st, rows);
    };
    // a stage is handed over when the K stages after it are under way
    constexpr int K = NST > 2 ? NST - 2 : 0;
    for (int r = 0; r < rounds + NST; ++r) {
      char* at = ring + (r % NST) * SB;
      if (r >= NST) {
        const int q = r - NST;
        if (q >= rounds || !wait(&bars.done[r % NST], q)) break;
        if (!G::SUM) {
          const int t0 = first_step(q);
          const int rows = a.time - t0 < L ? (int)(a.time - t0) : L;
          if (OP == FWD) empty(at + XO, AH, a.h, a.h_stride_b, a.h_stride_t, t0, rows);
          if (OP == BWD) empty(at + XO, ADX, a.dx, a.dx_stride_b, a.dx_stride_t, t0, rows);
          if (OP == BWD && GATE == OWN) empty(at, ADZ, a.dz, a.dz_stride_b, a.dz_stride_t, t0, rows);
          if (OP == BWD && GATE == HEAD)
            sum_heads<T, LAY, G>(at + DO, a, pl, b, t0, rw.row0, rw.row0 + rw.R, c0, D, lane, [&](int row) { return rw.shift(row); });
          if (OP == BWD && GATE == SPREAD) rw.template empty_spread<LAY>(at, at + DO, pl.part + (b * a.time + t0) * D + c0, D, rows);
          __syncwarp();  // both warps have to have emptied the stage
          if (lane == 0) mbar_arrive(smem_u32(&bars.emptied));
          if (!wait(&bars.emptied, q * NST)) break;
        }
      }
      if (r < rounds) {
        const int t0 = first_step(r);
        const int rows = n - t0 < L ? n - t0 : L;  // rows that are there (none behind the end)
        if (rows > 0) {
          if (G::X) fill(at + XO, AX, a.x, a.x_stride_b, a.x_stride_t, t0, rows);
          if (G::D) fill(at + DO, ADH, a.dh, a.dh_stride_b, a.dh_stride_t, t0, rows);
          if (GATE == OWN) fill(at, AZ, a.z, a.z_stride_b, a.z_stride_t, t0, rows);
          if (GATE == SPREAD) rw.fill_each(at, src(a.z, a.z_stride_b, a.z_stride_t, t0), a.z_stride_t, rows, ha, hb);
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
        off[j < (TMA ? 8 : S) ? j : 0] = row * G::PITCH + (warp * 8 + pr * 2) * (int)sizeof(T) +
                                         (int)((reinterpret_cast<uintptr_t>(x) + row * (x_stride_t * sizeof(T))) & 15);
      }
    }
    auto pos = [&](int i) { return TMA ? off[i & 7] + i * 128 : off[i < (TMA ? 8 : S) ? i : 0]; };
    GateTable<T, L> gates;
    if (GATE == HEAD) {
      gates.p = static_cast<const T*>(a.z) + b * a.z_stride_b + (c0 + warp * 8 < D ? c0 + warp * 8 : 0) / (int)a.width +
                (int64_t)(first_step(0) + lane) * a.z_stride_t;
      gates.stride = 32 * a.z_stride_t;
      gates.piece = (UP ? L : -L) * a.z_stride_t;
      gates.load(n - first_step(0), lane);
    }
    // the value carried along the pieces: the state, or R; composed over the segments before
    ulonglong2* sums = pl.sums + ((int64_t)b * pl.segments * tiles + tile) * 32 + warp * 4 + pr;
    f2 s = 0, tot = kOne2;  // SUM: (tot, s) of the pieces so far
    if (!G::SUM && pl.segments > 1) asm volatile("griddepcontrol.wait;" ::: "memory");  // the sums are there
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
              sts2<T, LAY>(at + pos(i), dz);
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

template <typename T, int GATE, int LAY, int OP>
cudaError_t launch_one(const Maps& m, const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st) {
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
  cfg.blockDim = dim3(32 * (kWarps + (LAY == SWZ ? 1 : kLoaders)));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = pl.segments > 1 && segs == pl.segments ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, m, a, pl, gave_up);
}

template <typename T, int GATE, int LAY, bool BACK>
cudaError_t run( const Maps& m, const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st) {
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
  bool tma = gate != SPREAD, two = true;
  pl.same = 0;
  for (int i = 0; i < 6; ++i) {
    if (!all[i].used) continue;
    tma = tma && map_ok(all[i].p, all[i].sb, all[i].st, a, e);
    // rows that start where x's do in their 16-byte chunks (and a piece's fit 32-bit offsets)
    const uintptr_t d = reinterpret_cast<uintptr_t>(all[i].p) - reinterpret_cast<uintptr_t>(a.x);
    if (d % 16 == 0 && all[i].st == a.x_stride_t && (all[i].sb - a.x_stride_b) * e % 16 == 0 && a.x_stride_t < (1 << 22))
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
    const auto enc = gate == OWN ? encode<T, Geo<T, OWN, FWD>::L> : encode<T, Geo<T, HEAD, FWD>::L>;
    for (int i = 0; i < 6; ++i)
      if (all[i].used && !enc(m.*all[i].map, all[i].p, all[i].sb, all[i].st, a)) return cudaErrorInvalidValue;
    return gate == OWN ? run<T, OWN, SWZ, BACK>(m, a, pl, gave_up, st) : run<T, HEAD, SWZ, BACK>(m, a, pl, gave_up, st);
  }
  if (gate == HEAD) return run<T, HEAD, ELEM, BACK>(m, a, pl, gave_up, st);
  if (gate == OWN) return two ? run<T, OWN, PAIR, BACK>(m, a, pl, gave_up, st) : run<T, OWN, ELEM, BACK>(m, a, pl, gave_up, st);
  return two ? run<T, SPREAD, PAIR, BACK>(m, a, pl, gave_up, st) : run<T, SPREAD, ELEM, BACK>(m, a, pl, gave_up, st);
}

cudaError_t run_fwd_bf16(const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st);
cudaError_t run_fwd_f32(const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st);
cudaError_t run_bwd_bf16(const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st);
cudaError_t run_bwd_f32(const pnn_recur_args& a, const Plan& pl, int* gave_up, cudaStream_t st);

}  // namespace recur
}  // namespace pnn
