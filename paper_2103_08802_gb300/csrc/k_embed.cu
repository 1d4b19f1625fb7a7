// Embedding lookup with scaling, and its gradient by sorted tokens.
#include <algorithm>
#include <atomic>

#include "pnn_internal.h"
#include "pnn_seq.h"
#include "seq_common.cuh"
#include "tc_ptx.cuh"

namespace pnn {
namespace {
using namespace seq;

__device__ __forceinline__ int64_t token_id(const pnn_embed_args& a, int64_t n) {
  return a.ids_bits == 64 ? static_cast<const int64_t*>(a.ids)[n] : (int64_t)static_cast<const int32_t*>(a.ids)[n];
}

// ---------------------------------------------------------------- columns
// A warp takes 256 columns of a row, a lane 8 of them: G groups of VW
// neighbouring ones, 32 VW columns apart, so that rows of any alignment are
// read and written in whole 32-lane spans (VW = 8 or, with fp32 on either side,
// 4: 16-byte aligned rows; 2, 1: rows aligned to two values or one).  fp32 with
// 8 neighbouring columns a lane would touch every 32-byte sector twice.
constexpr int kCols = 256;

// Loads stay where they are written: left to itself the compiler moves each one
// down to its use, where it waits alone (the sums of 65536 x 2048 values took
// 190 us so).
template <int BYTES>
__device__ __forceinline__ void ld_here(void* to, const void* p) {
  if constexpr (BYTES == 2) {  // (a register each: packed in pairs they would be waited for at once)
    asm volatile("ld.global.L1::no_allocate.u16 %0, [%1];" : "=r"(*static_cast<uint32_t*>(to)) : "l"(p));
  } else if constexpr (BYTES == 4) {
    asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(*static_cast<uint32_t*>(to)) : "l"(p));
  } else if constexpr (BYTES == 8) {
    uint32_t* w = static_cast<uint32_t*>(to);
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
  } else {
    uint32_t* w = static_cast<uint32_t*>(to);
#pragma unroll
    for (int i = 0; i < BYTES / 4; i += 4)
      asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3])
                   : "l"(static_cast<const char*>(p) + i * 4));
  }
}

template <typename T, int VW>
struct alignas(VW * sizeof(T) < 16 ? VW * sizeof(T) : 16) Vec {
  T v[VW];
};
template <>
struct alignas(4) Vec<bf16, 1> {
  bf16 v[1], none;
};
template <typename T, int VW, int NC = 8>
struct Cols {
  static constexpr int G = NC / VW;
  Vec<T, VW> g[G];
  // n: columns left of the row from this lane's first one on
  __device__ __forceinline__ void load(const T* p, int n) {
#pragma unroll
    for (int i = 0; i < G; ++i) {
      if (i * 32 * VW + VW <= n) {
        ld_here<VW * (int)sizeof(T)>(&g[i], p + i * 32 * VW);
      } else {
#pragma unroll
        for (int j = 0; j < VW; ++j)
          if (i * 32 * VW + j < n) g[i].v[j] = p[i * 32 * VW + j];
      }
    }
  }
  // ONCE: first to leave L2, which the rows that are read share (bf16 in 8-byte pieces is better kept: 21 us against 23
  // for 32768 x 1000)
  template <bool ONCE = false>
  __device__ __forceinline__ void store(T* p, int n) const {
#pragma unroll
    for (int i = 0; i < G; ++i) {
      if (VW > 1 && i * 32 * VW + VW <= n) {
        put<ONCE>(p + i * 32 * VW, g[i]);
      } else {
#pragma unroll
        for (int j = 0; j < VW; ++j)
          if (i * 32 * VW + j < n) p[i * 32 * VW + j] = g[i].v[j];
      }
    }
  }
  template <bool ONCE>
  static __device__ __forceinline__ void put(T* p, const Vec<T, VW>& v) {
    constexpr int N = VW * (int)sizeof(T);
    if constexpr (ONCE && N >= 16) {
#pragma unroll
      for (int q = 0; q < N / 16; ++q) __stcs(reinterpret_cast<uint4*>(p) + q, reinterpret_cast<const uint4*>(&v)[q]);
    } else if constexpr (ONCE && N == 8 && sizeof(T) == 4) {
      __stcs(reinterpret_cast<uint2*>(p), *reinterpret_cast<const uint2*>(&v));
    } else {
      *reinterpret_cast<Vec<T, VW>*>(p) = v;
    }
  }
  __device__ __forceinline__ float at(int k) const { return ld(&g[k / VW].v[k % VW]); }
  __device__ __forceinline__ void set(int k, float x) { st(&g[k / VW].v[k % VW], x); }
};

template <typename A, typename B>
constexpr int kWide = sizeof(A) + sizeof(B) == 4 ? 8 : 4;
// The widest VW whose accesses every row of the arrays allows (8: kWide).
int width_of(const void* p, int64_t stride, int64_t esz) {
  const uintptr_t u = reinterpret_cast<uintptr_t>(p);
  if (u % 16 == 0 && stride * esz % 16 == 0) return 8;
  return u % (2 * esz) == 0 && stride % 2 == 0 ? 2 : 1;
}

// ---------------------------------------------------------------- lookup
// A warp takes the same 256 columns of U consecutive tokens, so that U rows are
// on their way at a time (4 of bf16, 2 of fp32, or 1 where that would leave SMs
// without work).
// Bound: HBM and L2; 32768 x 2048 bf16 33 us (5.6 TB/s of unique rows read and
// rows written), rows of 2047 52; a call of 64 tokens is its launch.
template <typename TI, typename TO, int VW, int U>
__global__ void __launch_bounds__(256) k_embed_fwd(const __grid_constant__ pnn_embed_args a, int blocks) {
  const int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int64_t n0 = unit / blocks * U;
  if (n0 >= a.tokens) return;
  const int lane = threadIdx.x & 31;
  const int64_t c = (unit % blocks) * kCols + lane * VW;
  const int left = a.width - c < kCols ? (int)(a.width - c) : kCols;
  int64_t mine = -1;
  if (lane < U && n0 + lane < a.tokens) mine = token_id(a, n0 + lane);
  Cols<TI, VW> x[U];
  bool ok[U];
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t v = __shfl_sync(0xffffffffu, mine, u);
    ok[u] = v >= 0 && v < a.vocab;
    x[u].load(static_cast<const TI*>(a.table) + (ok[u] ? v : 0) * a.table_stride + c, left);
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (n0 + u >= a.tokens) break;
    Cols<TO, VW> y;
#pragma unroll
    for (int k = 0; k < 8; ++k) y.set(k, ok[u] ? a.scale * x[u].at(k) : 0.f);
    y.template store<true>(static_cast<TO*>(a.out) + (n0 + u) * a.out_stride + c, left);
  }
}

// ---------------------------------------------------------------- sorting the tokens
// Stable sort of (id, position) by id, least significant digit first, by one
// cluster of CTAs; padding (key = vocab) comes last.  Each warp of the cluster
// owns a contiguous range of the tokens.  A pass counts every warp's digits,
// forms each warp's first place for each digit (digits in order, within a digit
// CTAs and warps in order) and walks the ranges again to place the pairs: equal
// digits keep their order whatever runs when.  Counting sorts with atomics
// would be one launch less but leave the order of equal tokens, and with it the
// rounding of their sum, to chance.
//
// The other CTAs of the launch meanwhile zero the gradient's table.
constexpr int kSortThreads = 1024, kSortWarps = kSortThreads / 32, kMaxBits = 9, kBins = 1 << kMaxBits, kMaxSortCtas = 16;
constexpr int kAhead = 4;  // keys a lane loads at a time; a warp with no more keeps them between its two walks
struct SortShared {
  uint32_t cnt[kSortWarps][kBins];      // counts, then next places from the digit's first (sum)
  uint32_t tot[kMaxSortCtas][kBins];    // of each CTA of the cluster
  uint32_t sum[kBins];
  uint32_t part[kSortWarps];
};

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void put_remote(const uint32_t* place, uint32_t rank, uint32_t v) {
  uint32_t at = static_cast<uint32_t>(__cvta_generic_to_shared(place)), to;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(to) : "r"(at), "r"(rank));
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(to), "r"(v) : "memory");
}

// The lanes with this lane's digit, among those that are on: a ballot for each
// bit (match.any answers a warp in about 60 cycles, one at a time for the whole
// SM: the sort of 65536 tokens took 40 us with it).
__device__ __forceinline__ uint32_t equal_digits(uint32_t d, int bits, bool on) {
  uint32_t same = __ballot_sync(0xffffffffu, on);
#pragma unroll
  for (int i = 0; i < kMaxBits; ++i)
    if (i < bits) {
      const bool one = d >> i & 1;
      const uint32_t b = __ballot_sync(0xffffffffu, one);
      same &= one ? b : ~b;
    }
  return same;
}

__global__ void __launch_bounds__(kSortThreads, 1) k_embed_sort(const __grid_constant__ pnn_embed_args a, uint2* buf0, uint2* buf1, int passes,
                                                               int bits, int C, int fill, int64_t fill_bytes) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  extern __shared__ __align__(128) char raw[];
  SortShared& s = *reinterpret_cast<SortShared*>(raw);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  if ((int)blockIdx.x >= C) {
    // zeros: contiguous rows as one span, by bulk copies of a block of zeros in shared memory; strided ones row by row
    const int esz = a.dtable_dtype == PNN_DT_BF16 ? 2 : 4;
    char* p = static_cast<char*>(a.dtable);
    if (fill == 1) {
      constexpr int BLOCK = 32768;
      for (int i = tid; i < BLOCK / 16; i += kSortThreads) reinterpret_cast<uint4*>(raw)[i] = make_uint4(0, 0, 0, 0);
      tc::fence_proxy_async();
      __syncthreads();
      const int64_t whole = fill_bytes / 16 * 16;
      if (tid == 0) {
        for (int64_t at = (int64_t)(blockIdx.x - C) * BLOCK; at < whole; at += (int64_t)(gridDim.x - C) * BLOCK) {
          const int n = whole - at < BLOCK ? (int)(whole - at) : BLOCK;
          asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(p + at), "r"(tc::smem_u32(raw)), "r"(n)
                       : "memory");
          tc::bulk_commit();
        }
        tc::bulk_wait_all();
      }
      if (blockIdx.x == C && tid < (fill_bytes - whole) / 2) *reinterpret_cast<uint16_t*>(p + whole + tid * 2) = 0;
    } else if (fill == 2) {
      const int64_t halves = a.width * esz / 2;
      for (int64_t r = (int64_t)(blockIdx.x - C) * kSortWarps + warp; r < a.vocab; r += (int64_t)(gridDim.x - C) * kSortWarps) {
        uint16_t* q = reinterpret_cast<uint16_t*>(p + r * a.dtable_stride * esz);
        for (int64_t i = lane; i < halves; i += 32) q[i] = 0;
      }
    }
    return;
  }
  const int rank = C > 1 ? (int)cluster_rank() : 0;
  const int64_t N = a.tokens;
  const int64_t per = (N + C * kSortThreads - 1) / (C * kSortThreads) * 32;  // tokens of a warp
  const int64_t lo = ((int64_t)rank * kSortWarps + warp) * per, hi = lo + per < N ? lo + per : N;
  const uint32_t mask = (1u << bits) - 1;
  for (int pass = 0; pass < passes; ++pass) {
    const uint2* in = pass & 1 ? buf0 : buf1;
    uint2* out = pass & 1 ? buf1 : buf0;
    const int shift = pass * bits;
    auto fetch = [&](int64_t i) {
      if (i >= hi) return make_uint2(0xffffffffu, 0u);
      if (pass) return in[i];
      const int64_t v = token_id(a, i);
      return make_uint2(v >= 0 && v < a.vocab ? (uint32_t)v : (uint32_t)a.vocab, (uint32_t)i);
    };
    uint2 e[kAhead];
    const bool once = per <= 32 * kAhead;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) e[k] = fetch(lo + k * 32 + lane);
    for (int i = tid; i < kSortWarps * kBins / 4; i += kSortThreads) reinterpret_cast<uint4*>(s.cnt)[i] = make_uint4(0, 0, 0, 0);
    if (C > 1 && pass == 0) cluster_sync();  // every CTA of the cluster runs before its shared memory is written
    else __syncthreads();
    for (int64_t i0 = lo; i0 < hi; i0 += 32 * kAhead) {
      if (i0 > lo) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) e[k] = fetch(i0 + k * 32 + lane);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (i0 + k * 32 + lane < hi) atomicAdd(&s.cnt[warp][(e[k].x >> shift) & mask], 1u);
      }
    }
    __syncthreads();
    // places within the CTA, and its totals for all of the cluster
    if (tid < kBins) {
      uint32_t n = 0;
#pragma unroll 8
      for (int w = 0; w < kSortWarps; ++w) {
        const uint32_t c = s.cnt[w][tid];
        s.cnt[w][tid] = n;
        n += c;
      }
      if (C > 1)
        for (int r = 0; r < C; ++r) put_remote(&s.tot[rank][tid], r, n);
      else s.tot[0][tid] = n;
    }
    if (C > 1) cluster_sync();
    else __syncthreads();
    // first place of each digit: those of the digits before, then the CTAs before
    if (tid < kBins) {
      uint32_t n = 0, before = 0;
      for (int r = 0; r < C; ++r) {
        if (r == rank) before = n;
        n += s.tot[r][tid];
      }
      uint32_t run = n;
#pragma unroll
      for (int o = 1; o < 32; o *= 2) {
        const uint32_t u = __shfl_up_sync(0xffffffffu, run, o);
        if (lane >= o) run += u;
      }
      if (lane == 31) s.part[warp] = run;
      s.sum[tid] = run - n + before;
    }
    __syncthreads();
    if (tid < kBins) {
      uint32_t n = s.sum[tid];
      for (int w = 0; w < warp; ++w) n += s.part[w];
      s.sum[tid] = n;
    }
    __syncthreads();
    for (int64_t i0 = lo; i0 < hi; i0 += 32 * kAhead) {
      if (!once) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k) e[k] = fetch(i0 + k * 32 + lane);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const bool on = i0 + k * 32 + lane < hi;
        const uint32_t d = (e[k].x >> shift) & mask, same = equal_digits(d, bits, on);
        const uint32_t before = __popc(same & ((1u << lane) - 1)), at = on ? s.sum[d] + s.cnt[warp][d] + before : 0;
        __syncwarp();
        if (on && before == 0) s.cnt[warp][d] += __popc(same);
        __syncwarp();
        if (on) out[at] = e[k];
      }
    }
    if (pass + 1 == passes) return;
    if (C > 1) cluster_sync();
    else __syncthreads();
  }
}

// ---------------------------------------------------------------- adding the rows
// The sorted pairs are cut into pieces of `piece` (16 or more).  A warp adds the
// rows of one piece's runs of equal ids, 256 columns of them, in order.  A run
// that lies in the piece is written; of one that goes on into other pieces its
// part is put down in fp32 (parts[piece][0]: the run began before, [1]: it
// begins here and goes on), and k_embed_join adds those, again in order.
//
// accumulate into fp32: every element is added to once in the whole call, so
// one red.add for each (no wait for the old value) has one result.  It takes
// subnormal values for 0 and gives 0 for a subnormal sum (measured), which loses
// less than 2^-125.  bf16 rows
// are read beside the rows that are added (at a run's end, each with its whole
// latency, 65536 x 1000 took 92 us instead of 82).
//
// Bound: the latency of a batch of rows times a piece's batches, then HBM.
// With the sort and the zero fill: 8192 x 1000 bf16 into 32000 fp32 rows 37 us
// (18 sort beside fill, 9 sums, 9 joins), 65536 x 2048 bf16 added to fp32 119
// (5.0 TB/s), to bf16 102, 65536 x 1023 bf16 into 50000 fp32 rows 114.
struct SumPlan {
  const uint2* sorted;
  float* parts;  // [pieces][2][pitch], rows of width
  int64_t pitch;
  int64_t pieces;
  int piece, blocks;
};

// y: bf16 rows that are added to, as they were
template <typename TO, int VW, int NC>
__device__ __forceinline__ void write_row(const pnn_embed_args& a, uint32_t id, int64_t c, int left, const float (&acc)[NC], Cols<TO, VW, NC> y) {
  TO* p = static_cast<TO*>(a.dtable) + (int64_t)id * a.dtable_stride + c;
  if (a.accumulate) {
    if constexpr (sizeof(TO) == 4) {
#pragma unroll
      for (int g = 0; g < NC / VW; ++g) {
        float* q = reinterpret_cast<float*>(p) + g * 32 * VW;
        if (VW >= 4 && g * 32 * VW + VW <= left) {
#pragma unroll
          for (int k = 0; k < VW; k += 4)
            asm volatile("red.global.add.v4.f32 [%0], {%1, %2, %3, %4};" ::"l"(q + k), "f"(a.scale * acc[g * VW + k]), "f"(a.scale * acc[g * VW + k + 1]),
                         "f"(a.scale * acc[g * VW + k + 2]), "f"(a.scale * acc[g * VW + k + 3])
                         : "memory");
        } else {
#pragma unroll
          for (int k = 0; k < VW; ++k)
            if (g * 32 * VW + k < left) asm volatile("red.global.add.f32 [%0], %1;" ::"l"(q + k), "f"(a.scale * acc[g * VW + k]) : "memory");
        }
      }
      return;
    } else {
#pragma unroll
      for (int k = 0; k < NC; ++k) y.set(k, y.at(k) + a.scale * acc[k]);
    }
  } else {
#pragma unroll
    for (int k = 0; k < NC; ++k) y.set(k, a.scale * acc[k]);
  }
  y.store(p, left);
}
template <int VW>
__device__ __forceinline__ float* part_at(const pnn_embed_args& a, const SumPlan& pl, int64_t piece, int which, int64_t c) {
  return pl.parts + (piece * 2 + which) * pl.pitch + c;
}

template <typename TI, typename TO, int VW>
__global__ void __launch_bounds__(256, 2) k_embed_sum(const __grid_constant__ pnn_embed_args a, const __grid_constant__ SumPlan pl) {
  constexpr int B = sizeof(TI) == 2 && VW > 1 ? 8 : 4;  // rows on their way at a time (VW = 1 has 32 registers for 4)
  asm volatile("griddepcontrol.launch_dependents;\n\tgriddepcontrol.wait;" ::: "memory");  // the tokens are sorted, the table zeroed
  const int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), p = unit / pl.blocks;
  if (p >= pl.pieces) return;
  const int lane = threadIdx.x & 31;
  const int64_t cb = (unit - p * pl.blocks) * kCols, c = cb + lane * VW;
  const int left = a.width - c < kCols ? (int)(a.width - c) : kCols;
  const int64_t N = a.tokens, i0 = p * pl.piece, i1 = i0 + pl.piece < N ? i0 + pl.piece : N;
  const uint32_t V = (uint32_t)a.vocab, none = 0xffffffffu;
  const uint32_t prev = i0 ? pl.sorted[i0 - 1].x : none, next = i1 < N ? pl.sorted[i1].x : none;
  uint32_t cur = none;
  bool here = true;  // the present run began in this piece
  float acc[8];
  constexpr bool OLD = sizeof(TO) == 2;  // rows that are read before they are written (fp32 ones are added to in memory)
  Cols<TO, VW> old;                      // the present run's row
  auto put = [&](bool goes_on) {
    if (cur >= V) return;
    if (here && !goes_on) {
      write_row<TO, VW, 8>(a, cur, c, left, acc, old);
    } else {
      float* q = part_at<VW>(a, pl, p, here ? 1 : 0, c);
      Cols<float, VW> y;
#pragma unroll
      for (int k = 0; k < 8; ++k) y.set(k, acc[k]);
      y.store(q, left);
    }
  };
  for (int64_t j0 = i0; j0 < i1; j0 += 32) {
    const uint2 mine = j0 + lane < i1 ? pl.sorted[j0 + lane] : make_uint2(none, 0);
    const int n = i1 - j0 < 32 ? (int)(i1 - j0) : 32;
    for (int e0 = 0; e0 < n; e0 += B) {
      Cols<TI, VW> x[B];
      Cols<TO, VW> row[OLD ? B : 1];
      uint32_t id[B];
#pragma unroll
      for (int e = 0; e < B; ++e) {
        id[e] = __shfl_sync(0xffffffffu, mine.x, e0 + e);
        const uint32_t pos = __shfl_sync(0xffffffffu, mine.y, e0 + e);
        x[e].load(static_cast<const TI*>(a.dout) + (int64_t)pos * a.dout_stride + c, left);  // (some row where there is no pair)
        if (OLD && a.accumulate && id[e] < V && id[e] != (e ? id[e - 1] : cur))
          row[e].load(static_cast<const TO*>(a.dtable) + (int64_t)id[e] * a.dtable_stride + c, left);
      }
#pragma unroll
      for (int e = 0; e < B; ++e) {
        if (e0 + e >= n) break;
        if (id[e] != cur || (j0 == i0 && e0 + e == 0)) {
          put(false);
          cur = id[e];
          if constexpr (OLD) old = row[e];
          here = !(j0 == i0 && e0 + e == 0 && cur == prev);
#pragma unroll
          for (int k = 0; k < 8; ++k) acc[k] = 0.f;
        }
        if (cur < V) {
#pragma unroll
          for (int k = 0; k < 8; ++k) acc[k] += x[e].at(k);
        }
      }
    }
  }
  put(cur == next);
}

// The run that begins in a piece and goes on: its part there and the parts of
// the pieces after, in order.  Few warps find one: they are small, so that many
// look at once.
template <typename TO, int VW>
__global__ void __launch_bounds__(256, 4) k_embed_join(const __grid_constant__ pnn_embed_args a, const __grid_constant__ SumPlan pl, int blocks) {
  constexpr int NC = 4, B = 8;
  asm volatile("griddepcontrol.wait;" ::: "memory");  // the parts are there
  const int64_t unit = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), p = unit / blocks;
  const int64_t N = a.tokens, i0 = p * pl.piece, i1 = i0 + pl.piece;
  if (p >= pl.pieces || i1 >= N) return;
  const uint32_t id = pl.sorted[i1 - 1].x;
  const int lane = threadIdx.x & 31;
  // the pieces after that begin within the run, 32 looked at a time
  auto within = [&](int64_t q0) { return __ballot_sync(0xffffffffu, q0 + lane < pl.pieces && pl.sorted[(q0 + lane) * pl.piece].x == id); };
  uint32_t in = within(p + 1);
  if (id >= (uint32_t)a.vocab || !(in & 1)) return;                         // nothing goes on
  if (pl.sorted[i0].x == id && i0 && pl.sorted[i0 - 1].x == id) return;     // it began before
  const int64_t c = (unit - p * blocks) * 32 * NC + lane * VW;
  const int left = a.width - c < 32 * NC ? (int)(a.width - c) : 32 * NC;
  Cols<float, VW, NC> v[B];
  float acc[NC];
  v[0].load(part_at<VW>(a, pl, p, 1, c), left);
#pragma unroll
  for (int k = 0; k < NC; ++k) acc[k] = v[0].at(k);
  for (int64_t q0 = p + 1;; q0 += 32) {
    const int n = ~in ? __ffs(~in) - 1 : 32;
    for (int q = 0; q < n; q += B) {
#pragma unroll
      for (int i = 0; i < B; ++i) v[i].load(part_at<VW>(a, pl, q0 + (q + i < n ? q + i : 0), 0, c), left);
#pragma unroll
      for (int i = 0; i < B; ++i)
        if (q + i < n) {
#pragma unroll
          for (int k = 0; k < NC; ++k) acc[k] += v[i].at(k);
        }
    }
    if (n < 32) break;
    in = within(q0 + 32);
  }
  Cols<TO, VW, NC> old;
  if (sizeof(TO) == 2 && a.accumulate) old.load(static_cast<const TO*>(a.dtable) + (int64_t)id * a.dtable_stride + c, left);
  write_row<TO, VW, NC>(a, id, c, left, acc, old);
}

template <typename TI, typename TO, int VW>
cudaError_t forward(const pnn_embed_args& a, cudaStream_t st) {
  const int blocks = (int)((a.width + kCols - 1) / kCols);
  constexpr int U = sizeof(TI) == 2 ? 4 : 2;
  const bool many = a.tokens * blocks >= (int64_t)device_sm_count() * 16 * U;  // 16 warps an SM or more
  const int64_t units = (many ? (a.tokens + U - 1) / U : a.tokens) * blocks;
  const unsigned g = (unsigned)((units + 7) / 8);
  if (many) k_embed_fwd<TI, TO, VW, U><<<g, 256, 0, st>>>(a, blocks);
  else k_embed_fwd<TI, TO, VW, 1><<<g, 256, 0, st>>>(a, blocks);
  return cudaGetLastError();
}
template <typename TI, typename TO>
cudaError_t forward(const pnn_embed_args& a, cudaStream_t st) {
  const int w = std::min(width_of(a.table, a.table_stride, sizeof(TI)), width_of(a.out, a.out_stride, sizeof(TO)));
  return w == 8 ? forward<TI, TO, kWide<TI, TO>>(a, st) : w == 2 ? forward<TI, TO, 2>(a, st) : forward<TI, TO, 1>(a, st);
}

template <typename TI, typename TO, int VW>
cudaError_t add_up(const pnn_embed_args& a, const SumPlan& pl, cudaStream_t st) {
  // each launch may begin beside the one before and waits for it in the kernel
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(256);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  cfg.gridDim = dim3((unsigned)((pl.pieces * pl.blocks + 7) / 8));
  const cudaError_t e = cudaLaunchKernelEx(&cfg, k_embed_sum<TI, TO, VW>, a, pl);
  if (e != cudaSuccess || pl.pieces == 1) return e;
  const int blocks = (int)((a.width + 127) / 128);
  cfg.gridDim = dim3((unsigned)((pl.pieces * blocks + 7) / 8));
  return cudaLaunchKernelEx(&cfg, k_embed_join<TO, VW == 8 ? 4 : VW>, a, pl, blocks);
}
template <typename TI, typename TO>
cudaError_t add_up(const pnn_embed_args& a, const SumPlan& pl, cudaStream_t st) {
  const int w = std::min(width_of(a.dout, a.dout_stride, sizeof(TI)), width_of(a.dtable, a.dtable_stride, sizeof(TO)));
  return w == 8 ? add_up<TI, TO, kWide<TI, TO>>(a, pl, st) : w == 2 ? add_up<TI, TO, 2>(a, pl, st) : add_up<TI, TO, 1>(a, pl, st);
}

// Pairs of a piece: so many that the warps (a piece's 256 columns each) fill the
// 16 places of every SM once, or a whole number of times with 192 pairs or so,
// 16 at least.
SumPlan plan_of(const pnn_embed_args& a) {
  SumPlan pl{};
  pl.blocks = (int)((a.width + kCols - 1) / kCols);
  const int64_t places = (int64_t)device_sm_count() * 16, units = a.tokens * pl.blocks, waves = std::max<int64_t>(1, (units / places + 96) / 192);
  pl.piece = std::max<int64_t>(16, (units + places * waves - 1) / (places * waves));
  pl.piece = (pl.piece + 7) / 8 * 8;
  pl.pieces = (a.tokens + pl.piece - 1) / pl.piece;
  pl.pitch = (a.width + 3) / 4 * 4;
  return pl;
}
size_t al256(size_t x) { return (x + 255) & ~(size_t)255; }
}  // namespace

cudaError_t launch_embed_fwd(const pnn_embed_args& a, cudaStream_t st) {
  if (a.table_dtype == PNN_DT_BF16) return a.out_dtype == PNN_DT_BF16 ? forward<bf16, bf16>(a, st) : forward<bf16, float>(a, st);
  return a.out_dtype == PNN_DT_BF16 ? forward<float, bf16>(a, st) : forward<float, float>(a, st);
}

size_t embed_workspace(const pnn_embed_args& a) {
  const SumPlan pl = plan_of(a);
  return 2 * al256((size_t)a.tokens * sizeof(uint2)) + (size_t)pl.pieces * 2 * pl.pitch * 4;
}

cudaError_t launch_embed_bwd(const pnn_embed_args& a, void* ws, cudaStream_t st) {
  SumPlan pl = plan_of(a);
  char* p = static_cast<char*>(ws);
  uint2 *b0 = reinterpret_cast<uint2*>(p), *b1 = reinterpret_cast<uint2*>(p + al256((size_t)a.tokens * sizeof(uint2)));
  pl.parts = reinterpret_cast<float*>(p + 2 * al256((size_t)a.tokens * sizeof(uint2)));
  int bits = 1;
  while (a.vocab >> bits) ++bits;  // of the largest key, vocab
  const int passes = (bits + kMaxBits - 1) / kMaxBits, digit = (bits + passes - 1) / passes;
  int C = 1;
  while (C < kMaxSortCtas && (int64_t)C * kSortThreads * kAhead < a.tokens) C *= 2;
  // the zeros: 0 none, 1 one span, 2 row by row
  const int64_t esz = a.dtable_dtype == PNN_DT_BF16 ? 2 : 4, bytes = a.vocab * a.width * esz;
  const int fill = a.accumulate ? 0 : a.dtable_stride == a.width && reinterpret_cast<uintptr_t>(a.dtable) % 16 == 0 ? 1 : 2;
  int64_t fillers = 0;
  if (fill) fillers = std::min<int64_t>(std::max(device_sm_count() - C, 1), (bytes / 16 + kSortThreads - 1) / kSortThreads + 1);
  fillers = (fillers + C - 1) / C * C;
  static std::atomic<uint64_t> ready{0};  // one bit a device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(k_embed_sort, cudaFuncAttributeMaxDynamicSharedMemorySize, sizeof(SortShared));
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_embed_sort, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(C + fillers));
  cfg.blockDim = dim3(kSortThreads);
  cfg.dynamicSmemBytes = sizeof(SortShared);
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = C > 1 ? 1 : 0;
  e = cudaLaunchKernelEx(&cfg, k_embed_sort, a, b0, b1, passes, digit, C, fill, bytes);
  if (e != cudaSuccess || a.tokens == 0) return e;
  pl.sorted = passes & 1 ? b0 : b1;
  if (a.dout_dtype == PNN_DT_BF16) return a.dtable_dtype == PNN_DT_BF16 ? add_up<bf16, bf16>(a, pl, st) : add_up<bf16, float>(a, pl, st);
  return a.dtable_dtype == PNN_DT_BF16 ? add_up<float, bf16>(a, pl, st) : add_up<float, float>(a, pl, st);
}

}  // namespace pnn
