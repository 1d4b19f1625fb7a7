// Distillation from a teacher's top logits mixed with the labels' cross
// entropy: loss and gradient in one pass over the logits.
//
// A team (a warp, a CTA, or a cluster of CTAs) holds one row in its registers:
// the row is read once, every warp forms the softmax sums from its own maximum,
// the warps' (maximum, sums) meet once in shared memory
//   S = sum_w s_w exp((m_w - m) / tau),
// and the gradient is written from the registers.  The row's few places that
// the teacher or the label names are written again after that with what they
// take off; pairs of the same id add up in the order of the list.
//
// Exponents are (s - m) k with k = log2(e) / tau, the difference first: it is
// exact to one rounding however large the logits are (a fused s k - m k would
// lose all of it there, at the type's lowest value for instance).
//
// Bound: HBM (one read, one write of the row) for long rows; for those of one
// CTA's registers 17 instructions an element, in long dependent stretches that
// 24 warps an SM do not cover (half the issue slots are used; the exponentials'
// pipe is a quarter busy).  4096 x 32000 bf16 take 88 us with one temperature (6.0 TB/s),
// 103 mixed with labels at tau = 2; 4096 x 128003 399 (2.5 GB moved, 6.3 TB/s);
// 256 x 1000 fp32 6.
#include <math.h>

#include <atomic>

#include "pnn_internal.h"
#include "pnn_seq.h"
#include "row_logits.cuh"
#include "tc_ptx.cuh"

namespace pnn {
namespace {
using namespace seq;

// A pair of the teacher, or the label, as a place of the row.
struct Entry {
  int id;
  float t, s;  // the teacher's logit (then its probability), the student's
};

// How the two softmaxes are formed.  ONE: a single temperature serves (tau = 1,
// or only one term).  TWO: two exponentials.  SQUARE, FOURTH: tau is 2 or 4, so
// that exp(s - m) is a power of exp((s - m) / tau).  Rows in registers take, with
// labels and 32 ids, at tau 2, 4 and (TWO) 3: 4096 x 32000 bf16 104, 104 and 115
// us, 8192 rows 200, 198 and 225, 16384 x 8000 129, 144 and 152, 16384 x 2000 32,
// 33 and 36; rows walked twice and fp32 ones, bound by HBM, 402, 400 and 417
// (4096 x 128000 bf16), 172, 171 and 173 (4096 x 32000 fp32).
enum { ONE, TWO, SQUARE, FOURTH };
// exp(y) from y = s - m and e = exp(y / tau)
template <int MODE>
__device__ __forceinline__ f2 second(f2 y, f2 e) {
  if constexpr (MODE == TWO) return ex2p(mul2(y, pk(kLog2e, kLog2e)));
  else if constexpr (MODE == SQUARE) return mul2(e, e);
  else return mul2(mul2(e, e), mul2(e, e));
}
template <int MODE>
__device__ __forceinline__ float second1(float y, float e) {
  return MODE == TWO ? ex2(y * kLog2e) : MODE == SQUARE ? e * e : (e * e) * (e * e);
}

// What every team computes with, from the arguments.
struct Terms {
  int V, K;
  float kt;  // log2(e) / tau (or at 1 where the label's term is alone)
  bool teach, labelled;
  __device__ __forceinline__ explicit Terms(const pnn_distill_args& a) {
    V = (int)a.vocab;
    K = a.k;
    teach = K > 0 && a.alpha > 0.f;
    labelled = a.labels && a.alpha < 1.f;
    kt = (teach ? 1.f / a.tau : 1.f) * kLog2e;
  }
  // pair j of row r as it stands in memory (fp32 or 16 bits of the teacher's logit), the label for j = K
  __device__ __forceinline__ void raw(const pnn_distill_args& a, int64_t r, int j, int& id, uint32_t& t) const {
    id = -1;
    t = 0;
    if (j < K && teach) {
      id = a.ids[r * K + j];
      t = a.teacher_dtype == PNN_DT_BF16 ? static_cast<const uint16_t*>(a.teacher)[r * K + j] : static_cast<const uint32_t*>(a.teacher)[r * K + j];
    } else if (j == K && labelled) {
      id = a.labels[r];
    }
  }
  __device__ __forceinline__ void read(const pnn_distill_args& a, int j, uint32_t raw, int& id, float& t) const {
    const bool on = id >= 0 && id < V;
    t = on && j < K ? __uint_as_float(a.teacher_dtype == PNN_DT_BF16 ? raw << 16 : raw) : -INFINITY;
    if (!on) id = -1;
  }
  __device__ __forceinline__ void entry(const pnn_distill_args& a, int64_t r, int j, int& id, float& t) const {
    uint32_t v;
    raw(a, r, j, id, v);
    read(a, j, v, id, t);
  }
};

// A row's sums over all its warps, and the factors of its gradient
//   gt exp((s - m) / tau) + gh exp(s - m).
template <int MODE>
struct Result {
  float b, t, h, mt, w;  // base and sums of the student's exponentials, the teacher's maximum and sum
  float k;
  bool soft, hard;
  float gt, gh, ct, ch;
  __device__ __forceinline__ Result(const pnn_distill_args& a, const Terms& q, float m, float t_, float h_, float mt_, float w_, bool label,
                                    int64_t row)
      : b(base_of(m)), t(t_), h(MODE == ONE ? t_ : h_), mt(mt_), w(w_), k(q.kt) {
    soft = q.teach && w != 0.f && t != 0.f;
    hard = label && h != 0.f;
    const float wt = a.weight && a.dlogits ? a.weight[row] : 1.f;
    ct = soft ? wt * a.alpha * a.tau : 0.f;
    ch = hard ? wt * (1.f - a.alpha) : 0.f;
    const float x = soft ? __fdividef(ct, t) : 0.f, y = hard ? __fdividef(ch, h) : 0.f;
    gt = MODE == ONE ? x + y : x;
    gh = y;
  }
  __device__ __forceinline__ float grad(float s) const {
    const float y = s - b, e = ex2(y * k);
    float g = gt * e;
    if (MODE != ONE) g = fmaf(gh, second1<MODE>(y, e), g);
    return soft || hard ? g : 0.f;
  }
  // by one warp: the loss.  The teacher's term is alpha tau sum p_j x_j with x_j = (t_j - mt) - (s_j - b) + tau (log t - log w),
  // in the logits' units and with p summing to 1: nothing in between overflows where the loss does not, not even at a logit of
  // the type's lowest value
  __device__ __forceinline__ void loss(const pnn_distill_args& a, const Terms& q, const Entry* ent, int64_t row, int lane) const {
    float sum = 0.f;
    if (soft) {
      const float c = a.tau * kLn2 * (log2f(t) - log2f(w)), iw = 1.f / w;
      for (int j = lane; j < q.K; j += 32) {
        const Entry e = ent[j];
        const float y = e.t - mt, p = ex2(y * q.kt) * iw;
        if (p != 0.f) sum += p * (y - (e.s - b) + c);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    }
    if (lane == 0) {
      float l = 0.f;
      if (soft) l = a.alpha * a.tau * sum;
      if (hard) l += (1.f - a.alpha) * (logf(h) - (ent[q.K].s - b));
      a.loss[row] = l;
    }
  }
  // the gradient where a teacher's entry points alone, or beside the label
  __device__ __forceinline__ float at_single(const Terms& q, const Entry& e, bool label) const {
    float g = grad(e.s);
    if (soft) g -= ex2((e.t - mt) * q.kt) * __fdividef(ct, w);
    return label && hard ? g - ch : g;
  }
  // the gradient where an entry points, whatever the others do
  __device__ __forceinline__ float at_entry(const Terms& q, const Entry* ent, const Entry& e) const {
    float off = 0.f;
    if (soft) {
#pragma unroll 4
      for (int i = 0; i < q.K; ++i)
        if (ent[i].id == e.id) off += ex2((ent[i].t - mt) * q.kt);
      off *= __fdividef(ct, w);
    }
    float g = grad(e.s) - off;
    if (hard && e.id == ent[q.K].id) g -= ch;
    return g;
  }
};

// Whether the teacher names a place twice, by one warp: more than 32 ids go into
// a table of twice as many slots (a power of two), each to the first free one
// from its hash on.  (Comparing all pairs, a row of 32000 logits with 128 ids
// kept its helper busy for 21 us and the other warps waiting.)
__host__ __device__ inline int table_bits(int k) {
  int b = 6;
  while ((1 << b) < 2 * k) ++b;
  return b;
}
__device__ __forceinline__ bool repeats(const Entry* ent, int K, int* table, int bits, int lane) {
  if (K <= 32) {
    const int id = lane < K ? ent[lane].id : -1;
    const uint32_t same = __match_any_sync(0xffffffffu, id);
    return __any_sync(0xffffffffu, id >= 0 && (same & (same - 1)));
  }
  const int size = 1 << bits;
  __syncwarp();  // the row before has been looked up
  for (int i = lane; i < size; i += 32) table[i] = -1;
  __syncwarp();
  bool twice = false;
  for (int j = lane; j < K; j += 32) {
    const int id = ent[j].id;
    if (id < 0) continue;
    for (uint32_t h = (uint32_t)id * 2654435769u >> (32 - bits);; h = (h + 1) & (size - 1)) {
      const int there = atomicCAS(&table[h], -1, id);
      twice |= there == id;
      if (there == -1 || there == id) break;
    }
  }
  return __any_sync(0xffffffffu, twice);
}
// The gradient where the entries point, by one warp; mine(id): whether it is this team's to write.
template <typename T, int MODE, typename F>
__device__ __forceinline__ void write_entries(const Result<MODE>& r, const Terms& q, const Entry* ent, bool twice, T* d, int lane, F mine) {
  const int label = ent[q.K].id;
  if (twice) {
    for (int j = lane; j <= q.K; j += 32) {
      const Entry e = ent[j];
      if (e.id >= 0 && mine(e.id)) ::pnn::seq::st(d + e.id, r.at_entry(q, ent, e));
    }
    return;
  }
  bool met = false;
  for (int j = lane; j < q.K; j += 32) {
    const Entry e = ent[j];
    if (e.id < 0) continue;
    met |= e.id == label;
    if (mine(e.id)) ::pnn::seq::st(d + e.id, r.at_single(q, e, e.id == label));
  }
  met = __any_sync(0xffffffffu, met);
  if (lane == 0 && label >= 0 && !met && mine(label)) ::pnn::seq::st(d + label, r.grad(ent[q.K].s) - (r.hard ? r.ch : 0.f));
}

// The sums of a thread's vectors; the warp's maximum is m.
template <typename T, int MODE, int NV>
__device__ __forceinline__ void sums(const uint4 (&x)[NV], int used, float b, float k, float& t, float& h) {
  const f2 k2 = pk(k, k), nb = pk(-b, -b);
  f2 at = 0, ah = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (i < used) {
#pragma unroll
      for (int p = 0; p < kPairs<T>; ++p) {
        const f2 y = add2(pair_of<T>(x[i], p), nb), e = ex2p(mul2(y, k2));
        at = add2(at, e);
        if (MODE == SQUARE) ah = fma2(e, e, ah);
        else if (MODE != ONE) ah = add2(ah, second<MODE>(y, e));
      }
    }
  float u, v;
  upk(at, u, v);
  t = u + v;
  upk(ah, u, v);
  h = u + v;
}
// The gradient of a vector.
template <typename T, int MODE>
__device__ __forceinline__ uint4 grads(const uint4& x, const Result<MODE>& r) {
  const f2 k2 = pk(r.k, r.k), nb = pk(-r.b, -r.b);
  const f2 gt = pk(r.gt, r.gt), gh = pk(r.gh, r.gh);
  uint4 o;
  uint32_t* w = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
  for (int p = 0; p < kPairs<T>; ++p) {
    const f2 y = add2(pair_of<T>(x, p), nb), e = ex2p(mul2(y, k2));
    f2 g;
    if (MODE == ONE) g = mul2(gt, e);
    else if (MODE == SQUARE) g = mul2(e, fma2(gh, e, gt));
    else g = fma2(gh, second<MODE>(y, e), mul2(gt, e));
    float u, v;
    upk(g, u, v);
    if constexpr (sizeof(T) == 2) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(u, v);
      w[p] = *reinterpret_cast<const uint32_t*>(&b);
    } else {
      w[2 * p] = __float_as_uint(u);
      w[2 * p + 1] = __float_as_uint(v);
    }
  }
  return o;
}
// ---------------------------------------------------------------- a warp a row
constexpr int kWarpVecs = 8;
template <typename T, int MODE>
__global__ void __launch_bounds__(128) k_distill_warp(const __grid_constant__ pnn_distill_args a, int bits) {
  extern __shared__ Entry entries[];  // [warp][K + 1], then the warps' tables
  const int lane = threadIdx.x & 31, team = threadIdx.x >> 5;
  const int64_t row = (int64_t)blockIdx.x * 4 + team;
  if (row >= a.rows) return;
  const Terms q(a);
  const Span<T> sp(a.logits, a.logits_stride, q.V, row, 0, 1);
  Entry* ent = entries + team * (q.K + 1);
  uint4 x[kWarpVecs];
#pragma unroll
  for (int i = 0; i < kWarpVecs; ++i) x[i] = i * 32 + lane < sp.nv ? ld_once(sp.vec() + i * 32 + lane) : minus_inf<T>();
  const int lone = sp.lone(q.V, 0, lane);
  const float one = lone >= 0 ? ld(sp.s + lone) : -INFINITY;
  float mt = -INFINITY;
  for (int j = lane; j <= q.K; j += 32) {
    Entry e;
    q.entry(a, row, j, e.id, e.t);
    e.s = e.id >= 0 ? ld(sp.s + e.id) : 0.f;
    ent[j] = e;
    mt = fmaxf(mt, e.t);
  }
  const float m = warp_max<T>(x, one);
  const float b = base_of(m);
  float t, h;
  sums<T, MODE>(x, (sp.nv + 31) / 32, b, q.kt, t, h);
  if (lone >= 0) {
    const float e = ex2((one - b) * q.kt);
    t += e;
    if (MODE != ONE) h += second1<MODE>(one - b, e);
  }
  t = warp_sum(t);
  if (MODE != ONE) h = warp_sum(h);
#pragma unroll
  for (int o = 16; o; o >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, o));
  if (mt == -INFINITY) mt = 0.f;
  __syncwarp();
  float w = 0.f;
  for (int j = lane; j < q.K; j += 32) w += ex2((ent[j].t - mt) * q.kt);
  const Result<MODE> r(a, q, m, t, h, mt, warp_sum(w), ent[q.K].id >= 0, row);
  r.loss(a, q, ent, row, lane);
  if (!a.dlogits) return;
  T* d = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
  const bool same = ((reinterpret_cast<uintptr_t>(d) ^ reinterpret_cast<uintptr_t>(sp.s)) & 15) == 0, some = r.soft || r.hard;
#pragma unroll
  for (int i = 0; i < kWarpVecs; ++i)
    if (i * 32 + lane < sp.nv) put<T>(d + sp.head + (i * 32 + lane) * Span<T>::E, some ? grads<T, MODE>(x[i], r) : make_uint4(0, 0, 0, 0), same);
  if (lone >= 0) ::pnn::seq::st(d + lone, r.grad(one));
  if (!some) return;
  __syncwarp();  // the row is written (votes and matches order no memory) before its entries' places are written again
  int* table = reinterpret_cast<int*>(entries + 4 * (q.K + 1)) + (team << bits);
  const bool twice = repeats(ent, q.K, table, bits, lane);
  write_entries<T, MODE>(r, q, ent, twice, d, lane, [](int) { return true; });
}

// ---------------------------------------------------------------- a CTA or a cluster a row
// W warps compute, one more helps.  The helper keeps the next row on its way
// into shared memory (a bulk copy, begun as soon as the warps have taken the
// present row into their registers), fetches the teacher's pairs a row ahead,
// writes the loss and the entries' places.  The computing warps meet once a
// row.  Two CTAs of 12 warps an SM, three of 8, or six of 4.  (Loading the next row into
// registers instead, as the gradient frees them, took 211 us where a CTA a row
// without any prefetch took 149: the loads hold the scoreboards that the
// exponentials need.)
constexpr int kNv = 12;  // vectors of a thread: 48 registers of logits
template <int W> constexpr int kCtas = 24 / (W + 1);  // CTAs of an SM: 24 warps of 80 registers
template <int W>
struct Bars {
  uint64_t full, taken, written;
  int abort_;
};

template <typename T, int W, int MODE, bool CL>
__global__ void __launch_bounds__(32 * (W + 1), kCtas<W>) k_distill(const __grid_constant__ pnn_distill_args a, int C, int bits, int* gave_up) {
  constexpr int N = 32 * W;              // computing threads
  constexpr int CHUNK = N * kNv;         // vectors of a CTA at a time
  extern __shared__ __align__(16) char raw[];
  uint4* buf = reinterpret_cast<uint4*>(raw);                          // [CHUNK]
  Entry* entries = reinterpret_cast<Entry*>(raw + CHUNK * 16);         // [row parity][K + 1], then the ids' table
  __shared__ float4 stats[2][(CL ? kMaxCluster : 1) * W];
  __shared__ float2 soft_of[2];
  __shared__ Bars<W> bars;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int rank = CL ? (int)cluster_rank() : 0;
  const int64_t step = gridDim.x / C, row0 = blockIdx.x / C;
  const Terms q(a);
  if (tid == 0) {
    tc::mbar_init(tc::smem_u32(&bars.full), 1);
    tc::mbar_init(tc::smem_u32(&bars.taken), W);
    tc::mbar_init(tc::smem_u32(&bars.written), W);
    bars.abort_ = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (CL) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");  // every peer runs
  // A wait that gives up marks the call; the CTA then goes on without waiting (its outputs are wrong, and reported).
  auto wait = [&](uint64_t* bar, uint32_t n) {
    if (tc::mbar_wait(tc::smem_u32(bar), n & 1, &bars.abort_)) return;
    *reinterpret_cast<volatile int*>(&bars.abort_) = 1;
    count_give_up(gave_up);
  };
  // all warps meet with their sums
  auto meet = [&](int par, float m, float t, float h, bool computing) {
    float4* stat = stats[par];
    __syncwarp();
    if (CL) {
      if (computing && lane < C) put_remote(&stat[rank * W + warp], lane, make_float4(m, t, h, 0.f));
      asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
      if (computing && lane == 0) stat[warp] = make_float4(m, t, h, 0.f);
      __syncthreads();
    }
  };
  auto result = [&](int par, int64_t row) {
    const float4* stat = stats[par];
    const int n = (CL ? C : 1) * W;
    float m = -INFINITY, t = 0.f, h = 0.f;
    for (int i = lane; i < n; i += 32) m = fmaxf(m, stat[i].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float b = base_of(m);
    for (int i = lane; i < n; i += 32) {
      const float4 v = stat[i];
      t = fmaf(v.y, rebase(v.x, b, q.kt), t);
      if (MODE != ONE) h = fmaf(v.z, rebase(v.x, b, kLog2e), h);
    }
    return Result<MODE>(a, q, m, warp_sum(t), MODE != ONE ? warp_sum(h) : 0.f, soft_of[par].x, soft_of[par].y,
                        entries[par * (q.K + 1) + q.K].id >= 0, row);
  };
  // a row is one chunk in registers, or several that are loaded again for the gradient
  const int most = (q.V / Span<T>::E + C - 1) / C, chunks = most > CHUNK ? (most + CHUNK - 1) / CHUNK : 1;
  // (for the gradient backwards: the last chunk is still in registers, the others the likelier in L2 the later they came)
  const int loads = a.dlogits ? 2 * chunks - 1 : chunks;  // of a row
  uint32_t n = 0;                                                       // loads so far

  if (warp == W) {
    // -------------------------------------------------------------- the helper
    auto issue = [&](int64_t row, int k) {  // load k of a row
      if (lane != 0) return;
      const Span<T> sp(a.logits, a.logits_stride, q.V, row, rank, C);
      const int c = k < chunks ? k : 2 * chunks - 2 - k, v = sp.nv - c * CHUNK < CHUNK ? sp.nv - c * CHUNK : CHUNK;
      if (v <= 0) {
        tc::mbar_arrive(tc::smem_u32(&bars.full));
        return;
      }
      tc::mbar_expect_tx(tc::smem_u32(&bars.full), v * 16);
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(tc::smem_u32(buf)),
                   "l"(sp.vec() + c * CHUNK), "r"(v * 16), "r"(tc::smem_u32(&bars.full))
                   : "memory");
    };
    auto follow = [&](int64_t row, int k) {  // the load after load k, once that one has been taken
      wait(&bars.taken, n);
      ++n;
      const bool same = k + 1 < loads;
      if ((same || row + step < a.rows) && !*reinterpret_cast<volatile int*>(&bars.abort_)) issue(same ? row : row + step, same ? k + 1 : 0);
    };
    constexpr int PRE = 5;  // entries of a lane that are fetched ahead (128 and the label)
    int id[PRE];
    uint32_t raw_t[PRE];
    float t[PRE], s[PRE];
    bool twice = false, next_twice = false;
    auto fetch = [&](int64_t row) {
#pragma unroll
      for (int i = 0; i < PRE; ++i) q.raw(a, row, lane + 32 * i, id[i], raw_t[i]);
    };
    auto gather = [&](int64_t row) {
      const T* p = static_cast<const T*>(a.logits) + row * a.logits_stride;
#pragma unroll
      for (int i = 0; i < PRE; ++i) {
        q.read(a, lane + 32 * i, raw_t[i], id[i], t[i]);
        s[i] = id[i] >= 0 ? ld(p + id[i]) : 0.f;
      }
    };
    auto lay_out = [&](int64_t row, int par) {
      Entry* ent = entries + par * (q.K + 1);
      const T* p = static_cast<const T*>(a.logits) + row * a.logits_stride;
      float mt = -INFINITY;
#pragma unroll
      for (int i = 0; i < PRE; ++i) {
        if (lane + 32 * i <= q.K) ent[lane + 32 * i] = Entry{id[i], t[i], s[i]};
        mt = fmaxf(mt, t[i]);
      }
      for (int j = lane + 32 * PRE; j <= q.K; j += 32) {
        Entry e;
        q.entry(a, row, j, e.id, e.t);
        e.s = e.id >= 0 ? ld(p + e.id) : 0.f;
        ent[j] = e;
        mt = fmaxf(mt, e.t);
      }
#pragma unroll
      for (int o = 16; o; o >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, o));
      if (mt == -INFINITY) mt = 0.f;
      float w = 0.f;
#pragma unroll
      for (int i = 0; i < PRE; ++i) w += ex2((t[i] - mt) * q.kt);
      for (int j = lane + 32 * PRE; j < q.K; j += 32) w += ex2((ent[j].t - mt) * q.kt);
      w = warp_sum(w);
      if (lane == 0) soft_of[par] = make_float2(mt, w);
      __syncwarp();
      if (a.dlogits) next_twice = repeats(ent, q.K, reinterpret_cast<int*>(entries + 2 * (q.K + 1)), bits, lane);
    };
    issue(row0, 0);
    fetch(row0);
    gather(row0);
    lay_out(row0, 0);
    twice = next_twice;
    int par = 0;
    uint32_t rows = 0;
    for (int64_t row = row0; row < a.rows; row += step, par ^= 1, ++rows) {
      for (int k = 0; k < chunks; ++k) follow(row, k);
      const bool more = row + step < a.rows;
      if (more) fetch(row + step);
      meet(par, 0.f, 0.f, 0.f, false);
      const Result<MODE> r = result(par, row);
      const Entry* ent = entries + par * (q.K + 1);
      if (rank == 0) r.loss(a, q, ent, row, lane);
      if (more) {  // (all but the places themselves before the row is written: the warps' next meeting waits for the helper)
        gather(row + step);
        lay_out(row + step, par ^ 1);
      }
      if (a.dlogits) {
        for (int k = chunks; k < loads; ++k) follow(row, k);
        wait(&bars.written, rows);
        if (r.soft || r.hard) {
          const Span<T> sp(a.logits, a.logits_stride, q.V, row, rank, C);
          T* d = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
          write_entries<T, MODE>(r, q, ent, twice, d, lane, [&](int id) {  // in a cluster each place by the CTA that wrote it
            const int p = id - sp.head;
            return !CL || (p < 0 || p >= sp.all * Span<T>::E ? 0 : p / Span<T>::E / sp.each) == rank;
          });
        }
      }
      twice = next_twice;
    }
    if (*reinterpret_cast<volatile int*>(&bars.abort_) && lane == 0) tc::mbar_wait_drain(tc::smem_u32(&bars.full), n & 1);
  } else {
    // -------------------------------------------------------------- the computing warps
    int par = 0;
    uint4 x[kNv];
    auto take = [&](int v) {  // the buffer's v vectors
      wait(&bars.full, n);
      ++n;
#pragma unroll
      for (int i = 0; i < kNv; ++i) x[i] = i * N + tid < v ? buf[i * N + tid] : minus_inf<T>();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tc::smem_u32(&bars.taken));
    };
    for (int64_t row = row0; row < a.rows; row += step, par ^= 1) {
      const Span<T> sp(a.logits, a.logits_stride, q.V, row, rank, C);
      const int lone = sp.lone(q.V, rank, tid);
      const float one = lone >= 0 ? ld(sp.s + lone) : -INFINITY;
      float m = -INFINITY, t = 0.f, h = 0.f;
      for (int c = 0; c < chunks; ++c) {
        const int v = sp.nv - c * CHUNK;
        take(v);
        const float mc = warp_max<T>(x, c ? m : one);  // (not below what came before)
        const float b = base_of(mc);
        float tc_, hc;
        sums<T, MODE>(x, (v + N - 1) / N, b, q.kt, tc_, hc);
        if (c == 0 && lone >= 0) {
          const float e = ex2((one - b) * q.kt);
          tc_ += e;
          if (MODE != ONE) hc += second1<MODE>(one - b, e);
        }
        if (c) {
          t = fmaf(t, rebase(m, b, q.kt), tc_);
          if (MODE != ONE) h = fmaf(h, rebase(m, b, kLog2e), hc);
        } else {
          t = tc_;
          h = hc;
        }
        m = mc;
      }
      t = warp_sum(t);
      if (MODE != ONE) h = warp_sum(h);
      meet(par, m, t, h, true);
      if (!a.dlogits) continue;
      const Result<MODE> r = result(par, row);
      T* d = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
      const bool same = ((reinterpret_cast<uintptr_t>(d) ^ reinterpret_cast<uintptr_t>(sp.s)) & 15) == 0, some = r.soft || r.hard;
      for (int c = chunks - 1; c >= 0; --c) {
        const int v = sp.nv - c * CHUNK;
        if (c < chunks - 1) take(v);
        T* to = d + sp.head + (int64_t)(sp.v0 + c * CHUNK + tid) * Span<T>::E;
        if (some) {
#pragma unroll
          for (int i = 0; i < kNv; ++i)
            if (i * N + tid < v) put<T>(to + i * N * Span<T>::E, grads<T, MODE>(x[i], r), same);
        } else {
          for (int i = tid; i < v && i < CHUNK; i += N) put<T>(to + (i - tid) * Span<T>::E, make_uint4(0, 0, 0, 0), same);
        }
      }
      if (lone >= 0) ::pnn::seq::st(d + lone, r.grad(one));
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tc::smem_u32(&bars.written));
    }
  }
  __syncwarp();
  if (CL) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// ---------------------------------------------------------------- the loss alone
// Nothing is kept of a row, so that its vectors need not wait for one another:
// each of 8 warps walks over its share, 4 vectors a thread on their way while 4
// are added up, and four CTAs an SM fill one another's gaps.  2048 x 50001 bf16
// take 42 us (4.9 TB/s, 48 by the kernel above), 4096 x 32000 51 (56), 16384 x
// 12000 103 (117); rows of 5000 take 60 us above and 79 here, a CTA's beginning
// and end being most of them.
template <typename T, int MODE>
__global__ void __launch_bounds__(256, 4) k_distill_loss(const __grid_constant__ pnn_distill_args a) {
  extern __shared__ Entry entries[];  // [K + 1]
  __shared__ float4 stats[8];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t row = blockIdx.x;
  const Terms q(a);
  const Span<T> sp(a.logits, a.logits_stride, q.V, row, 0, 1);
  const uint4* vec = sp.vec();
  const int lone = sp.lone(q.V, 0, tid);
  const float one = lone >= 0 ? ld(sp.s + lone) : -INFINITY;
  float m = -INFINITY, t = 0.f, h = 0.f, mt = -INFINITY;
  constexpr int U = kWarpVecs / 2, STEP = 256 * U;  // vectors of a batch
  auto load = [&](uint4 (&x)[U], int v0) {
#pragma unroll
    for (int i = 0; i < U; ++i) x[i] = v0 + i * 256 + tid < sp.nv ? ld_once(vec + v0 + i * 256 + tid) : minus_inf<T>();
  };
  auto add = [&](const uint4 (&x)[U], int v0) {
    const float mc = warp_max<T>(x, v0 ? m : one), b = base_of(mc);  // (not below what came before)
    float tc_, hc;
    sums<T, MODE>(x, (sp.nv - v0 + 255) / 256, b, q.kt, tc_, hc);
    t = fmaf(t, rebase(m, b, q.kt), tc_);
    if (MODE != ONE) h = fmaf(h, rebase(m, b, kLog2e), hc);
    m = mc;
  };
  uint4 x[U], y[U];
  load(x, 0);
  load(y, STEP);
  if (warp == 0) {
    for (int j = lane; j <= q.K; j += 32) {
      Entry e;
      q.entry(a, row, j, e.id, e.t);
      e.s = e.id >= 0 ? ld(sp.s + e.id) : 0.f;
      entries[j] = e;
      mt = fmaxf(mt, e.t);
    }
  }
  for (int v0 = 0; v0 < sp.nv || v0 == 0; v0 += 2 * STEP) {
    add(x, v0);
    load(x, v0 + 2 * STEP);
    if (v0 + STEP >= sp.nv) break;
    add(y, v0 + STEP);
    load(y, v0 + 3 * STEP);
  }
  if (lone >= 0) {
    const float b = base_of(m), e = ex2((one - b) * q.kt);
    t += e;
    if (MODE != ONE) h += second1<MODE>(one - b, e);
  }
  t = warp_sum(t);
  if (MODE != ONE) h = warp_sum(h);
  if (lane == 0) stats[warp] = make_float4(m, t, h, 0.f);
  __syncthreads();
  if (warp) return;
#pragma unroll
  for (int o = 16; o; o >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, o));
  if (mt == -INFINITY) mt = 0.f;
  float w = 0.f;
  for (int j = lane; j < q.K; j += 32) w += ex2((entries[j].t - mt) * q.kt);
  const float4 v = lane < 8 ? stats[lane] : make_float4(-INFINITY, 0.f, 0.f, 0.f);
  m = v.x;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  const float b = base_of(m);
  t = warp_sum(v.y * rebase(v.x, b, q.kt));
  h = MODE != ONE ? warp_sum(v.z * rebase(v.x, b, kLog2e)) : 0.f;
  const Result<MODE> r(a, q, m, t, h, mt, warp_sum(w), entries[q.K].id >= 0, row);
  r.loss(a, q, entries, row, lane);
}

template <typename T, int W, int MODE, bool CL>
cudaError_t launch(const pnn_distill_args& a, int C, cudaStream_t st) {
  const auto kernel = k_distill<T, W, MODE, CL>;
  const int bits = table_bits(a.k), smem = 32 * W * kNv * 16 + 2 * (a.k + 1) * (int)sizeof(Entry) + (4 << bits);
  // the limit of 48 KB without this also counts the kernel's own static memory
  static std::atomic<uint64_t> ready{0};  // one bit a device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(ready.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 32 * W * kNv * 16 + 2 * 1025 * (int)sizeof(Entry) + (4 << table_bits(1024)));
    if (e != cudaSuccess) return e;
    ready.fetch_or(bit, std::memory_order_release);
  }
  int* word = seq_gave_up_word();
  if (!word) return cudaGetLastError();
  cudaLaunchConfig_t cfg = {};
  const int64_t fit = (int64_t)device_sm_count() * kCtas<W> / C;  // teams that run at once
  cfg.gridDim = dim3((unsigned)((a.rows < fit ? a.rows : fit > 0 ? fit : 1) * C));
  cfg.blockDim = dim3(32 * (W + 1));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeClusterDimension;
  at[0].val.clusterDim.x = C;
  at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
  cfg.attrs = at;
  cfg.numAttrs = C > 1 ? 1 : 0;
  return cudaLaunchKernelEx(&cfg, kernel, a, C, bits, word);
}

// The smallest team whose registers hold the row: a warp (2048 bf16 values), a
// CTA of 3, 7 or 11 computing warps (9216, 21504, 33792); see below for longer
// ones, and above for rows of more than 9216 whose loss alone is wanted.
template <typename T, int MODE>
cudaError_t pick(const pnn_distill_args& a, cudaStream_t st) {
  constexpr int64_t E = 16 / sizeof(T);
  const int64_t n = a.vocab;
  if (n <= 32 * kWarpVecs * E && a.k < 512) {
    const int bits = table_bits(a.k);
    k_distill_warp<T, MODE><<<(unsigned)((a.rows + 3) / 4), 128, 4 * ((a.k + 1) * sizeof(Entry) + (4 << bits)), st>>>(a, bits);
    return cudaGetLastError();
  }
  if (n <= 3 * 32 * kNv * E) return launch<T, 3, MODE, false>(a, 1, st);
  if (a.dlogits && n <= 7 * 32 * kNv * E) return launch<T, 7, MODE, false>(a, 1, st);
  // Rows longer than one CTA's registers: few of them are shared by clusters, many are read twice by one CTA each, the
  // second time from L2 (304 rows of 256 KB are 78 MB there), since a cluster's meeting stops all of its CTAs: 4096 x
  // 128003 bf16 took 1009 us in clusters of 4.
  int C = 1;
  while (C < kMaxCluster && C * 11 * 32 * kNv * E < n && a.rows * C <= device_sm_count()) C *= 2;
  if (C > 1) return launch<T, 11, MODE, true>(a, C, st);
  if (a.dlogits) return launch<T, 11, MODE, false>(a, 1, st);
  k_distill_loss<T, MODE><<<(unsigned)a.rows, 256, (a.k + 1) * sizeof(Entry), st>>>(a);
  return cudaGetLastError();
}
template <typename T>
cudaError_t mode(const pnn_distill_args& a, cudaStream_t st) {
  const bool both = a.k > 0 && a.alpha > 0.f && a.labels && a.alpha < 1.f;
  if (!both || a.tau == 1.f) return pick<T, ONE>(a, st);
  if (a.tau == 2.f) return pick<T, SQUARE>(a, st);
  return a.tau == 4.f ? pick<T, FOURTH>(a, st) : pick<T, TWO>(a, st);
}
}  // namespace

cudaError_t launch_distill(const pnn_distill_args& a, cudaStream_t st) {
  return a.dtype == PNN_DT_BF16 ? mode<bf16>(a, st) : mode<float>(a, st);
}

}  // namespace pnn
