// Clipped policy loss with a KL term: loss, log-probabilities and gradient in
// one pass over the logits.
//
// A row's gradient is slope / tau (e_label - softmax(s / tau)): all of its places
// take a number that is known once the row's sum is, so the row is read into
// registers (or, longer than a CTA's, read a second time out of L2), its sum
// formed warp by warp, each from its own maximum, and the gradient written from
// the registers; the label's place is written again after that.  The teams are
// the distillation's: a warp, a CTA whose spare warp keeps the next row on its
// way, or a cluster of CTAs.
//
// lp = (s_label - m) / tau - log(sum): the difference first, so that it is exact
// to one rounding however large the logits are.
//
// Bound: HBM.  4096 x 32000 bf16 take 88 us (524 MB, 6.0 TB/s), 4096 x 128003 394 (2.5
// GB moved, 6.4 TB/s: a fifth of each row comes twice from DRAM), the loss alone of 2048
// x 50001 41; 256 x 1000 fp32 6.
#include <math.h>

#include <atomic>

#include "pnn_internal.h"
#include "pnn_seq.h"
#include "row_logits.cuh"
#include "tc_ptx.cuh"

namespace pnn {
namespace {
using namespace seq;

// What a row's loss needs beside its logits.
struct Sample {
  int label;  // -1: none
  float s, adv, old, ref, weight;
};
__device__ __forceinline__ Sample sample_of(const pnn_policy_args& a, int64_t row) {
  Sample q;
  q.label = a.labels[row];
  q.adv = a.advantage[row];
  q.old = a.old ? a.old[row] : 0.f;
  q.ref = a.ref ? a.ref[row] : 0.f;
  q.weight = a.weight ? a.weight[row] : 1.f;
  if (q.label < 0 || q.label >= a.vocab) q.label = -1;
  q.s = 0.f;
  return q;
}
template <typename T>
__device__ __forceinline__ void see(const pnn_policy_args& a, int64_t row, Sample& q) {
  if (q.label >= 0) q.s = ld(static_cast<const T*>(a.logits) + row * a.logits_stride + q.label);
}

// A row's result: the gradient is at * [label] - g exp((s - b) / tau).
struct Result {
  float b, g, at, loss, lp;
  bool live;
  __device__ __forceinline__ Result(const pnn_policy_args& a, const Sample& q, float m, float sum) {
    b = base_of(m);
    live = q.label >= 0 && q.s != -INFINITY;
    lp = q.label < 0 ? 0.f : -INFINITY;
    loss = g = at = 0.f;
    if (!live) return;
    lp = __fdiv_rn(q.s - b, a.tau) - logf(sum);
    const float r = a.old ? expf(lp - q.old) : 1.f;
    // -min(r A, clamp(r) A): the bound that holds is the upper one for A > 0, the lower one for A < 0
    float slope = 0.f;
    if (q.adv > 0.f) {
      const float hi = 1.f + a.clip_high;
      loss = -q.adv * fminf(r, hi);
      if (r <= hi) slope = -q.adv * r;
    } else if (q.adv < 0.f) {
      const float lo = 1.f - a.clip_low;
      loss = -q.adv * fmaxf(r, lo);
      if (r >= lo) slope = -q.adv * r;
    } else {
      loss = slope = q.adv;  // 0 (NaN stays)
    }
    if (r != r) loss = slope = r;
    if (a.ref && a.beta != 0.f) {
      const float u = q.ref - lp, e = expm1f(u);
      loss = fmaf(a.beta, e - u, loss);
      slope = fmaf(-a.beta, e, slope);
    }
    at = __fdiv_rn(slope * q.weight, a.tau);
    g = at / sum;
  }
  __device__ __forceinline__ void tell(const pnn_policy_args& a, int64_t row) const {
    a.loss[row] = loss;
    if (a.logp) a.logp[row] = lp;
  }
};
// the gradient of one logit
__device__ __forceinline__ float grad(const Result& r, float k, float s) { return r.live ? -r.g * ex2((s - r.b) * k) : 0.f; }
__device__ __forceinline__ float grad_label(const Result& r, float k, float s) { return fmaf(-r.g, ex2((s - r.b) * k), r.at); }

// The sum of a thread's vectors from the base b.
template <typename T, int NV>
__device__ __forceinline__ float sum_of(const uint4 (&x)[NV], int used, float b, float k) {
  const f2 k2 = pk(k, k), nb = pk(-b, -b);
  f2 at = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i)
    if (i < used) {
#pragma unroll
      for (int p = 0; p < kPairs<T>; ++p) at = add2(at, ex2p(mul2(add2(pair_of<T>(x[i], p), nb), k2)));
    }
  float u, v;
  upk(at, u, v);
  return u + v;
}
template <typename T>
__device__ __forceinline__ uint4 grads(const uint4& x, const Result& r, float k) {
  const f2 k2 = pk(k, k), nb = pk(-r.b, -r.b), g2 = pk(-r.g, -r.g);
  uint4 o;
  uint32_t* w = reinterpret_cast<uint32_t*>(&o);
#pragma unroll
  for (int p = 0; p < kPairs<T>; ++p) {
    const f2 g = mul2(g2, ex2p(mul2(add2(pair_of<T>(x, p), nb), k2)));
    float u, v;
    upk(g, u, v);
    if constexpr (sizeof(T) == 2) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(u, v);
      w[p] = *reinterpret_cast<const uint32_t*>(&h);
    } else {
      w[2 * p] = __float_as_uint(u);
      w[2 * p + 1] = __float_as_uint(v);
    }
  }
  return o;
}

// ---------------------------------------------------------------- a warp a row
constexpr int kWarpVecs = 8;
template <typename T>
__global__ void __launch_bounds__(128) k_policy_warp(const __grid_constant__ pnn_policy_args a, float k) {
  const int lane = threadIdx.x & 31;
  const int64_t row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= a.rows) return;
  const Span<T> sp(a.logits, a.logits_stride, (int)a.vocab, row, 0, 1);
  uint4 x[kWarpVecs];
#pragma unroll
  for (int i = 0; i < kWarpVecs; ++i) x[i] = i * 32 + lane < sp.nv ? ld_once(sp.vec() + i * 32 + lane) : minus_inf<T>();
  Sample q = sample_of(a, row);
  const int lone = sp.lone((int)a.vocab, 0, lane);
  const float one = lone >= 0 ? ld(sp.s + lone) : -INFINITY;
  see<T>(a, row, q);
  const float m = warp_max<T>(x, one), b = base_of(m);
  float t = sum_of<T>(x, (sp.nv + 31) / 32, b, k);
  if (lone >= 0) t += ex2((one - b) * k);
  const Result r(a, q, m, warp_sum(t));
  if (lane == 0) r.tell(a, row);
  if (!a.dlogits) return;
  T* d = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
  const bool same = ((reinterpret_cast<uintptr_t>(d) ^ reinterpret_cast<uintptr_t>(sp.s)) & 15) == 0;
#pragma unroll
  for (int i = 0; i < kWarpVecs; ++i)
    if (i * 32 + lane < sp.nv) put<T>(d + sp.head + (i * 32 + lane) * Span<T>::E, r.live ? grads<T>(x[i], r, k) : make_uint4(0, 0, 0, 0), same);
  if (lone >= 0) st(d + lone, grad(r, k, one));
  if (!r.live) return;
  __syncwarp();  // the row is written before the label's place is written again
  if (lane == 0) st(d + q.label, grad_label(r, k, q.s));
}

// ---------------------------------------------------------------- a CTA or a cluster a row
// W warps compute; one more keeps the next row on its way into shared memory (a
// bulk copy, begun as soon as the warps have taken the present row into their
// registers), fetches the next row's sample, writes the loss and the label's place.
constexpr int kNv = 12;  // vectors of a thread: 48 registers of logits
template <int W> constexpr int kCtas = 24 / (W + 1);  // CTAs of an SM: 24 warps of 80 registers

template <typename T, int W, bool CL>
__global__ void __launch_bounds__(32 * (W + 1), kCtas<W>) k_policy(const __grid_constant__ pnn_policy_args a, float k, int C, int* gave_up) {
  constexpr int N = 32 * W;              // computing threads
  constexpr int CHUNK = N * kNv;         // vectors of a CTA at a time
  extern __shared__ __align__(16) char raw[];
  uint4* buf = reinterpret_cast<uint4*>(raw);  // [CHUNK]
  __shared__ float4 stats[2][(CL ? kMaxCluster : 1) * W];
  __shared__ Sample samples[2];
  __shared__ uint64_t full, taken, written;
  __shared__ int abort_;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, V = (int)a.vocab;
  const int rank = CL ? (int)cluster_rank() : 0;
  const int64_t step = gridDim.x / C, row0 = blockIdx.x / C;
  if (tid == 0) {
    tc::mbar_init(tc::smem_u32(&full), 1);
    tc::mbar_init(tc::smem_u32(&taken), W);
    tc::mbar_init(tc::smem_u32(&written), W);
    abort_ = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncthreads();
  if (CL) asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");  // every peer runs
  // A wait that gives up marks the call; the CTA then goes on without waiting (its outputs are wrong, and reported).
  auto wait = [&](uint64_t* bar, uint32_t n) {
    if (tc::mbar_wait(tc::smem_u32(bar), n & 1, &abort_)) return;
    *reinterpret_cast<volatile int*>(&abort_) = 1;
    count_give_up(gave_up);
  };
  auto meet = [&](int par, float m, float t, bool computing) {  // all warps, with their sums
    float4* stat = stats[par];
    __syncwarp();
    if (CL) {
      if (computing && lane < C) put_remote(&stat[rank * W + warp], lane, make_float4(m, t, 0.f, 0.f));
      asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
    } else {
      if (computing && lane == 0) stat[warp] = make_float4(m, t, 0.f, 0.f);
      __syncthreads();
    }
  };
  auto result = [&](int par) {
    const float4* stat = stats[par];
    const int n = (CL ? C : 1) * W;
    float m = -INFINITY, t = 0.f;
    for (int i = lane; i < n; i += 32) m = fmaxf(m, stat[i].x);
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float b = base_of(m);
    for (int i = lane; i < n; i += 32) t = fmaf(stat[i].y, rebase(stat[i].x, b, k), t);
    return Result(a, samples[par], m, warp_sum(t));
  };
  // a row is one chunk in registers, or several that are loaded again for the gradient
  const int most = (V / Span<T>::E + C - 1) / C, chunks = most > CHUNK ? (most + CHUNK - 1) / CHUNK : 1;
  // (for the gradient backwards: the last chunk is still in registers, the others the likelier in L2 the later they came)
  const int loads = a.dlogits ? 2 * chunks - 1 : chunks;  // of a row
  uint32_t n = 0;                                         // loads so far

  if (warp == W) {
    // -------------------------------------------------------------- the helper
    auto issue = [&](int64_t row, int i) {  // load i of a row
      if (lane != 0) return;
      const Span<T> sp(a.logits, a.logits_stride, V, row, rank, C);
      const int c = i < chunks ? i : 2 * chunks - 2 - i, v = sp.nv - c * CHUNK < CHUNK ? sp.nv - c * CHUNK : CHUNK;
      if (v <= 0) {
        tc::mbar_arrive(tc::smem_u32(&full));
        return;
      }
      tc::mbar_expect_tx(tc::smem_u32(&full), v * 16);
      asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(tc::smem_u32(buf)),
                   "l"(sp.vec() + c * CHUNK), "r"(v * 16), "r"(tc::smem_u32(&full))
                   : "memory");
    };
    auto follow = [&](int64_t row, int i) {  // the load after load i, once that one has been taken
      wait(&taken, n);
      ++n;
      const bool same = i + 1 < loads;
      if ((same || row + step < a.rows) && !*reinterpret_cast<volatile int*>(&abort_)) issue(same ? row : row + step, same ? i + 1 : 0);
    };
    issue(row0, 0);
    Sample q = sample_of(a, row0);
    see<T>(a, row0, q);
    if (lane == 0) samples[0] = q;
    int par = 0;
    uint32_t rows = 0;
    for (int64_t row = row0; row < a.rows; row += step, par ^= 1, ++rows) {
      const bool more = row + step < a.rows;
      if (more) q = sample_of(a, row + step);
      for (int i = 0; i < chunks; ++i) follow(row, i);
      if (more) see<T>(a, row + step, q);
      meet(par, 0.f, 0.f, false);
      const Result r = result(par);
      const int label = samples[par].label;
      const float s = samples[par].s;
      if (rank == 0 && lane == 0) r.tell(a, row);
      if (more && lane == 0) samples[par ^ 1] = q;  // (seen by the warps behind the next meeting)
      if (a.dlogits) {
        for (int i = chunks; i < loads; ++i) follow(row, i);
        wait(&written, rows);
        if (r.live && lane == 0) {
          const Span<T> sp(a.logits, a.logits_stride, V, row, rank, C);
          const int p = label - sp.head;  // in a cluster the place is written by the CTA that wrote it
          if (!CL || (p < 0 || p >= sp.all * Span<T>::E ? 0 : p / Span<T>::E / sp.each) == rank)
            st(static_cast<T*>(a.dlogits) + row * a.dlogits_stride + label, grad_label(r, k, s));
        }
        __syncwarp();
      }
    }
    if (*reinterpret_cast<volatile int*>(&abort_) && lane == 0) tc::mbar_wait_drain(tc::smem_u32(&full), n & 1);
  } else {
    // -------------------------------------------------------------- the computing warps
    int par = 0;
    uint4 x[kNv];
    auto take = [&](int v) {  // the buffer's v vectors
      wait(&full, n);
      ++n;
#pragma unroll
      for (int i = 0; i < kNv; ++i) x[i] = i * N + tid < v ? buf[i * N + tid] : minus_inf<T>();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tc::smem_u32(&taken));
    };
    for (int64_t row = row0; row < a.rows; row += step, par ^= 1) {
      const Span<T> sp(a.logits, a.logits_stride, V, row, rank, C);
      const int lone = sp.lone(V, rank, tid);
      const float one = lone >= 0 ? ld(sp.s + lone) : -INFINITY;
      float m = -INFINITY, t = 0.f;
      for (int c = 0; c < chunks; ++c) {
        const int v = sp.nv - c * CHUNK;
        take(v);
        const float mc = warp_max<T>(x, c ? m : one), b = base_of(mc);  // (not below what came before)
        float s = sum_of<T>(x, (v + N - 1) / N, b, k);
        if (c == 0 && lone >= 0) s += ex2((one - b) * k);
        t = c ? fmaf(t, rebase(m, b, k), s) : s;
        m = mc;
      }
      t = warp_sum(t);
      meet(par, m, t, true);
      if (!a.dlogits) continue;
      const Result r = result(par);
      T* d = static_cast<T*>(a.dlogits) + row * a.dlogits_stride;
      const bool same = ((reinterpret_cast<uintptr_t>(d) ^ reinterpret_cast<uintptr_t>(sp.s)) & 15) == 0;
      for (int c = chunks - 1; c >= 0; --c) {
        const int v = sp.nv - c * CHUNK;
        if (c < chunks - 1) take(v);
        T* to = d + sp.head + (int64_t)(sp.v0 + c * CHUNK + tid) * Span<T>::E;
        if (r.live) {
#pragma unroll
          for (int i = 0; i < kNv; ++i)
            if (i * N + tid < v) put<T>(to + i * N * Span<T>::E, grads<T>(x[i], r, k), same);
        } else {
          for (int i = tid; i < v && i < CHUNK; i += N) put<T>(to + (i - tid) * Span<T>::E, make_uint4(0, 0, 0, 0), same);
        }
      }
      if (lone >= 0) st(d + lone, grad(r, k, one));
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(tc::smem_u32(&written));
    }
  }
  __syncwarp();
  if (CL) asm volatile("barrier.cluster.arrive.aligned;\n\tbarrier.cluster.wait.aligned;" ::: "memory");
}

// ---------------------------------------------------------------- the loss alone
// Nothing is kept of a row: each of 8 warps walks over its share, 4 vectors a
// thread on their way while 4 are added up, four CTAs an SM.
template <typename T>
__global__ void __launch_bounds__(256, 4) k_policy_loss(const __grid_constant__ pnn_policy_args a, float k) {
  __shared__ float2 stats[8];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int64_t row = blockIdx.x;
  const Span<T> sp(a.logits, a.logits_stride, (int)a.vocab, row, 0, 1);
  const uint4* vec = sp.vec();
  const int lone = sp.lone((int)a.vocab, 0, tid);
  const float one = lone >= 0 ? ld(sp.s + lone) : -INFINITY;
  float m = -INFINITY, t = 0.f;
  constexpr int U = kWarpVecs / 2, STEP = 256 * U;  // vectors of a batch
  auto load = [&](uint4 (&x)[U], int v0) {
#pragma unroll
    for (int i = 0; i < U; ++i) x[i] = v0 + i * 256 + tid < sp.nv ? ld_once(vec + v0 + i * 256 + tid) : minus_inf<T>();
  };
  auto add = [&](const uint4 (&x)[U], int v0) {
    const float mc = warp_max<T>(x, v0 ? m : one), b = base_of(mc);  // (not below what came before)
    t = fmaf(t, rebase(m, b, k), sum_of<T>(x, (sp.nv - v0 + 255) / 256, b, k));
    m = mc;
  };
  uint4 x[U], y[U];
  load(x, 0);
  load(y, STEP);
  Sample q;
  if (warp == 0) {
    q = sample_of(a, row);
    see<T>(a, row, q);
  }
  for (int v0 = 0; v0 < sp.nv || v0 == 0; v0 += 2 * STEP) {
    add(x, v0);
    load(x, v0 + 2 * STEP);
    if (v0 + STEP >= sp.nv) break;
    add(y, v0 + STEP);
    load(y, v0 + 3 * STEP);
  }
  if (lone >= 0) t += ex2((one - base_of(m)) * k);
  t = warp_sum(t);
  if (lane == 0) stats[warp] = make_float2(m, t);
  __syncthreads();
  if (warp) return;
  const float2 v = lane < 8 ? stats[lane] : make_float2(-INFINITY, 0.f);
  m = v.x;
#pragma unroll
  for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
  t = warp_sum(v.y * rebase(v.x, base_of(m), k));
  if (lane == 0) Result(a, q, m, t).tell(a, row);
}

template <typename T, int W, bool CL>
cudaError_t launch(const pnn_policy_args& a, float k, int C, cudaStream_t st) {
  const auto kernel = k_policy<T, W, CL>;
  constexpr int smem = 32 * W * kNv * 16;
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
  return cudaLaunchKernelEx(&cfg, kernel, a, k, C, word);
}

// The smallest team whose registers hold the row, as in the distillation: a warp
// (2048 bf16 values), a CTA of 3, 7 or 11 computing warps (9216, 21504, 33792);
// longer rows in clusters while there are few of them, else read twice.
template <typename T>
cudaError_t pick(const pnn_policy_args& a, cudaStream_t st) {
  constexpr int64_t E = 16 / sizeof(T);
  const int64_t n = a.vocab;
  const float k = kLog2e / a.tau;
  if (n <= 32 * kWarpVecs * E) {
    k_policy_warp<T><<<(unsigned)((a.rows + 3) / 4), 128, 0, st>>>(a, k);
    return cudaGetLastError();
  }
  if (n <= 3 * 32 * kNv * E) return launch<T, 3, false>(a, k, 1, st);
  if (a.dlogits && n <= 7 * 32 * kNv * E) return launch<T, 7, false>(a, k, 1, st);
  int C = 1;
  while (C < kMaxCluster && C * 11 * 32 * kNv * E < n && a.rows * C <= device_sm_count()) C *= 2;
  if (C > 1) return launch<T, 11, true>(a, k, C, st);
  if (a.dlogits) return launch<T, 11, false>(a, k, 1, st);
  k_policy_loss<T><<<(unsigned)a.rows, 256, 0, st>>>(a, k);
  return cudaGetLastError();
}
}  // namespace

cudaError_t launch_policy(const pnn_policy_args& a, cudaStream_t st) {
  return a.dtype == PNN_DT_BF16 ? pick<seq::bf16>(a, st) : pick<float>(a, st);
}

}  // namespace pnn
