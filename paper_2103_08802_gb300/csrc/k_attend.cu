// Linear attention with a decay for each head: passes of any widths, strides
// and types; joining the segments of long sequences; one token on a pool of
// states.  attend.cuh has the mathematics.
#include <cuda_runtime.h>

#include <atomic>

#include "attend.cuh"
#include "pnn_internal.h"

namespace pnn {
namespace attend {
namespace {
using namespace seq;

// ---------------------------------------------------------------- passes of any shape
// A CTA owns 64 columns of a head's state (columns of z do not meet) and walks
// over its segment in chunks of 32 tokens, everything in shared memory as fp32.
// Products run on the tensor cores in tf32, each fp32 operand as the sum of two
// tf32 numbers (x = hi + lo to 2^-22; three products, lo lo left out), the large
// product and the two small ones in accumulators of their own: the adder cuts
// off what is below its sum's last place, which would add up over a long state.
// For the same reason a chunk's product starts from zero and is added to the
// state by an ordinary rounded sum.
constexpr int C = 32, BZ = 64, LDZ = BZ + 8, LDP = C + 4, NT = 256;

__device__ __forceinline__ uint32_t tf32(float x) {
  uint32_t r;
  asm("cvt.rna.tf32.f32 %0, %1;" : "=r"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], const uint32_t (&b)[2]) {
  asm("mma.sync.aligned.m16n8k8.row.col.f32.tf32.tf32.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b[0]), "r"(b[1]));
}
// c = A (16 x K) B (K x 8 N): a(m, k) and b(k, n) read one element; K a multiple of 8
template <int N, typename FA, typename FB>
__device__ __forceinline__ void tile(float (&c)[N][4], int K, FA a, FB b) {
  const int g = (threadIdx.x & 31) >> 2, t = threadIdx.x & 3;
  float small[N][4];
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) c[u][i] = small[u][i] = 0.f;
#pragma unroll 2
  for (int k = 0; k < K; k += 8) {
    const float av[4] = {a(g, k + t), a(g + 8, k + t), a(g, k + t + 4), a(g + 8, k + t + 4)};
    uint32_t ah[4], al[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ah[i] = tf32(av[i]);
      al[i] = tf32(av[i] - __uint_as_float(ah[i]));
    }
#pragma unroll
    for (int u = 0; u < N; ++u) {
      const float bv[2] = {b(k + t, 8 * u + g), b(k + t + 4, 8 * u + g)};
      uint32_t bh[2], bl[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        bh[i] = tf32(bv[i]);
        bl[i] = tf32(bv[i] - __uint_as_float(bh[i]));
      }
      mma(small[u], al, bh);
      mma(small[u], ah, bl);
      mma(c[u], ah, bh);
    }
  }
#pragma unroll
  for (int u = 0; u < N; ++u)
#pragma unroll
    for (int i = 0; i < 4; ++i) c[u][i] += small[u][i];
}
// Rows of a chunk on their way in registers: warp w has rows w, w + 8, w + 16, w + 24, a lane every 32nd column.
template <typename T, int COLS>
struct Ahead {
  float v[4][COLS];
  __device__ __forceinline__ void load(const T* p, int64_t stride, int n, int width) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < COLS; ++j) {
        const int r = warp + 8 * i, d = lane + 32 * j;
        v[i][j] = r < n && d < width ? seq::ld(p + r * stride + d) : 0.f;
      }
  }
  // row r times f(r)
  template <typename F>
  __device__ __forceinline__ void put(float* to, int ld, int most, F f) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = f(warp + 8 * i);
#pragma unroll
      for (int j = 0; j < COLS; ++j)
        if (lane + 32 * j < most) to[(warp + 8 * i) * ld + lane + 32 * j] = v[i][j] * x;
    }
  }
};

__host__ __device__ constexpr int round_up(int a, int b) { return (a + b - 1) / b * b; }
__host__ __device__ constexpr int ld_of(int dx) { return round_up(dx, 32) + 4; }
__host__ constexpr int any_smem(int dx) { return (3 * C * ld_of(dx) + C * LDZ + C * LDP + round_up(dx, 16) * LDZ) * 4; }

// NX: columns of x and y, in units of 32
template <typename T, int NX, bool SUM>
__global__ void __launch_bounds__(NT, NX <= 4 ? 2 : 1) k_attend_any(const __grid_constant__ Work w) {
  extern __shared__ float smem[];
  __shared__ float pw[C + 1];
  const Pass& ps = w.pass[blockIdx.z];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int dx = ps.dx, dz = ps.dz, zblocks = (dz + BZ - 1) / BZ;
  const int zb = blockIdx.y % zblocks, sg = blockIdx.y / zblocks;
  if (sg >= w.segments) return;  // (another pass has more columns)
  const int z0 = zb * BZ, nz = dz - z0 < BZ ? dz - z0 : BZ;
  const int b = blockIdx.x / w.heads, h = blockIdx.x % w.heads;
  const int kx = round_up(dx, 8), ms = round_up(dx, 16), ld = ld_of(dx);
  float* X = smem;
  float* Y = X + C * ld;
  float* W = Y + C * ld;  // y with its decays
  float* Z = W + C * ld;
  float* P = Z + C * LDZ;
  float* S = P + C * LDP;  // ms x LDZ
  const float a = decay_of(w, h);
  const int len = length_of(w, b);
  if (tid <= C) pw[tid] = power(a, tid);
  const T* xp = static_cast<const T*>(ps.x.p) + b * ps.x.b + h * ps.x.h;
  const T* yp = static_cast<const T*>(ps.y.p) + b * ps.y.b + h * ps.y.h;
  const T* zp = static_cast<const T*>(ps.z.p) + b * ps.z.b + h * ps.z.h + z0;
  T* op = static_cast<T*>(ps.out.p) + b * ps.out.b + h * ps.out.h + z0;
  const int64_t bh = (int64_t)b * w.heads + h, area = (int64_t)dx * dz;
  const int first = sg * w.seg, last = first + w.seg < w.time ? first + w.seg : w.time;  // tokens of the segment
  const int end = len < last ? len : last, chunks = end > first ? (end - first + C - 1) / C : 0;
  auto start = [&](int c) { return first + (ps.rev ? chunks - 1 - c : c) * C; };
  auto tokens = [&](int t0) { return end - t0 < C ? end - t0 : C; };
  Ahead<T, NX> ax, ay;
  Ahead<T, BZ / 32> az;
  auto fetch = [&](int c) {
    const int t0 = start(c), n = tokens(t0);
    if (!SUM) ax.load(xp + t0 * ps.x.t, ps.x.t, n, dx);
    ay.load(yp + t0 * ps.y.t, ps.y.t, n, dx);
    az.load(zp + t0 * ps.z.t, ps.z.t, n, nz);
  };
  if (chunks) fetch(0);
  // the state that comes in
  const float* in = SUM ? nullptr : w.segments > 1 ? ps.carry + (bh * w.segments + sg) * area : ps.init ? ps.init + bh * area : nullptr;
  const bool turned = w.segments == 1 && ps.init_t;
#pragma unroll 4
  for (int i = tid; i < ms * BZ; i += NT) {
    const int m = turned ? i % ms : i / BZ, n = turned ? i / ms : i % BZ;
    S[m * LDZ + n] = in && m < dx && n < nz ? in[turned ? (int64_t)(z0 + n) * dx + m : (int64_t)m * dz + z0 + n] : 0.f;
  }
  if (!SUM) {  // chunks without tokens
    const int t0 = first + chunks * C;
    for (int r = t0 + warp; r < last; r += NT / 32)
      for (int d = lane; d < nz; d += 32) st(op + r * ps.out.t + d, 0.f);
  }
  for (int c = 0; c < chunks; ++c) {
    const int t0 = start(c), n = tokens(t0), rows = last - t0 < C ? last - t0 : C;
    __syncthreads();
    const auto same = [](int) { return 1.f; };
    if (!SUM) {
      ax.put(X, ld, ms, same);
      ay.put(Y, ld, ms, same);  // (columns behind dx are zero, and so are rows behind n)
    }
    ay.put(W, ld, ms, [&](int r) { return ps.fs * pw[ps.rev ? r + 1 : (n - 1 - r) & 31]; });
    az.put(Z, LDZ, BZ, same);
    __syncthreads();
    if (c + 1 < chunks) fetch(c + 1);
    if (!SUM) {
      const int i0 = (warp & 1) * 16, n0 = (warp >> 1) * 16;
      {
        const int j0 = (warp >> 1) * 8;
        float s[1][4];
        tile<1>(s, kx, [&](int m, int k) { return X[(i0 + m) * ld + k]; }, [&](int k, int n_) { return Y[(j0 + n_) * ld + k]; });
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = i0 + g + (e >> 1) * 8, j = j0 + 2 * t + (e & 1), d = ps.rev ? j - i : i - j;
          const float v = ps.fp * pw[d & 31] * s[0][e];  // (a load for every lane: no branch)
          P[i * LDP + j] = d >= 0 ? v : 0.f;
        }
      }
      float out[2][4], v[2][4];
      tile<2>(out, kx, [&](int m, int k) { return X[(i0 + m) * ld + k]; }, [&](int k, int n_) { return S[k * LDZ + n0 + n_]; });
      __syncthreads();
      tile<2>(v, C, [&](int m, int k) { return P[(i0 + m) * LDP + k]; }, [&](int k, int n_) { return Z[k * LDZ + n0 + n_]; });
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = i0 + g + (e >> 1) * 8, d = n0 + 8 * u + 2 * t + (e & 1), p = ps.rev ? (n - 1 - i) & 31 : i + 1;
          const float x = fmaf(ps.fo * pw[p], out[u][e], v[u][e]);
          if (i < rows && d < nz) st(op + (t0 + i) * ps.out.t + d, i < n ? x : 0.f);
        }
    }
    // (every warp has read S: the barrier before the last product, or none reads it)
    const float pn = pw[n];
    for (int u = warp; u < ms / 16 * 2; u += NT / 32) {
      const int m0 = u / 2 * 16, n0 = u % 2 * 32;
      if (n0 >= nz) continue;
      float s[4][4];
      tile<4>(s, C, [&](int m, int k) { return W[k * ld + m0 + m]; }, [&](int k, int n_) { return Z[k * LDZ + n0 + n_]; });
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          float* at = &S[(m0 + g + (e >> 1) * 8) * LDZ + n0 + 8 * v + 2 * t + (e & 1)];
          *at = fmaf(pn, *at, s[v][e]);
        }
    }
  }
  float* to = SUM ? ps.carry + (bh * w.segments + sg) * area : ps.end && sg == (ps.rev ? 0 : w.segments - 1) ? ps.end + bh * area : nullptr;
  if (!to) return;
  __syncthreads();
  for (int i = tid; i < dx * BZ; i += NT) {
    const int m = i / BZ, n = i % BZ;
    if (n < nz) to[(int64_t)m * dz + z0 + n] = S[m * LDZ + n];
  }
}

// ---------------------------------------------------------------- joining segments
// carry[g] (a segment's own sum) becomes the state before segment g.
__global__ void __launch_bounds__(256) k_attend_join(const __grid_constant__ Work w) {
  const Pass& ps = w.pass[blockIdx.z];
  const int64_t area = (int64_t)ps.dx * ps.dz, bh = blockIdx.x;
  const int e = blockIdx.y * 256 + threadIdx.x;
  if (e >= area) return;
  const float a = decay_of(w, (int)(bh % w.heads)), whole = power(a, w.seg);
  const int len = length_of(w, (int)(bh / w.heads));
  float* c = ps.carry + bh * w.segments * area + e;
  float s = 0.f;
  if (ps.init) s = ps.init[bh * area + (ps.init_t ? (int64_t)(e % ps.dz) * ps.dx + e / ps.dz : e)];
  constexpr int U = 8;  // loads on their way (one after the other, 19 segments took 132 us)
  for (int i0 = 0; i0 < w.segments; i0 += U) {
    float own[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u, sg = ps.rev ? w.segments - 1 - i : i;
      own[u] = i < w.segments ? c[sg * area] : 0.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + u, sg = ps.rev ? w.segments - 1 - i : i, left = len - sg * w.seg, n = left < 0 ? 0 : left < w.seg ? left : w.seg;
      if (i >= w.segments) break;
      c[sg * area] = s;
      s = fmaf(n == w.seg ? whole : power(a, n), s, own[u]);
    }
  }
}

template <typename T, int NX>
cudaError_t launch_any(const Work& w, int zb, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};  // one bit a device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  constexpr int smem = any_smem(32 * NX);
  if (!(done.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(k_attend_any<T, NX, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attend_any<T, NX, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    done.fetch_or(bit, std::memory_order_release);
  }
  // (a pass with fewer columns has fewer CTAs a segment; the grid is the most that any needs)
  const dim3 all(w.batch * w.heads, zb * w.segments, w.passes);
  if (w.segments > 1) {
    k_attend_any<T, NX, true><<<all, NT, smem, st>>>(w);
    e = launch_join(w, st);
    if (e != cudaSuccess) return e;
  }
  k_attend_any<T, NX, false><<<all, NT, smem, st>>>(w);
  return cudaGetLastError();
}
template <typename T>
cudaError_t run_any(const Work& w, cudaStream_t st) {
  int dx = 0, zb = 0;
  for (int i = 0; i < w.passes; ++i) {
    dx = w.pass[i].dx > dx ? w.pass[i].dx : dx;
    const int n = (w.pass[i].dz + BZ - 1) / BZ;
    zb = n > zb ? n : zb;
  }
  if (dx <= 64) return launch_any<T, 2>(w, zb, st);
  return dx <= 128 ? launch_any<T, 4>(w, zb, st) : launch_any<T, 8>(w, zb, st);
}

// ---------------------------------------------------------------- one token
// A CTA: 32 or 128 columns of one head's state, its rows spread over the
// threads' groups, four columns a thread.
template <typename T, int V>
__global__ void __launch_bounds__(256) k_attend_step(const __grid_constant__ pnn_attend_step_args a, int cols) {
  __shared__ float part[256 * V];
  const int h = blockIdx.x % (int)a.heads, i = blockIdx.x / (int)a.heads, tid = threadIdx.x;
  const int per = cols / V, groups = 256 / per, col = blockIdx.y * cols + tid % per * V, grp = tid / per;
  const int dk = (int)a.dk, dv = (int)a.dv;
  T* o = static_cast<T*>(a.o) + i * a.o_stride_b + h * a.o_stride_h;
  const int slot = a.slot ? a.slot[i] : i;
  const bool on = col < dv;
  if (slot < 0 || slot >= a.slots) {
    if (grp == 0 && on)
      for (int e = 0; e < V; ++e) st(o + col + e, 0.f);
    return;
  }
  const T* q = static_cast<const T*>(a.q) + i * a.q_stride_b + h * a.q_stride_h;
  const T* k = static_cast<const T*>(a.k) + i * a.k_stride_b + h * a.k_stride_h;
  const T* v = static_cast<const T*>(a.v) + i * a.v_stride_b + h * a.v_stride_h;
  float* s = a.state + slot * a.state_stride + (int64_t)h * dk * dv + col;
  const float dec = fminf(fmaxf(a.decay[h], 0.f), 1.f);
  float vv[V], acc[V];
#pragma unroll
  for (int e = 0; e < V; ++e) {
    vv[e] = on ? seq::ld(v + col + e) : 0.f;
    acc[e] = 0.f;
  }
  if (on) {
#pragma unroll 4
    for (int r = grp; r < dk; r += groups) {
      const float kk = seq::ld(k + r), qq = seq::ld(q + r);
      float x[V];
      float* at = s + (int64_t)r * dv;
      if constexpr (V == 4) {
        const float4 f = __ldcs(reinterpret_cast<const float4*>(at));
        x[0] = f.x, x[1] = f.y, x[2] = f.z, x[3] = f.w;
      } else {
        x[0] = *at;
      }
#pragma unroll
      for (int e = 0; e < V; ++e) {
        x[e] = fmaf(dec, x[e], kk * vv[e]);
        acc[e] = fmaf(qq, x[e], acc[e]);
      }
      if constexpr (V == 4) __stcs(reinterpret_cast<float4*>(at), make_float4(x[0], x[1], x[2], x[3]));
      else *at = x[0];
    }
  }
#pragma unroll
  for (int e = 0; e < V; ++e) part[tid * V + e] = acc[e];
  __syncthreads();
  if (tid < cols && blockIdx.y * cols + tid < dv) {
    float sum = 0.f;
    for (int r = 0; r < groups; ++r) sum += part[r * cols + tid];
    st(o + blockIdx.y * cols + tid, a.scale * sum);
  }
}
template <typename T>
cudaError_t step(const pnn_attend_step_args& a, cudaStream_t st) {
  const unsigned heads = (unsigned)(a.batch * a.heads);
  const bool four = a.dv % 4 == 0 && a.state_stride % 4 == 0 && (reinterpret_cast<uintptr_t>(a.state) & 15) == 0;
  const int cols = four && heads >= (unsigned)device_sm_count() * 4 ? 128 : 32;
  const dim3 grid(heads, (unsigned)((a.dv + cols - 1) / cols));
  if (four) k_attend_step<T, 4><<<grid, 256, 0, st>>>(a, cols);
  else k_attend_step<T, 1><<<grid, 256, 0, st>>>(a, cols);
  return cudaGetLastError();
}

// ---------------------------------------------------------------- the plan
// Sequences are split into segments where their heads alone do not fill the GPU.  (By sizes and types alone: the
// workspace may be asked for before there are pointers.)
void split(Work& w) {
  const int dk = w.pass[0].dx, dv = w.pass[0].dz;
  const bool tc = w.dtype == PNN_DT_BF16 && dk <= 128 && dv <= 128;
  int64_t ctas = 0;
  for (int i = 0; i < w.passes; ++i) ctas += tc ? 1 : (w.pass[i].dz + BZ - 1) / BZ;
  ctas *= (int64_t)w.batch * w.heads;
  const int64_t want = (int64_t)device_sm_count() * (tc && (dk > 64 || dv > 64) ? 1 : 2);
  int64_t n = ctas >= want ? 1 : want / ctas;
  const int64_t most = (w.time + 255) / 256;  // segments of 256 tokens at least
  n = n < most ? n : most;
  int64_t seg = (w.time + n - 1) / n;
  seg = (seg + 127) / 128 * 128;
  w.seg = (int)seg;
  w.segments = (int)((w.time + seg - 1) / seg);
}
Rows rows(const pnn_head_rows& r) { return {r.p, r.stride_b, r.stride_t, r.stride_h}; }
Work plan(const pnn_attend_args& a, bool back) {
  Work w = {};
  w.passes = back ? 3 : 1;
  w.batch = (int)a.batch;
  w.time = (int)a.time;
  w.heads = (int)a.heads;
  w.dtype = a.dtype;
  w.lengths = a.lengths;
  w.decay = a.decay;
  const int dk = (int)a.dk, dv = (int)a.dv;
  const Rows q = rows(a.q), k = rows(a.k), v = rows(a.v), d = rows(a.dout);
  if (!back) {
    w.pass[0] = Pass{q, k, v, rows(a.o), dk, dv, false, a.scale, a.scale, 1.f, a.s0, false, a.s_last, nullptr};
  } else {
    w.pass[0] = Pass{d, v, k, rows(a.dq), dv, dk, false, a.scale, a.scale, 1.f, a.s0, true, nullptr, nullptr};
    w.pass[1] = Pass{v, d, q, rows(a.dk_out), dv, dk, true, a.scale, 1.f, a.scale, a.ds_last, true, nullptr, nullptr};
    w.pass[2] = Pass{k, q, d, rows(a.dv_out), dk, dv, true, a.scale, 1.f, a.scale, a.ds_last, false, a.ds0, nullptr};
  }
  split(w);
  return w;
}
size_t carry_bytes(const Work& w) {
  if (w.segments == 1) return 0;
  return (size_t)w.batch * w.heads * w.segments * w.pass[0].dx * w.pass[0].dz * 4;
}
}  // namespace

cudaError_t launch_join(const Work& w, cudaStream_t st) {
  const int64_t area = (int64_t)w.pass[0].dx * w.pass[0].dz;
  k_attend_join<<<dim3(w.batch * w.heads, (unsigned)((area + 255) / 256), w.passes), 256, 0, st>>>(w);
  return cudaGetLastError();
}
}  // namespace attend

size_t attend_workspace(const pnn_attend_args& a, bool back) {
  const attend::Work w = attend::plan(a, back);
  return attend::carry_bytes(w) * w.passes;
}
cudaError_t launch_attend(const pnn_attend_args& a, bool back, void* ws, cudaStream_t st) {
  attend::Work w = attend::plan(a, back);
  const size_t n = attend::carry_bytes(w);
  if (n)
    for (int i = 0; i < w.passes; ++i) w.pass[i].carry = reinterpret_cast<float*>(static_cast<char*>(ws) + i * n);
  if (attend::tc_fits(w)) {
    bool refused = false;
    const cudaError_t e = attend::run_tc(w, st, &refused);
    if (!refused) return e;
  }
  return a.dtype == PNN_DT_BF16 ? attend::run_any<seq::bf16>(w, st) : attend::run_any<float>(w, st);
}
cudaError_t launch_attend_step(const pnn_attend_step_args& a, cudaStream_t st) {
  return a.dtype == PNN_DT_BF16 ? attend::step<seq::bf16>(a, st) : attend::step<float>(a, st);
}

}  // namespace pnn
