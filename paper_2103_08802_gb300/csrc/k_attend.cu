// Linear attention with a decay for each head: passes of any widths, strides
// and types; joining the segments of long sequences; one token on a pool of
// states.  attend.cuh has the mathematics.
#include <cuda_runtime.h>

#include <atomic>
#include <type_traits>

#include "attend_walk.cuh"
#include "pnn_internal.h"

namespace pnn {
namespace attend {
namespace {
using namespace seq;

// ---------------------------------------------------------------- passes of any shape
// A CTA owns BZ columns of a head's state (columns of z do not meet) and walks
// over its segment in chunks of 32 tokens.  Products are bf16 mma.sync: an fp32
// operand goes as three bf16 numbers, the upper halves of itself and of what
// they leave (24 bits exactly), and of the nine products the six above 2^-24
// are formed, the largest in an accumulator of its own: the adder cuts off what is
// below its sum's last place, which would add up over a long state.  For the same
// reason a chunk's state product starts from zero and is added to the state, in
// fp32 in registers, by a rounded sum.  bf16 rows are one number each, P and the state
// on their way into an output two (16 bits: the output's own rounding is what remains), and K' is three.
//
// Bound: latency.  A chunk of 64 columns takes a CTA 9,900 cycles, 2,300 of which its
// products would at mma.sync's measured rate (1016 multiply-adds a cycle and SM); two CTAs an
// SM.  fp32 4 x 4096 x 16 x 64: 177 us and 67 for the segments' sums (40 at the copy
// bandwidth); 5 x 1531 x 7 x 40/72 ragged, forward and backward 271.  As sums of two tf32 numbers, split
// at every use, the latter took 460.
constexpr int C = 32, LDP = C + 8, NT = 256;

__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
template <bool TRANS>
__device__ __forceinline__ void ldsm(uint32_t (&r)[4], uint32_t at) {
  if constexpr (TRANS) asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
  else asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at));
}
// v as N bf16 numbers: one, rounded, or the upper halves of itself and of what they leave
template <int N>
__device__ __forceinline__ void split(float v0, float v1, uint32_t (&r)[N]) {
  if constexpr (N == 1) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(v0, v1);
    r[0] = *reinterpret_cast<const uint32_t*>(&h);
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      r[i] = __byte_perm(__float_as_uint(v0), __float_as_uint(v1), 0x7632);
      v0 -= __uint_as_float(r[i] << 16);
      v1 -= __uint_as_float(r[i] & 0xffff0000u);
    }
  }
}
// An operand in shared memory: its numbers `plane` bytes apart, rows `ld` bytes apart.
struct Op {
  uint32_t at, plane, ld;
};
// c += A (16 x 16 K) B (16 K x 16): two tiles of 8 columns.  A rows along its axis (AT: down the contraction's), B rows down
// its columns (BT: along them).  NA, NB: bf16 numbers of an operand.
template <int NA, int NB, bool AT, bool BT>
__device__ __forceinline__ void tile(float (&c)[2][4], float (&low)[2][4], int K, const Op& a, int m0, const Op& b, int n0, int k0 = 0) {
  const int l = threadIdx.x & 31, r = l & 7, q = l >> 3;
  // the four 8 x 8 matrices: A: (m, k), (m + 8, k), (m, k + 8), (m + 8, k + 8); B: (k, n), (k + 8, n), (k, n + 8), (k + 8, n + 8)
  uint32_t pa = AT ? a.at + (16 * k0 + (q >> 1) * 8 + r) * a.ld + (m0 + (q & 1) * 8) * 2 : a.at + (m0 + (q & 1) * 8 + r) * a.ld + (16 * k0 + (q >> 1) * 8) * 2;
  uint32_t pb = BT ? b.at + (16 * k0 + (q & 1) * 8 + r) * b.ld + (n0 + (q >> 1) * 8) * 2 : b.at + (n0 + (q >> 1) * 8 + r) * b.ld + (16 * k0 + (q & 1) * 8) * 2;
  for (int k = 0; k < K; ++k) {
    uint32_t x[NA][4], y[NB][4];
#pragma unroll
    for (int i = 0; i < NA; ++i) ldsm<AT>(x[i], pa + i * a.plane);
#pragma unroll
    for (int i = 0; i < NB; ++i) ldsm<BT>(y[i], pb + i * b.plane);
#pragma unroll
    for (int i = NA - 1; i >= 0; --i)
#pragma unroll
      for (int j = NB - 1; j >= 0; --j) {
        if (i + j > 2) continue;
#pragma unroll
        for (int u = 0; u < 2; ++u) mma(i + j ? low[u] : c[u], x[i], y[j][2 * u], y[j][2 * u + 1]);
      }
    pa += AT ? 16 * a.ld : 32;
    pb += BT ? 16 * b.ld : 32;
  }
}
__device__ __forceinline__ void clear(float (&c)[2][4]) {
#pragma unroll
  for (int u = 0; u < 2; ++u)
#pragma unroll
    for (int e = 0; e < 4; ++e) c[u][e] = 0.f;
}

// Rows of a chunk on their way in registers: warp w has rows w, w + 8, w + 16, w + 24, a lane two columns of every 64.  They
// stay as they came until they are put: a conversion would wait for each of them in turn (bf16 2 x 3000 x 5 x 256 971 us
// instead of 418).
template <typename T, int PAIRS>
struct Ahead {
  uint32_t v[4][PAIRS][2];  // two values, or of two bf16 on an even place both in the first
  __device__ __forceinline__ void load(const T* p, int64_t stride, int n, int width, bool even) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < PAIRS; ++j) {
        const int r = warp + 8 * i, d = 2 * lane + 64 * j;
        const T* at = p + r * stride + d;
        v[i][j][0] = v[i][j][1] = 0;
        if (r >= n || d >= width) continue;
        if (even) {  // (an even width: both are there)
          if constexpr (sizeof(T) == 4) {
            const uint2 f = *reinterpret_cast<const uint2*>(at);
            v[i][j][0] = f.x, v[i][j][1] = f.y;
          } else {
            v[i][j][0] = *reinterpret_cast<const uint32_t*>(at);
          }
        } else {
          using U = typename std::conditional<sizeof(T) == 4, uint32_t, unsigned short>::type;
          const U* u = reinterpret_cast<const U*>(at);
          v[i][j][0] = u[0];
          if (d + 1 < width) v[i][j][1] = u[1];
        }
      }
  }
  __device__ __forceinline__ float value(int i, int j, int k, bool even) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(v[i][j][k]);
    else if (k == 0) return __uint_as_float(v[i][j][0] << 16);
    else return __uint_as_float(even ? v[i][j][0] & 0xffff0000u : v[i][j][1] << 16);
  }
  // row r times f(r), as N numbers; columns below `most`, zeros behind the width
  template <int N, typename F>
  __device__ __forceinline__ void put(const Op& to, int most, bool even, F f) const {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = warp + 8 * i;
      const float x = f(r);
#pragma unroll
      for (int j = 0; j < PAIRS; ++j) {
        const int d = 2 * lane + 64 * j;
        if (d >= most) continue;
        uint32_t w[N];
        split<N>(value(i, j, 0, even) * x, value(i, j, 1, even) * x, w);
#pragma unroll
        for (int k = 0; k < N; ++k) asm volatile("st.shared.u32 [%0], %1;" ::"r"(to.at + k * to.plane + r * to.ld + d * 2), "r"(w[k]) : "memory");
      }
    }
  }
};

__host__ __device__ constexpr int round_up(int a, int b) { return (a + b - 1) / b * b; }
// Columns of the state that a CTA owns, where it has dx rows.
__host__ __device__ constexpr int any_columns(int dx) { return dx > 128 ? 32 : 64; }
// The most that a kernel's shape can take.  NS: numbers of x, y and z, NP: of P and S; BX: 16 times the most tiles of the state's rows.
template <typename T, int BX>
struct Form {
  static constexpr int NS = sizeof(T) == 4 ? 3 : 1, NP = sizeof(T) == 4 ? 3 : 2, BZ = any_columns(BX);
  // bytes of a row (an odd number of 16: eight rows in a column meet in no bank), and of one number's plane
  static constexpr int LDX = (BX + 8) * 2, LDZ = (BZ + 8) * 2, LDQ = LDP * 2;
  static constexpr int X = C * LDX, Z = C * LDZ, P = C * LDQ, S = BX * LDZ;
  static constexpr int BYTES = (2 * NS + 3) * X + NS * Z + NP * (P + S);
  static constexpr int MT = BX / 16;                                             // row tiles of the state, shared by 8 warps:
  static constexpr int PER = MT <= 8 ? 1 : MT / 8, GROUPS = MT < 8 ? 8 / MT : 1; // PER of a warp, or its columns by GROUPS of them
  static constexpr int NT2 = BZ / 16 / GROUPS;                                   // tiles of 16 columns of a warp
};

template <typename T, int BX, bool SUM>
__global__ void __launch_bounds__(NT, BX <= 64 ? 2 : 1) k_attend_any(const __grid_constant__ Work w) {
  using F = Form<T, BX>;
  constexpr int NS = F::NS, NP = F::NP, BZ = F::BZ;
  extern __shared__ __align__(128) char smem[];
  __shared__ float pw[C + 1];
  const Pass& ps = w.pass[blockIdx.z];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int dx = ps.dx, dz = ps.dz, zblocks = (dz + BZ - 1) / BZ;
  const int zb = blockIdx.y % zblocks, sg = blockIdx.y / zblocks;
  if (sg >= w.segments) return;  // (another pass has more columns)
  const int z0 = zb * BZ, nz = dz - z0 < BZ ? dz - z0 : BZ;
  const int b = blockIdx.x / w.heads, h = blockIdx.x % w.heads;
  const int kx = round_up(dx, 16);
  const uint32_t base = static_cast<uint32_t>(__cvta_generic_to_shared(smem));
  const Op W{base, F::X, F::LDX}, Z{base + 3 * F::X, F::Z, F::LDZ}, X{Z.at + NS * F::Z, F::X, F::LDX}, Y{X.at + NS * F::X, F::X, F::LDX},
      P{Y.at + NS * F::X, F::P, F::LDQ}, S{P.at + NP * F::P, F::S, F::LDZ};
  const float a = decay_of(w, h);
  const int len = length_of(w, b);
  if (tid <= C) pw[tid] = power(a, tid);
  const T* xp = static_cast<const T*>(ps.x.p) + b * ps.x.b + h * ps.x.h;
  const T* yp = static_cast<const T*>(ps.y.p) + b * ps.y.b + h * ps.y.h;
  const T* zp = static_cast<const T*>(ps.z.p) + b * ps.z.b + h * ps.z.h + z0;
  T* op = static_cast<T*>(ps.out.p) + b * ps.out.b + h * ps.out.h + z0;
  auto even = [&](const T* p, const Rows& r, int width) { return width % 2 == 0 && r.t % 2 == 0 && (reinterpret_cast<uintptr_t>(p) & (2 * sizeof(T) - 1)) == 0; };
  const bool ex = even(xp, ps.x, dx), ey = even(yp, ps.y, dx), ez = even(zp, ps.z, nz), eo = even(op, ps.out, nz);
  const int64_t bh = (int64_t)b * w.heads + h, area = (int64_t)dx * dz;
  const int first = sg * w.seg, last = first + w.seg < w.time ? first + w.seg : w.time;  // tokens of the segment
  const int end = len < last ? len : last, chunks = end > first ? (end - first + C - 1) / C : 0;
  auto start = [&](int c) { return first + (ps.rev ? chunks - 1 - c : c) * C; };
  auto tokens = [&](int t0) { return end - t0 < C ? end - t0 : C; };
  Ahead<T, (BX + 63) / 64> ax, ay;
  Ahead<T, 1> az;
  auto fetch = [&](int c) {
    const int t0 = start(c), n = tokens(t0);
    if (!SUM) ax.load(xp + t0 * ps.x.t, ps.x.t, n, dx, ex);
    ay.load(yp + t0 * ps.y.t, ps.y.t, n, dx, ey);
    az.load(zp + t0 * ps.z.t, ps.z.t, n, nz, ez);
  };
  if (chunks) fetch(0);
  // the state that comes in: a warp's tiles, as the products leave them
  const int mt = F::MT < 8 ? warp % F::MT : warp * F::PER, nt = F::MT < 8 ? warp / F::MT * F::NT2 : 0;  // its first tile of rows, of 16 columns
  float s[F::PER][F::NT2][2][4];
  auto each = [&](auto f) {  // f(the value, its row, its column)
#pragma unroll
    for (int i = 0; i < F::PER; ++i)
#pragma unroll
      for (int j = 0; j < F::NT2; ++j)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) f(s[i][j][u][e], (mt + i) * 16 + g + (e >> 1) * 8, (nt + j) * 16 + u * 8 + 2 * t + (e & 1));
  };
  {
    const float* in = SUM ? nullptr : w.segments > 1 ? ps.carry + (bh * w.segments + sg) * area : ps.init ? ps.init + bh * area : nullptr;
    const bool turned = w.segments == 1 && ps.init_t;
    each([&](float& v, int m, int n) { v = in && m < dx && n < nz ? in[turned ? (int64_t)(z0 + n) * dx + m : (int64_t)m * dz + z0 + n] : 0.f; });
  }
  auto show = [&]() {  // the state as an operand
#pragma unroll
    for (int i = 0; i < F::PER; ++i)
#pragma unroll
      for (int j = 0; j < F::NT2; ++j)
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            uint32_t r[NP];
            split<NP>(s[i][j][u][2 * e], s[i][j][u][2 * e + 1], r);
#pragma unroll
            for (int k = 0; k < NP; ++k)
              asm volatile("st.shared.u32 [%0], %1;" ::"r"(S.at + k * S.plane + ((mt + i) * 16 + g + e * 8) * S.ld + ((nt + j) * 16 + u * 8 + 2 * t) * 2), "r"(r[k]) : "memory");
          }
  };
  if (!SUM) {
    show();
    const int t0 = first + chunks * C;  // chunks without tokens
    for (int r = t0 + warp; r < last; r += NT / 32)
      for (int d = lane; d < nz; d += 32) st(op + r * ps.out.t + d, 0.f);
  }
  for (int c = 0; c < chunks; ++c) {
    const int t0 = start(c), n = tokens(t0), rows = last - t0 < C ? last - t0 : C;
    __syncthreads();
    const auto same = [](int) { return 1.f; };
    if (!SUM) {
      ax.template put<NS>(X, kx, ex, same);
      ay.template put<NS>(Y, kx, ey, same);
    }
    ay.template put<3>(W, kx, ey, [&](int r) { return ps.fs * pw[ps.rev ? r + 1 : (n - 1 - r) & 31]; });  // (rows behind n are zero)
    az.template put<NS>(Z, BZ, ez, same);
    __syncthreads();
    if (c + 1 < chunks) fetch(c + 1);
    if (!SUM) {
      const int i0 = (warp & 1) * 16;
      float o[2][4], v[2][4], low[2][4];
      // scores: four warps a tile of 16 x 16 each, but the one that no row sees
      if (warp < 4) {
        const int j0 = (warp >> 1) * 16;
        clear(v), clear(low);
        if (ps.rev ? j0 >= i0 : j0 <= i0) tile<NS, NS, false, false>(v, low, kx / 16, X, i0, Y, j0);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x[2];
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const int i = i0 + g + e * 8, j = j0 + u * 8 + 2 * t + k, d = ps.rev ? j - i : i - j;
              const float f = ps.fp * pw[d & 31];  // (a load for every lane: no branch)
              x[k] = d >= 0 ? f * (v[u][2 * e + k] + low[u][2 * e + k]) : 0.f;
            }
            uint32_t r[NP];
            split<NP>(x[0], x[1], r);
#pragma unroll
            for (int k = 0; k < NP; ++k) asm volatile("st.shared.u32 [%0], %1;" ::"r"(P.at + k * P.plane + (i0 + g + e * 8) * P.ld + (j0 + u * 8 + 2 * t) * 2), "r"(r[k]) : "memory");
          }
      }
      // what the state before the chunk gives: the warps that form no scores begin with it
      const int n0 = (warp >> 1) * 16;
      const bool on = n0 < nz && n0 < BZ;
      clear(o), clear(low);
      if (on) tile<NS, NP, false, true>(o, low, kx / 16, X, i0, S, n0);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int i = i0 + g + (e >> 1) * 8;
          o[u][e] = (o[u][e] + low[u][e]) * (ps.fo * pw[ps.rev ? (n - 1 - i) & 31 : i + 1]);
        }
      __syncthreads();
      clear(v), clear(low);
      if (on) tile<NP, NS, false, true>(v, low, ps.rev == (i0 > 0) ? 1 : 2, P, i0, Z, n0, ps.rev && i0 ? 1 : 0);
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int i = i0 + g + e * 8, d = n0 + u * 8 + 2 * t;
          const float x = i < n ? v[u][2 * e] + low[u][2 * e] + o[u][2 * e] : 0.f, y = i < n ? v[u][2 * e + 1] + low[u][2 * e + 1] + o[u][2 * e + 1] : 0.f;
          if (i >= rows || !on || d >= nz) continue;
          T* to = op + (t0 + i) * ps.out.t + d;
          if (eo) {
            if constexpr (sizeof(T) == 4) {
              *reinterpret_cast<float2*>(to) = make_float2(x, y);
            } else {
              uint32_t r[1];
              split<1>(x, y, r);
              *reinterpret_cast<uint32_t*>(to) = r[0];
            }
          } else {
            st(to, x);
            if (d + 1 < nz) st(to + 1, y);
          }
        }
    }
    // (every warp has read S: the barrier before the last product, or none reads it)
    const float pn = pw[n];
#pragma unroll
    for (int i = 0; i < F::PER; ++i)
#pragma unroll
      for (int j = 0; j < F::NT2; ++j) {
        float v[2][4], low[2][4];
        clear(v), clear(low);
        if ((mt + i) * 16 < dx && (nt + j) * 16 < nz) tile<3, NS, true, true>(v, low, C / 16, W, (mt + i) * 16, Z, (nt + j) * 16);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[i][j][u][e] = fmaf(pn, s[i][j][u][e], v[u][e] + low[u][e]);
      }
    if (!SUM) show();
  }
  float* to = SUM ? ps.carry + (bh * w.segments + sg) * area : ps.end && sg == (ps.rev ? 0 : w.segments - 1) ? ps.end + bh * area : nullptr;
  if (to) each([&](float& v, int m, int n) {
    if (m < dx && n < nz) to[(int64_t)m * dz + z0 + n] = v;
  });
  if (!SUM) {
    static_assert((BX * BZ + kWalkMore) * 4 <= F::BYTES, "room for the walk");
    float odd = 0.f;  // NaN if a column is not finite (which it is in all rows, or none, of its own products)
#pragma unroll
    for (int j = 0; j < F::NT2; ++j)
#pragma unroll
      for (int u = 0; u < 2; ++u) odd = fmaf(s[0][j][u][0], 0.f, fmaf(s[0][j][u][1], 0.f, odd));
    if (__syncthreads_or(odd != odd)) {
      const int3 at = cta_again();
      const int width = w.pass[at.z].dz, blocks = (width + BZ - 1) / BZ, from = at.y % blocks * BZ;
      walk<T>(w, w.pass[at.z], at.x / w.heads, at.x % w.heads, at.y / blocks, from, width - from < BZ ? width - from : BZ, C, reinterpret_cast<float*>(smem));
    }
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

template <typename T, int BX>
cudaError_t launch_any(const Work& w, cudaStream_t st) {
  using F = Form<T, BX>;
  static std::atomic<uint64_t> done{0};  // one bit a device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return e;
  const uint64_t bit = 1ull << (dev & 63);
  if (!(done.load(std::memory_order_acquire) & bit)) {
    e = cudaFuncSetAttribute(k_attend_any<T, BX, true>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::BYTES);
    if (e == cudaSuccess) e = cudaFuncSetAttribute(k_attend_any<T, BX, false>, cudaFuncAttributeMaxDynamicSharedMemorySize, F::BYTES);
    if (e != cudaSuccess) return e;
    done.fetch_or(bit, std::memory_order_release);
  }
  int zb = 0;  // (a pass with fewer columns has fewer CTAs a segment; the grid is the most that any needs)
  for (int i = 0; i < w.passes; ++i) {
    const int n = (w.pass[i].dz + F::BZ - 1) / F::BZ;
    zb = n > zb ? n : zb;
  }
  const dim3 all(w.batch * w.heads, zb * w.segments, w.passes);
  if (w.segments > 1) {
    k_attend_any<T, BX, true><<<all, NT, F::BYTES, st>>>(w);
    e = launch_join(w, st);
    if (e != cudaSuccess) return e;
  }
  k_attend_any<T, BX, false><<<all, NT, F::BYTES, st>>>(w);
  return cudaGetLastError();
}
int most_rows(const Work& w) {  // of a state
  int dx = 0;
  for (int i = 0; i < w.passes; ++i) dx = w.pass[i].dx > dx ? w.pass[i].dx : dx;
  return dx;
}
template <typename T>
cudaError_t run_any(const Work& w, cudaStream_t st) {
  const int dx = most_rows(w);
  if (dx <= 32) return launch_any<T, 32>(w, st);
  if (dx <= 64) return launch_any<T, 64>(w, st);
  return dx <= 128 ? launch_any<T, 128>(w, st) : launch_any<T, 256>(w, st);
}

// ---------------------------------------------------------------- one token
// A CTA: 32 or 128 columns of one head's state, its rows spread over the
// threads' groups, four columns a thread.  Bound: HBM, the state read and written:
// 96 states of 16 x 128 x 128 take 39 us (201 MB, 5.2 TB/s; 64 columns or loads 16 deep
// the same).
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
int64_t ctas_of(const Work& w, int columns) {  // a segment's
  int64_t n = 0;
  for (int i = 0; i < w.passes; ++i) n += (w.pass[i].dz + columns - 1) / columns;
  return n * w.batch * w.heads;
}
// Few tokens: a chunk of the other kernel instead of a padded one of the tensor-core kernel's, and finer outputs.  64 columns: 1 x 1 x 4
// 5.2 us instead of 7.3, 256 x 32 x 16 84 instead of 116.  128 columns, a CTA an SM: 1 x 7 x 4 7.4 instead of 10.7, but with
// more CTAs than SMs 20 x 29 x 16 33 instead of 31, 256 x 32 x 16 352 instead of 280.
bool few(const Work& w) {
  const int dx = most_rows(w), columns = any_columns(dx);
  return w.time <= C && (dx <= 64 || ctas_of(w, columns) <= device_sm_count());
}
// Sequences are split into segments where their heads alone do not fill the GPU.  The tensor-core kernel: one wave of CTAs
// (4 x 4096 x 16 x 64 76 us, in two waves 84; 65536 x 8 x 128 189 and 222), of 256 tokens at least.  The other one: no
// segments, or up to three waves of 128 tokens at least, whichever has the fewest tokens one after another, those of the
// segments' sums counted as 0.4 each and two more launches as 64 (fp32 4 x 2048 x 16 x 128 as one segment 376 us, as two
// 532; 1 x 1024 x 4 x 64 as eight 33, as four 51).  Sequences with lengths of their own: two waves, so that long ones
// find the places of short ones (5 x 1531 x 7 x 40/72 forward 71 us, in one 99).  By sizes, types and
// whether there are lengths alone.
void split(Work& w, bool ragged) {
  const int dk = w.pass[0].dx, dv = w.pass[0].dz, dx = most_rows(w);
  const bool tc = w.dtype == PNN_DT_BF16 && dk <= 128 && dv <= 128 && dk % 8 == 0 && dv % 8 == 0 && !few(w);
  const int columns = tc ? 128 : any_columns(dx), unit = tc ? 128 : C;
  const int64_t ctas = ctas_of(w, columns);
  const int64_t slots = (int64_t)device_sm_count() * ((tc && dv > dx ? dv : dx) > 64 ? 1 : 2);  // CTAs that run at once
  const int64_t most = tc ? (w.time + 255) / 256 : w.time < 256 ? 1 : w.time / 128;
  const auto segments = [&](int64_t waves) {
    const int64_t n = waves * slots / ctas;
    return n < 1 ? 1 : n < most ? n : most;
  };
  const auto length = [&](int64_t n) { return ((w.time + n - 1) / n + unit - 1) / unit * unit; };
  int64_t n = segments(tc ? 1 : 2);
  if (!tc && !ragged) {
    const auto cost = [&](int64_t n) {
      const int64_t walk = (ctas * n + slots - 1) / slots * length(n);
      return n == 1 ? walk : walk * 7 / 5 + 64;
    };
    n = 1;
    for (int waves = 1; waves <= 3; ++waves)
      if (cost(segments(waves)) < cost(n)) n = segments(waves);
  }
  w.seg = (int)length(n);
  w.segments = (w.time + w.seg - 1) / w.seg;
}
Rows rows(const pnn_head_rows& r) { return {r.p, r.stride_b, r.stride_t, r.stride_h}; }
Work plan(const pnn_attend_args& a, bool back, bool ragged) {
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
  split(w, ragged);
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
  // (enough with lengths and without: they may be added after the question)
  const attend::Work w = attend::plan(a, back, false), r = attend::plan(a, back, true);
  const size_t n = attend::carry_bytes(w), m = attend::carry_bytes(r);
  return (n > m ? n : m) * w.passes;
}
cudaError_t launch_attend(const pnn_attend_args& a, bool back, void* ws, cudaStream_t st) {
  attend::Work w = attend::plan(a, back, a.lengths != nullptr);
  const size_t n = attend::carry_bytes(w);
  if (n)
    for (int i = 0; i < w.passes; ++i) w.pass[i].carry = reinterpret_cast<float*>(static_cast<char*>(ws) + i * n);
  if (!attend::few(w) && attend::tc_fits(w)) {
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
