// What the linear attention's passes leave to be done where a row of z is not finite.
//
// A chunk's outputs are P z, and P's zeros, at tokens that a row does not see, times an infinity or a NaN are NaN: of
// the rows of its chunk also those become so that come before it.  (Rows of x and y do no such harm: scores are selected,
// not multiplied.)  A column of z meets no other, and its state is not finite either from there on, which is how a CTA
// notices when it is done: the walk then goes over its segment once more, token by token, and writes those rows again in the
// columns concerned.  Bound: shared memory and its latency, 4,200 cycles a token at 128 x 128 and 600 at 64 x 64 (a NaN near
// the end of one head of 8 x 4096 x 16 x 128 makes a call of 126 us one of 9 ms).  A call without such values pays for the look
// at the last state alone, 0 to 1.6 % (most where a sequence is one token).
#pragma once
#include "attend.cuh"

namespace pnn {
namespace attend {

// blockIdx read anew, for a kernel's call of the walk: values that it kept for it all the time cost it registers (64 x 64 heads
// 4 %, where the walk itself costs nothing).
__device__ __forceinline__ int3 cta_again() {
  int3 r;
  asm volatile("mov.u32 %0, %%ctaid.x;\n\tmov.u32 %1, %%ctaid.y;\n\tmov.u32 %2, %%ctaid.z;" : "=r"(r.x), "=r"(r.y), "=r"(r.z));
  return r;
}

constexpr int kWalkMore = 128 + 2 * 256;

// All threads of a CTA (256 at least) come here, with what its columns z0 .. z0 + nz - 1 (nz <= 128) are for.  unit: tokens of a
// chunk.  S: dx x (nz rounded up to 32, 64 or 128) numbers of shared memory, and kWalkMore behind them.
template <typename T>
__device__ __noinline__ void walk(const Work& w, const Pass& ps, int b, int h, int sg, int z0, int nz, int unit, float* S) {
  const int tid = threadIdx.x, cols = nz <= 32 ? 32 : nz <= 64 ? 64 : 128, c = tid % cols, groups = 256 / cols, r0 = tid < 256 && c < nz ? tid / cols : ps.dx;
  const int first = sg * w.seg, last = first + w.seg < w.time ? first + w.seg : w.time, len = length_of(w, b), end = len < last ? len : last, n = end - first;
  const int dx = ps.dx, dz = ps.dz;
  const bool rev = ps.rev;
  const T* xp = static_cast<const T*>(ps.x.p) + b * ps.x.b + h * ps.x.h;
  const T* yp = static_cast<const T*>(ps.y.p) + b * ps.y.b + h * ps.y.h;
  const T* zp = static_cast<const T*>(ps.z.p) + b * ps.z.b + h * ps.z.h + z0;
  T* op = static_cast<T*>(ps.out.p) + b * ps.out.b + h * ps.out.h + z0;
  auto token = [&](int p) { return rev ? end - 1 - p : first + p; };  // at place p of the pass's order
  int* odd = reinterpret_cast<int*>(S + dx * cols);                  // a column's first place that is not finite, or n
  for (int i = tid; i < nz; i += blockDim.x) odd[i] = n;
  __syncthreads();
  for (int64_t e = tid; e < (int64_t)n * nz; e += blockDim.x) {
    const int p = (int)(e / nz), i = (int)(e % nz);
    if (!isfinite(seq::ld(zp + token(p) * ps.z.t + i))) atomicMin(&odd[i], p);
  }
  __syncthreads();
  int most = 0;  // places that some column has before its first
  for (int i = 0; i < nz; ++i)
    if (odd[i] < n && odd[i] > most) most = odd[i];
  if (!most) return;
  const int64_t bh = (int64_t)b * w.heads + h, area = (int64_t)dx * dz;
  const float* in = w.segments > 1 ? ps.carry + (bh * w.segments + sg) * area : ps.init ? ps.init + bh * area : nullptr;
  const bool turned = w.segments == 1 && ps.init_t;
  for (int r = r0; r < dx; r += groups) S[r * cols + c] = in ? in[turned ? (int64_t)(z0 + c) * dx + r : (int64_t)r * dz + z0 + c] : 0.f;
  const float a = decay_of(w, h);
  const int mine = tid < nz ? odd[tid] : n;
  // rows of y come through shared memory, one ahead (little is left of L1: from there a token took 7,400 cycles instead)
  float* ahead = S + dx * cols + 128;
  auto row = [&](int p) { return tid < dx ? seq::ld(yp + token(p) * ps.y.t + tid) : 0.f; };
  auto entry = [&](int p) { return r0 < dx ? ps.fs * seq::ld(zp + token(p) * ps.z.t + c) : 0.f; };
  if (tid < dx) ahead[tid] = row(0);
  float z = entry(0);
  __syncthreads();
  for (int p = 0; p < most; ++p) {
    const int t = token(p);
    const float f = rev && p == 0 ? 1.f : a;  // (a reverse state has its last token's decay in it)
    const float* y = ahead + (p & 1) * 256;
    const float next = p + 1 < most ? row(p + 1) : 0.f, z1 = p + 1 < most ? entry(p + 1) : 0.f;
#pragma unroll 4
    for (int r = r0; r < dx; r += groups) S[r * cols + c] = fmaf(f, S[r * cols + c], y[r] * z);
    if (tid < dx) ahead[(~p & 1) * 256 + tid] = next;
    z = z1;
    const bool wrong = mine < n && p < mine && (t - first) / unit == (token(mine) - first) / unit;
    if (!__syncthreads_or(wrong)) continue;
    if (wrong) {
      const T* x = xp + t * ps.x.t;
      float o = 0.f;
      for (int r = 0; r < dx; ++r) o = fmaf(seq::ld(x + r), S[r * cols + tid], o);
      seq::st(op + t * ps.out.t + tid, ps.fo * o);
    }
    __syncthreads();
  }
}

}  // namespace attend
}  // namespace pnn
