// Linear attention of bf16 rows on the 5th-generation tensor cores (attend.cuh
// has the mathematics): heads of up to 128, rows on 16-byte boundaries.
//
// A CTA walks over a segment of one head in chunks of 128 tokens.  TMA brings the
// tiles of x, y and z, [128 tokens][64 columns] with 128-byte swizzle, into a ring;
// the same tile serves as an operand along its columns or along its tokens.  For each
// chunk
//   A  = x y^T                        128 x 128, to TMEM
//   P  = A with its decays, in bf16   by the four score warps, back to TMEM
//   O1 = P z,  O2 = x S               two accumulators: O2's rows are scaled where they are read
//   U  = K'^T z                       K' = y with its decays
//   S := a^n S + U                    by the four state warps, fp32 in registers
// and S goes as bf16 into shared memory for the next chunk's O2.  K' is formed
// as b0 + b1 + b2 in bf16 (24 bits; b0 in place of y, b1 and b2 by halves of 64
// tokens), so that the state keeps fp32's precision: with b0 + b1 alone a state is
// off by 2.7e-6 of its norm, with b0 by 1.7e-3.  P and the S of O2 are rounded to bf16
// once, as the outputs are.  U starts from zero for every chunk and is added by
// a rounded sum, since the tensor cores' adder cuts off.
//
// Rows behind a sequence: their decays are zero (selected, not multiplied), and
// the rows of z that zeros would meet are cleared in shared memory.
#include <cuda_runtime.h>

#include <atomic>

#include "attend.cuh"
#include "pnn_internal.h"
#include "tc_ptx.cuh"

namespace pnn {
namespace attend {
namespace {
using namespace seq;
using namespace tc;

constexpr int C = 128, RING = 5, NT = 320;
constexpr int kTmaWarp = 8, kMmaWarp = 9;

struct Maps {
  __align__(64) char m[4][128];  // CUtensorMap
  int x[3], y[3], z[3];          // the maps of a pass
  int one_b[4], one_h[4];        // 0 where every sequence, or head, has the same rows
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
      : "memory");
}
// operand along a tile's columns (64 of them contiguous, `next` bytes to the next 64): the contraction runs over its rows, 8 of them 1024 bytes
__device__ __forceinline__ uint64_t mn128_desc(uint32_t addr, uint32_t next) {
  uint64_t d = 0;
  d |= (uint64_t)((addr & 0x3FFFF) >> 4);
  d |= (uint64_t)((next >> 4) & 0x3FFF) << 16;
  d |= (uint64_t)(1024 >> 4) << 32;
  d |= (uint64_t)1 << 46;
  d |= (uint64_t)2 << 61;
  return d;
}
constexpr uint32_t kMnA = 1u << 15, kMnB = 1u << 16;  // instruction descriptor: A, B along their rows' columns
// D = A (from TMEM) B
__device__ __forceinline__ void mma_bf16_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(accumulate)
      : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <int DX, int DZ>
struct Shape {
  static constexpr int XB = DX / 64, ZB = DZ / 64;      // 64-column blocks
  static constexpr int BLK = C * 128;                   // bytes of one: 128 rows of 128 bytes
  static constexpr int TILE = BLK * (XB > ZB ? XB : ZB);
  static constexpr int HALF = 64 * 128 * XB;            // b1 or b2 of 64 tokens
  static constexpr int SBLK = DX * 128, STATE = SBLK * ZB;
  static constexpr int BYTES = RING * TILE + 2 * HALF + STATE;
  // TMEM columns: the scores (their first half becomes P), O1, O2, U.  Of 64 columns O1 takes the scores' second half, and two CTAs share an SM.
  static constexpr int O1 = DZ == 64 ? 64 : 128, O2 = DZ == 64 ? 128 : 256, U = DZ == 64 ? 192 : 384, COLS = DZ == 64 ? 256 : 512;
  static constexpr int CTAS = DX == 64 && DZ == 64 ? 2 : 1;
};
struct Shared {
  uint64_t full[RING], empty[RING], scores, seen, p, o, read, k[2], half, u, state, clear, drain;
  int abort_;
  uint32_t tmem;
  alignas(16) float row[32];  // the decays of a block of 32 columns off the diagonal, times fp
  float pw[C + 1];
};

template <int DX, int DZ, bool SUM>
__global__ void __launch_bounds__(NT, Shape<DX, DZ>::CTAS) k_attend_tc(const __grid_constant__ Work w, const __grid_constant__ Maps maps, int* gave_up) {
  using L = Shape<DX, DZ>;
  extern __shared__ char raw[];
  __shared__ Shared sh;
  const uint32_t ring = (smem_u32(raw) + 1023) & ~1023u, b1 = ring + RING * L::TILE, b2 = b1 + L::HALF, sbf = b2 + L::HALF;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int pi = blockIdx.x % w.passes;
  const int64_t bh = blockIdx.x / w.passes;
  const Pass& ps = w.pass[pi];
  const int b = (int)(bh / w.heads), h = (int)(bh % w.heads), sg = blockIdx.y;
  const int first = sg * w.seg, last = first + w.seg < w.time ? first + w.seg : w.time;
  const int len = length_of(w, b), end = len < last ? len : last;
  const int chunks = end > first ? (end - first + C - 1) / C : 0;  // that have tokens
  const bool rev = ps.rev;
  auto start = [&](int c) { return first + (rev ? chunks - 1 - c : c) * C; };
  auto tokens = [&](int t0) { return end - t0 < C ? end - t0 : C; };
  const float a = decay_of(w, h);

  if (warp == kMmaWarp) tmem_alloc(smem_u32(&sh.tmem), L::COLS);
  if (tid == 0) {
    for (int i = 0; i < RING; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 1);
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    mbar_init(smem_u32(&sh.scores), 1);
    mbar_init(smem_u32(&sh.seen), 4);
    mbar_init(smem_u32(&sh.p), 4);
    mbar_init(smem_u32(&sh.o), 1);
    mbar_init(smem_u32(&sh.read), 4);
    mbar_init(smem_u32(&sh.k[0]), 4);
    mbar_init(smem_u32(&sh.k[1]), 4);
    mbar_init(smem_u32(&sh.half), 1);
    mbar_init(smem_u32(&sh.u), 1);
    mbar_init(smem_u32(&sh.state), 4);
    mbar_init(smem_u32(&sh.clear), 4);
    mbar_init(smem_u32(&sh.drain), 1);
    sh.abort_ = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid <= C) {
    const float p = power(a, tid);
    sh.pw[tid] = p;
    if (tid < 32) sh.row[rev ? tid : 31 - tid] = ps.fp * p;
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem;
  volatile int* abort_ = &sh.abort_;
  // A wait that gives up marks the call; everyone then leaves.
  auto wait1 = [&](uint64_t& bar, uint32_t n) {
    if (mbar_wait(smem_u32(&bar), n & 1, abort_)) return true;
    if (!*abort_) count_give_up(gave_up);
    *abort_ = 1;
    return false;
  };
  auto wait = [&](uint64_t& bar, uint32_t n) {  // by a whole warp
    const bool ok = mbar_wait(smem_u32(&bar), n & 1, abort_);
    if (__all_sync(0xffffffffu, ok)) return true;
    if (lane == 0 && !*abort_) count_give_up(gave_up);
    *abort_ = 1;
    return false;
  };
  auto arrive = [&](uint64_t& bar) {
    fence_before();
    __syncwarp();
    if (lane == 0) mbar_arrive(smem_u32(&bar));
  };
  // loads in the order x, y, z of each chunk (y, z for sums)
  constexpr int PER = SUM ? 2 : 3, IY = SUM ? 0 : 1, IZ = SUM ? 1 : 2;
  auto slot = [&](int n) { return ring + n % RING * L::TILE; };

  if (warp == kTmaWarp) {
    // -------------------------------------------------------------- loads
    if (lane == 0) {
      int n = 0;
      bool ok = true;
      for (int c = 0; c < chunks && ok; ++c) {
        const int t0 = start(c);
        for (int i = 0; i < PER && ok; ++i, ++n) {
          if (n >= RING) ok = wait1(sh.empty[n % RING], n / RING - 1);
          if (!ok) break;
          const int id = i == IY ? maps.y[pi] : i == IZ ? maps.z[pi] : maps.x[pi], blocks = i == IZ ? L::ZB : L::XB;
          const uint32_t bar = smem_u32(&sh.full[n % RING]);
          mbar_expect_tx(bar, blocks * L::BLK);
          for (int k = 0; k < blocks; ++k)
            tma_load_4d(slot(n) + k * L::BLK, maps.m[id], 64 * k, h * maps.one_h[id], t0, b * maps.one_b[id], bar);
        }
      }
      // the copies that were issued land before the CTA ends
      if (!ok)
        for (int i = n > RING ? n - RING : 0; i < n; ++i) mbar_wait_drain(smem_u32(&sh.full[i % RING]), (i / RING) & 1);
    }
    __syncwarp();
  } else if (warp == kMmaWarp) {
    // -------------------------------------------------------------- products
    if (lane == 0 && chunks) {
      const uint32_t id_a = idesc_bf16(128, 128), id_o = idesc_bf16(128, DZ) | kMnB, id_u = idesc_bf16(128, DZ) | kMnA | kMnB;
      bool ok = true, issued = false;
      auto full = [&](int n) { return wait1(sh.full[n % RING], n / RING); };
      auto scores = [&](int c) {
        ok = full(PER * c) && full(PER * c + IY);
        if (!ok) return;
        fence_after();
        const uint32_t x = slot(PER * c), y = slot(PER * c + IY);
        for (int k = 0; k < DX / 16; ++k) {
          const uint32_t at = k / 4 * L::BLK + k % 4 * 32;
          mma_bf16(tmem, sw128_desc(x + at), sw128_desc(y + at), id_a, k ? 1u : 0u);
        }
        issued = true;
        mma_commit(smem_u32(&sh.scores));
      };
      if (!SUM) scores(0);
      for (int c = 0; c < chunks && ok; ++c) {
        const uint32_t x = slot(PER * c), y = slot(PER * c + IY), z = slot(PER * c + IZ);
        const bool part = tokens(start(c)) < C;
        if (!(ok = full(PER * c + IZ))) break;
        if (!SUM) {
          if (!(ok = wait1(sh.p, c) && (!part || wait1(sh.clear, 0)))) break;
          fence_after();
          for (int k = 0; k < C / 16; ++k) mma_bf16_ts(tmem + L::O1, tmem + k * 8, mn128_desc(z + k * 2048, L::BLK), id_o, k ? 1u : 0u);
          if (!(ok = wait1(sh.state, c))) break;
          fence_after();
          for (int k = 0; k < DX / 16; ++k)
            mma_bf16(tmem + L::O2, sw128_desc(x + k / 4 * L::BLK + k % 4 * 32), mn128_desc(sbf + k * 2048, L::SBLK), id_o, k ? 1u : 0u);
          mma_commit(smem_u32(&sh.o));
          mma_commit(smem_u32(&sh.empty[(PER * c) % RING]));
          if (c + 1 < chunks) {
            // (a barrier may run one phase ahead of who waits for it, and the scores take the place of an O1 of 64 columns)
            if (!(ok = wait1(sh.seen, c) && (DZ > 64 || wait1(sh.read, c)))) break;
            scores(c + 1);
            if (!ok) break;
          }
        }
        for (int i = 0; i < 2; ++i) {
          if (!(ok = wait1(sh.k[i], c))) break;
          fence_after();
          const uint32_t from[3] = {b2, b1, y + i * 64 * 128};
          for (int j = 0; j < 3; ++j)  // the small ones first
            for (int k = 0; k < 4; ++k)
              mma_bf16(tmem + L::U, mn128_desc(from[j] + k * 2048, j < 2 ? 64 * 128 : L::BLK), mn128_desc(z + (4 * i + k) * 2048, L::BLK), id_u,
                       (i | j | k) ? 1u : 0u);
          issued = true;
          mma_commit(smem_u32(i ? &sh.u : &sh.half));
        }
        if (!ok) break;
        mma_commit(smem_u32(&sh.empty[(PER * c + IY) % RING]));
        mma_commit(smem_u32(&sh.empty[(PER * c + IZ) % RING]));
      }
      if (!ok && issued) {
        mma_commit(smem_u32(&sh.drain));
        mbar_wait_drain(smem_u32(&sh.drain), 0);
      }
    }
    __syncwarp();
  } else if (warp < 4) {
    // -------------------------------------------------------------- scores to P, outputs
    if (!SUM) {
      const int i = warp * 32 + lane;  // this thread's row
      const uint32_t lanes = (uint32_t)(warp * 32) << 16;
      bf16* out = static_cast<bf16*>(ps.out.p) + b * ps.out.b + h * ps.out.h;
      {
        const int z8 = ps.dz / 8, t0 = first + chunks * C;  // rows of chunks without tokens
        for (int64_t e = tid; e < (int64_t)(last - t0) * z8; e += 128)
          *reinterpret_cast<uint4*>(out + (t0 + e / z8) * ps.out.t + e % z8 * 8) = make_uint4(0, 0, 0, 0);
      }
      for (int c = 0; c < chunks; ++c) {
        const int t0 = start(c), n = tokens(t0);
        if (!wait(sh.scores, c)) break;
        fence_after();
#pragma unroll
        for (int cb = 0; cb < 4; ++cb) {
          uint32_t r[16];
          const int off = rev ? cb - warp : warp - cb;  // blocks of 32 columns off the diagonal
          if (off < 0) {
#pragma unroll
            for (int j = 0; j < 16; ++j) r[j] = 0;
          } else {
            uint32_t s[32];
            tmem_ld32(tmem + lanes + cb * 32, s);
            tmem_wait_ld();
            if (off > 0) {
              // a^|i-j| = a^(distance to the block's near column) times a^(distance inside)
              const float base = sh.pw[rev ? cb * 32 - i : i - cb * 32 - 31];
#pragma unroll
              for (int j = 0; j < 32; j += 4) {
                const float4 d = *reinterpret_cast<const float4*>(&sh.row[j]);
                float v[4] = {__uint_as_float(s[j]) * base * d.x, __uint_as_float(s[j + 1]) * base * d.y, __uint_as_float(s[j + 2]) * base * d.z,
                              __uint_as_float(s[j + 3]) * base * d.w};
                if (rev) {  // (forwards no row with a token sees a column without)
#pragma unroll
                  for (int e = 0; e < 4; ++e) v[e] = cb * 32 + j + e < n ? v[e] : 0.f;
                }
                r[j / 2] = pack_bf16(v[0], v[1]);
                r[j / 2 + 1] = pack_bf16(v[2], v[3]);
              }
            } else {
#pragma unroll
              for (int j = 0; j < 32; j += 2) {
                float v[2];
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                  const int d = rev ? j + e - lane : lane - j - e;
                  v[e] = d >= 0 && cb * 32 + j + e < n ? __uint_as_float(s[j + e]) * (ps.fp * sh.pw[d & 31]) : 0.f;
                }
                r[j / 2] = pack_bf16(v[0], v[1]);
              }
            }
          }
          tmem_st16(tmem + lanes + cb * 16, r);
        }
        tmem_wait_st();
        arrive(sh.p);
        if (!wait(sh.o, c)) break;
        fence_after();
        const float f = i < n ? ps.fo * sh.pw[rev ? n - 1 - i : i + 1] : 0.f;
        bf16* to = out + (t0 + i) * ps.out.t;
#pragma unroll
        for (int cb = 0; cb < DZ / 32; ++cb) {
          uint32_t u[32], v[32];
          tmem_ld32(tmem + lanes + L::O1 + cb * 32, u);
          tmem_ld32(tmem + lanes + L::O2 + cb * 32, v);
          tmem_wait_ld();
          if (cb == DZ / 32 - 1) arrive(sh.read);
#pragma unroll
          for (int j = 0; j < 32; j += 8) {
            float x[8];
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = i < n ? fmaf(f, __uint_as_float(v[j + e]), __uint_as_float(u[j + e])) : 0.f;
            if (cb * 32 + j < ps.dz && t0 + i < last) *reinterpret_cast<uint4*>(to + cb * 32 + j) = pack8(x);
          }
          __syncwarp();
        }
      }
    }
  } else {
    // -------------------------------------------------------------- the state
    const int q = warp - 4, m = q * 32 + lane, st = tid - 128;  // this thread's row of the state
    const uint32_t lanes = (uint32_t)(q * 32) << 16;
    const bool mine = q * 32 < DX;
    const int dx = ps.dx, dz = ps.dz;
    const int64_t area = (int64_t)dx * dz;
    float s[DZ];
    {
      const float* in = SUM ? nullptr : w.segments > 1 ? ps.carry + (bh * w.segments + sg) * area : ps.init ? ps.init + bh * area : nullptr;
      const bool turned = w.segments == 1 && ps.init_t;
#pragma unroll
      for (int j = 0; j < DZ; ++j) s[j] = in && m < dx && j < dz ? in[turned ? (int64_t)j * dx + m : (int64_t)m * dz + j] : 0.f;
    }
    auto show = [&]() {  // S for the next chunk's product
      if (mine) {
#pragma unroll
        for (int j = 0; j < DZ; j += 8) {
          const uint4 v = pack8(&s[j]);
          const uint32_t at = sbf + j / 64 * L::SBLK + swz(m, j % 64 / 8);
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
        }
      }
      fence_proxy_async();
      arrive(sh.state);
    };
    if (!SUM) show();
    for (int c = 0; c < chunks; ++c) {
      const int t0 = start(c), n = tokens(t0), ny = PER * c + IY, nz = PER * c + IZ;
      const uint32_t y = slot(ny), z = slot(nz);
      if (!wait(sh.full[ny % RING], ny / RING)) break;
      if (n < C) {
        if (!wait(sh.full[nz % RING], nz / RING)) break;
        for (int e = st; e < (C - n) * 8 * L::ZB; e += 128) {
          const int r = n + e / (8 * L::ZB), k = e % (8 * L::ZB);
          asm volatile("st.shared.v4.u32 [%0], {%1, %1, %1, %1};" ::"r"(z + k / 8 * L::BLK + r * 128 + k % 8 * 16), "r"(0) : "memory");
        }
        fence_proxy_async();
        arrive(sh.clear);
      }
      if (!SUM) {  // (b0 takes y's place)
        if (!wait(sh.scores, c)) break;
        arrive(sh.seen);
      }
      bool ok = true;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (i && !(ok = wait(sh.half, c))) break;
#pragma unroll 2
        for (int e = st; e < 64 * 8 * L::XB; e += 128) {
          const int blk = e / 512, r = e % 512 / 8, tok = i * 64 + r;
          const uint32_t at = y + blk * L::BLK + i * 64 * 128 + e % 512 * 16, lo = blk * 64 * 128 + e % 512 * 16;
          uint4 v;
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
          const float f = tok < n ? ps.fs * sh.pw[rev ? tok + 1 : n - 1 - tok] : 0.f;
          const uint32_t in[4] = {v.x, v.y, v.z, v.w};
          uint32_t o0[4], o1[4], o2[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t live = tok < n ? in[k] : 0u;
            const float p = __uint_as_float(live << 16) * f, g = __uint_as_float(live & 0xffff0000u) * f;
            o0[k] = pack_bf16(p, g);
            const float p1 = p - __uint_as_float(o0[k] << 16), g1 = g - __uint_as_float(o0[k] & 0xffff0000u);
            o1[k] = pack_bf16(p1, g1);
            o2[k] = pack_bf16(p1 - __uint_as_float(o1[k] << 16), g1 - __uint_as_float(o1[k] & 0xffff0000u));
          }
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(o0[0]), "r"(o0[1]), "r"(o0[2]), "r"(o0[3]) : "memory");
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(b1 + lo), "r"(o1[0]), "r"(o1[1]), "r"(o1[2]), "r"(o1[3]) : "memory");
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(b2 + lo), "r"(o2[0]), "r"(o2[1]), "r"(o2[2]), "r"(o2[3]) : "memory");
        }
        fence_proxy_async();
        arrive(sh.k[i]);
      }
      if (!ok || !wait(sh.u, c)) break;
      fence_after();
      if (mine) {
        const float pn = sh.pw[n];
#pragma unroll
        for (int cb = 0; cb < DZ / 32; ++cb) {
          uint32_t u[32];
          tmem_ld32(tmem + lanes + L::U + cb * 32, u);
          tmem_wait_ld();
#pragma unroll
          for (int j = 0; j < 32; ++j) s[cb * 32 + j] = fmaf(pn, s[cb * 32 + j], __uint_as_float(u[j]));
        }
      }
      if (!SUM) show();
    }
    float* to = SUM ? ps.carry + (bh * w.segments + sg) * area : ps.end && sg == (rev ? 0 : w.segments - 1) ? ps.end + bh * area : nullptr;
    if (to && m < dx) {
#pragma unroll
      for (int j = 0; j < DZ; j += 4)
        if (j < dz) *reinterpret_cast<float4*>(to + (int64_t)m * dz + j) = make_float4(s[j], s[j + 1], s[j + 2], s[j + 3]);
    }
  }
  fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    fence_after();
    tmem_dealloc(tmem, L::COLS);
  }
}

template <int DX, int DZ, bool SUM>
cudaError_t launch(const Work& w, const Maps& maps, int* word, cudaStream_t st) {
  const auto kernel = k_attend_tc<DX, DZ, SUM>;
  constexpr int smem = Shape<DX, DZ>::BYTES + 1024;
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
  kernel<<<dim3((unsigned)(w.batch * w.heads * w.passes), (unsigned)w.segments), NT, smem, st>>>(w, maps, word);
  return cudaGetLastError();
}
template <int DX, int DZ>
cudaError_t run(const Work& w, const Maps& maps, int* word, cudaStream_t st) {
  if (w.segments > 1) {
    cudaError_t e = launch<DX, DZ, true>(w, maps, word, st);
    if (e == cudaSuccess) e = launch_join(w, st);
    if (e != cudaSuccess) return e;
  }
  return launch<DX, DZ, false>(w, maps, word, st);
}
bool fits(const Rows& r, int d, const Work& w) {
  return d <= 128 && d % 8 == 0 && (reinterpret_cast<uintptr_t>(r.p) & 15) == 0 && (w.batch == 1 || r.b % 8 == 0) && (w.time == 1 || (r.t % 8 == 0 && r.t > 0)) &&
         (w.heads == 1 || r.h % 8 == 0);
}
}  // namespace

bool tc_fits(const Work& w) {
  if (w.dtype != PNN_DT_BF16) return false;
  for (int i = 0; i < w.passes; ++i) {
    const Pass& p = w.pass[i];
    if (!fits(p.x, p.dx, w) || !fits(p.y, p.dx, w) || !fits(p.z, p.dz, w) || !fits(p.out, p.dz, w)) return false;
    if ((reinterpret_cast<uintptr_t>(p.end) & 15) != 0) return false;
  }
  return true;
}

cudaError_t run_tc(const Work& w, cudaStream_t st, bool* refused) {
  Maps maps;
  int n = 0;
  const Rows* seen[4];
  int width[4];
  auto map_of = [&](const Rows& r, int d) {
    for (int i = 0; i < n; ++i)
      if (seen[i]->p == r.p && seen[i]->b == r.b && seen[i]->t == r.t && seen[i]->h == r.h && width[i] == d) return i;
    if (n == 4) return -1;
    const int64_t size[4] = {d, r.h || w.heads == 1 ? w.heads : 1, w.time, r.b || w.batch == 1 ? w.batch : 1};
    const int64_t stride[3] = {size[1] > 1 ? r.h : 64, size[2] > 1 ? r.t : 64, size[3] > 1 ? r.b : 64};
    const int box[4] = {64, 1, C, 1};
    const char* why = nullptr;
    if (encode_tensor_map_4d(maps.m[n], r.p, size, stride, box, &why)) return -1;
    maps.one_h[n] = size[1] > 1;
    maps.one_b[n] = size[3] > 1;
    seen[n] = &r;
    width[n] = d;
    return n++;
  };
  for (int i = 0; i < w.passes; ++i) {
    const Pass& p = w.pass[i];
    maps.x[i] = map_of(p.x, p.dx);
    maps.y[i] = map_of(p.y, p.dx);
    maps.z[i] = map_of(p.z, p.dz);
    if (maps.x[i] < 0 || maps.y[i] < 0 || maps.z[i] < 0) {
      *refused = true;
      return cudaSuccess;
    }
  }
  *refused = false;
  int* word = seq_gave_up_word();
  if (!word) return cudaGetLastError();
  // every pass has the widths of both: 64 or 128 each
  bool x64 = true, z64 = true;
  for (int i = 0; i < w.passes; ++i) {
    x64 = x64 && w.pass[i].dx <= 64;
    z64 = z64 && w.pass[i].dz <= 64;
  }
  if (x64) return z64 ? run<64, 64>(w, maps, word, st) : run<64, 128>(w, maps, word, st);
  return z64 ? run<128, 64>(w, maps, word, st) : run<128, 128>(w, maps, word, st);
}

}  // namespace attend
}  // namespace pnn
