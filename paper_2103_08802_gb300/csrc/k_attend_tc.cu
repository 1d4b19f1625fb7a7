// Linear attention of bf16 rows on the 5th-generation tensor cores (attend.cuh
// has the mathematics): heads of up to 128, rows on 16-byte boundaries.
//
// A CTA walks over a segment of one head in chunks of 128 tokens.  TMA brings the
// tiles of x, y and z, [128 tokens][64 columns] with 128-byte swizzle, into a ring;
// the same tile serves as an operand along its columns or along its tokens.  For each
// chunk
//   A  = x y^T                        128 x 128, to TMEM
//   P  = A with its decays, in bf16   by the four score warps, back to TMEM
//   O  = P z + x S                    its rows are scaled where they are read
//   U  = K'^T z                       K' = y with its decays, by the four decay warps
//   S := a^n S + U                    by the state warps, fp32 in registers, half of the columns each
// and S goes as bf16 into shared memory for the next chunk's O.  A row's decay is
// taken out of P, a^(i-j) = a^(i+1) a^-(j+1), so that P and S meet in one
// accumulator (a P of 16 bits has the exponents of 32); where a^128 is below 1e-12 P
// has its decays whole and x S an accumulator of its own.  The score warps
// leave the chunk's outputs in x's place, from where TMA stores them.  K' is formed
// as b0 + b1 + b2 in bf16 (24 bits; b0 in place of y, b1 and b2 by quarters of 32
// tokens in two buffers, so that a quarter is formed while another is multiplied),
// so that the state keeps fp32's precision: with b0 + b1 alone a state is off by
// 2.7e-6 of its norm, with b0 by 1.7e-3.  P and the S of O are rounded to bf16
// once, as the rows that came in and the outputs are: an output is off by 2.3e-3 of its
// norm instead of its own rounding's 1.7e-3, and second numbers of both would be a
// third more products and a tile less in the ring.  U starts from zero for every chunk
// and is added by a rounded sum, since the tensor cores' adder cuts off.
//
// Rows behind a sequence: their decays are zero (selected, not multiplied), and
// the rows of z that zeros would meet are cleared in shared memory.
//
// Bound: the latency of a chunk's chain (load, scores, P, O; K', U, S) in 7,500
// cycles for 128 columns, 3,100 of which the tensor cores work; inputs that lie in L2
// take as long.  8 x 4096 x 16 heads of 128: 126 us (537 MB, 4.3 TB/s; 79 at the copy
// bandwidth), its backward, three such passes, 342; 65536 x 8 x 128 in segments 189
// (63 of it the segments' own sums).  Before that: decays by the warps that hold the
// state 913 us forward and backward, by warps of their own 574, without divergent
// loads on the diagonal 514, operands in uniform registers and one accumulator 467.
// Outputs stored from registers, with a ring of four tiles and K' in buffers for all
// four quarters, took 149 us instead of 126.
#include <cuda_runtime.h>

#include <atomic>

#include "attend_ring.h"
#include "attend_walk.cuh"
#include "pnn_internal.h"
#include "tc_ptx.cuh"

namespace pnn {
namespace attend {
namespace {
using namespace seq;
using namespace tc;

constexpr int C = 128, QTR = 32;

struct Maps {
  __align__(64) char m[4][128];    // CUtensorMap
  __align__(64) char out[3][128];  // of a pass
  int x[3], y[3], z[3];            // the maps of a pass
  int one_b[4], one_h[4];        // 0 where every sequence, or head, has the same rows
};

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const void* map, int c0, int c1, int c2, int c3, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
      "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(bar)
      : "memory");
}
__device__ __forceinline__ void tma_store_4d(const void* map, int c0, int c1, int c2, int c3, uint32_t src) {
  asm volatile("cp.async.bulk.tensor.4d.global.shared::cta.bulk_group [%0, {%1, %2, %3, %4}], [%5];" ::"l"(map), "r"(c0), "r"(c1), "r"(c2),
               "r"(c3), "r"(src)
               : "memory");
}
// Operands in tiles of 128-byte rows with 128-byte swizzle: 8 rows are 1024 bytes.  A descriptor's upper half is the same
// for all; its lower half has the address / 16 in its lowest bits, so that steps are added to it.
constexpr uint32_t kDescHi = (1024 >> 4) | 1u << 14 | 2u << 29;
// along a row the contraction, down the rows the operand's other axis
__device__ __forceinline__ uint32_t k_operand(uint32_t addr) { return (addr & 0x3FFFF) >> 4 | 1u << 16; }
// the other way round; `next`: bytes to the columns after 64
__device__ __forceinline__ uint32_t mn_operand(uint32_t addr, uint32_t next) { return (addr & 0x3FFFF) >> 4 | (next >> 4) << 16; }
constexpr uint32_t kMnA = 1u << 15, kMnB = 1u << 16;  // instruction descriptor: A, B of the second kind
// The whole warp comes here and the one elected lane issues: without a branch the operands stay in uniform registers, where
// the instruction wants them.
__device__ __forceinline__ uint32_t elect() {
  uint32_t r;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(r));
  return r;
}
__device__ __forceinline__ void mma_ss(uint32_t leader, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %5};\n\tmov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHi), "r"(leader)
      : "memory");
}
// A from TMEM
__device__ __forceinline__ void mma_ts(uint32_t leader, uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t.reg .b64 db;\n\t"
      "mov.b64 db, {%2, %5};\n\t"
      "setp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %6, 0;\n\t"
      "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, p;\n\t}" ::"r"(d),
      "r"(a), "r"(b), "r"(idesc), "r"(accumulate), "n"(kDescHi), "r"(leader)
      : "memory");
}
__device__ __forceinline__ void commit(uint32_t leader, uint64_t& bar) {
  asm volatile(
      "{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %1, 0;\n\t"
      "@q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t}" ::"r"(smem_u32(&bar)),
      "r"(leader)
      : "memory");
}
__device__ __forceinline__ void tmem_ld(uint32_t addr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
        "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]),
        "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]),
        "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_ld(uint32_t addr, uint32_t (&r)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
                 "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
               : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_st(uint32_t addr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), "r"(r[0]),
      "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
      "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st(uint32_t addr, const uint32_t (&r)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]),
               "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

template <int DX, int DZ>
struct Shape {
  static constexpr int XB = DX / 64, ZB = DZ / 64;      // 64-column blocks
  static constexpr int BLK = C * 128;                   // bytes of one: 128 rows of 128 bytes
  static constexpr int TILE = BLK * (XB > ZB ? XB : ZB);
  static constexpr int PIECE = QTR * 128 * XB;          // b1 or b2 of a quarter
  static constexpr int SBLK = DX * 128, STATE = SBLK * ZB;
  static constexpr int BYTES = RING * TILE + 4 * PIECE + STATE;
  // TMEM columns: the scores (their first half becomes P), O, U, and O2 where decays are strong.  Of 64 columns O2 takes the
  // scores' second half, and two CTAs share an SM.
  static constexpr int O = 128, O2 = DZ == 64 ? 64 : 256, U = DZ == 64 ? 192 : 384, COLS = DZ == 64 ? 256 : 512;
  static constexpr int CTAS = DX == 64 && DZ == 64 ? 2 : 1;
  // Warps: 0 to 3 scores and outputs, 4 to 11 the state (a warp reads the 32 lanes of TMEM, rows of the state, that its
  // number modulo 4 gives).  64 rows need half of those, the other four form K'; else four more do.
  static constexpr int kTma = DX == 64 ? 12 : 16, kMma = kTma + 1, kStore = kTma + 2, NT = 32 * (kTma + 3);
  static constexpr int STATES = DX == 64 ? 4 : 8, COLUMNS = DZ / 2;
};
struct Shared {
  // loads; scores ready / seen by the decay warps; P; O ready / read; K' quarter ready / free; U ready / free; S; z cleared; outputs staged
  uint64_t full[RING], empty[RING], scores, seen, p, o, read, k[2], kfree[2], u[2], ufree[2], state, clear, staged, drain;
  int abort_, odd;  // odd: the last state is not finite
  uint32_t tmem;
  alignas(16) float row[32];  // strong decays: those of a block of 32 columns off the diagonal, times fp
  alignas(16) float col[C];   // else a column's
  float pw[C + 1];
};

template <int DX, int DZ, bool SUM>
__global__ void __launch_bounds__(Shape<DX, DZ>::NT, Shape<DX, DZ>::CTAS)
    k_attend_tc(const __grid_constant__ Work w, const __grid_constant__ Maps maps, int* gave_up) {
  using L = Shape<DX, DZ>;
  extern __shared__ char raw[];
  __shared__ Shared sh;
  const uint32_t ring = (smem_u32(raw) + 1023) & ~1023u, pieces = ring + RING * L::TILE, sbf = pieces + 4 * L::PIECE;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
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
  constexpr int TW = SUM ? 8 : 4;  // warps that form K': where there are no scores, theirs too

  if (warp == L::kMma) tmem_alloc(smem_u32(&sh.tmem), L::COLS);
  if (tid == 0) {
    for (int i = 0; i < RING; ++i) {
      mbar_init(smem_u32(&sh.full[i]), 1);
      mbar_init(smem_u32(&sh.empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(smem_u32(&sh.k[i]), TW);
      mbar_init(smem_u32(&sh.kfree[i]), 1);
      mbar_init(smem_u32(&sh.u[i]), 1);
      mbar_init(smem_u32(&sh.ufree[i]), L::STATES);
    }
    mbar_init(smem_u32(&sh.scores), 1);
    mbar_init(smem_u32(&sh.seen), 4);
    mbar_init(smem_u32(&sh.p), 4);
    mbar_init(smem_u32(&sh.o), 1);
    mbar_init(smem_u32(&sh.read), 4);
    mbar_init(smem_u32(&sh.state), L::STATES);
    mbar_init(smem_u32(&sh.clear), TW);
    mbar_init(smem_u32(&sh.staged), 4);
    mbar_init(smem_u32(&sh.drain), 1);
    sh.abort_ = sh.odd = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (tid <= C) {
    const float p = power(a, tid);
    sh.pw[tid] = p;
    if (tid < 32) sh.row[rev ? tid : 31 - tid] = ps.fp * p;
    if (rev ? tid < C : tid > 0) sh.col[rev ? C - 1 - tid : tid - 1] = __fdiv_rn(rev ? ps.fp : 1.f, p);
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem;
  const bool strong = sh.pw[C] < 1e-12f;
  volatile int* abort_ = &sh.abort_;
  // A wait that gives up marks the call; everyone then leaves.  (A barrier may complete one phase more than who waits for
  // it has seen, not two: what it announces next is held back by something that the waiting warps do after the wait.)
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
  // quarter g (of all chunks): its b1, then b2
  auto piece = [&](int g) { return pieces + (g & 1) * 2 * L::PIECE; };

  if (warp == L::kTma) {
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
      // the copies that were issued land before the CTA ends, whether or not who consumes them has given up
      for (int i = n > RING ? n - RING : 0; i < n; ++i) mbar_wait_drain(smem_u32(&sh.full[i % RING]), (i / RING) & 1);
    }
    __syncwarp();
  } else if (warp == L::kMma) {
    // -------------------------------------------------------------- products
    if (chunks) {
      const uint32_t leader = elect();
      const uint32_t id_a = idesc_bf16(128, 128), id_o = idesc_bf16(128, DZ) | kMnB, id_u = idesc_bf16(128, DZ) | kMnA | kMnB;
      const uint32_t before = mn_operand(sbf, L::SBLK), lower = mn_operand(pieces, QTR * 128);
      constexpr int NEXT_AT = DZ == 64 ? 0 : -1;  // the quarter of U behind which the next scores are issued (-1: before it; measured)
      bool ok = true, issued = false;
      auto full = [&](int n) { return wait(sh.full[n % RING], n / RING); };
      auto scores = [&](int c) {
        ok = full(PER * c) && full(PER * c + IY);
        if (!ok) return;
        fence_after();
        const uint32_t x = k_operand(slot(PER * c)), y = k_operand(slot(PER * c + IY));
#pragma unroll
        for (int k = 0; k < DX / 16; ++k) {
          const uint32_t at = (k / 4 * L::BLK + k % 4 * 32) >> 4;
          mma_ss(leader, tmem, x + at, y + at, id_a, k ? 1u : 0u);
        }
        issued = true;
        commit(leader, sh.scores);
      };
      // the next chunk's scores, which the decay warps have to be ready for; an O2 of 64 columns is in their place
      auto next_scores = [&](int c) {
        if (c + 1 >= chunks) return;
        ok = wait(sh.seen, c) && (DZ > 64 || !strong || wait(sh.read, c));
        if (ok) scores(c + 1);
      };
      if (!SUM) scores(0);
      for (int c = 0; c < chunks && ok; ++c) {
        const uint32_t x = k_operand(slot(PER * c)), y = mn_operand(slot(PER * c + IY), L::BLK), z = mn_operand(slot(PER * c + IZ), L::BLK);
        const bool part = tokens(start(c)) < C;
        if (!(ok = full(PER * c + IZ))) break;
        if (!SUM) {
          if (!(ok = wait(sh.p, c) && (!part || wait(sh.clear, 0)))) break;
          fence_after();
#pragma unroll
          for (int k = 0; k < C / 16; ++k) mma_ts(leader, tmem + L::O, tmem + k * 8, z + (k * 2048 >> 4), id_o, k ? 1u : 0u);
        }
        // S is there, and U has been read; without scores their columns are a second U
        if (SUM && c < 2) {
        } else if (!(ok = SUM ? wait(sh.ufree[c & 1], (c >> 1) - 1) : wait(sh.state, c))) {
          break;
        }
        fence_after();
        if (!SUM) {
#pragma unroll
          for (int k = 0; k < DX / 16; ++k)
            mma_ss(leader, tmem + (strong ? L::O2 : L::O), x + ((k / 4 * L::BLK + k % 4 * 32) >> 4), before + (k * 2048 >> 4), id_o, k || !strong ? 1u : 0u);
          commit(leader, sh.o);
          if (NEXT_AT < 0) next_scores(c);
          if (!ok) break;
        }
#pragma unroll 1
        for (int i = 0; i < 4; ++i) {
          const int g = 4 * c + i;
          if (!(ok = wait(sh.k[g & 1], g >> 1))) break;
          fence_after();
          const uint32_t u_at = SUM && c & 1 ? tmem : tmem + L::U;
          const uint32_t small = lower + (g & 1 ? 2 * L::PIECE >> 4 : 0), large = y + (i * QTR * 128 >> 4), rows = z + (i * QTR * 128 >> 4);
#pragma unroll
          for (int j = 0; j < 3; ++j)  // the small ones first
#pragma unroll
            for (int k = 0; k < 2; ++k)
              mma_ss(leader, u_at, j < 2 ? small + (((1 - j) * L::PIECE + k * 2048) >> 4) : large + (k * 2048 >> 4), rows + (k * 2048 >> 4),
                     id_u, (i | j | k) ? 1u : 0u);
          issued = true;
          if (buffer_again(g, chunks)) commit(leader, sh.kfree[g & 1]);
          if (!SUM && i == NEXT_AT) {
            next_scores(c);
            if (!ok) break;
          }
        }
        if (!ok) break;
        commit(leader, sh.u[SUM ? c & 1 : 0]);
        if (place_again(PER * c + IY, PER * chunks)) commit(leader, sh.empty[(PER * c + IY) % RING]);
        if (place_again(PER * c + IZ, PER * chunks)) commit(leader, sh.empty[(PER * c + IZ) % RING]);
      }
      if (!ok && issued) {
        commit(leader, sh.drain);
        mbar_wait_drain(smem_u32(&sh.drain), 0);
      }
    }
    __syncwarp();
  } else if (warp == L::kStore) {
    // -------------------------------------------------------------- outputs, from x's place
    if (!SUM && lane == 0) {
      for (int c = 0; c < chunks; ++c) {
        if (!wait1(sh.staged, c)) break;
        for (int k = 0; k < L::ZB; ++k)
          if (64 * k < ps.dz) tma_store_4d(maps.out[pi], 64 * k, h, start(c), b, slot(PER * c) + k * L::BLK);
        bulk_commit();
        bulk_wait_read<0>();
        mbar_arrive(smem_u32(&sh.empty[(PER * c) % RING]));
      }
      bulk_wait_all();
    }
    __syncwarp();
  } else if (!SUM && warp < 4) {
    // -------------------------------------------------------------- scores to P, outputs
    if constexpr (!SUM) {
      constexpr int W = L::CTAS == 2 ? 16 : 32;  // columns at a time: registers
      const int i = tid;                         // this thread's row
      const uint32_t lanes = (uint32_t)(warp * 32) << 16;
      {
        bf16* out = static_cast<bf16*>(ps.out.p) + b * ps.out.b + h * ps.out.h;
        const int z8 = ps.dz / 8, t0 = first + chunks * C;  // rows of chunks without tokens
        for (int64_t e = tid; e < (int64_t)(last - t0) * z8; e += 128)
          *reinterpret_cast<uint4*>(out + (t0 + e / z8) * ps.out.t + e % z8 * 8) = make_uint4(0, 0, 0, 0);
      }
      // the columns of a block of 32 that this row sees: on the diagonal up to itself, and those with a token
      auto sees = [&](int off, int cb, int n) {
        uint32_t m = off ? ~0u : rev ? ~0u << lane : ~0u >> (31 - lane);
        if (n < cb * 32 + 32) m &= n > cb * 32 ? (1u << (n - cb * 32)) - 1 : 0u;
        return m;
      };
      // a^-(31 - lane), or a^-lane, for the blocks on the diagonal: while it does not overflow, nor a^31 times it lose bits
      const bool mild = sh.pw[31] > 1e-30f;
      const float near = mild ? __fdiv_rn(1.f, sh.pw[rev ? lane : 31 - lane]) : 1.f;
      for (int c = 0; c < chunks; ++c) {
        const int t0 = start(c), n = tokens(t0);
        if (!wait(sh.scores, c)) break;
        fence_after();
        if (strong) {
#pragma unroll 1
          for (int c0 = 0; c0 < C; c0 += W) {
            uint32_t r[W / 2];
            const int cb = c0 / 32, off = rev ? cb - warp : warp - cb;  // blocks of 32 columns off the diagonal
            if (off < 0) {
#pragma unroll
              for (int j = 0; j < W / 2; ++j) r[j] = 0;
            } else {
              uint32_t s[W];
              tmem_ld(tmem + lanes + c0, s);
              const uint32_t mask = sees(off, cb, n) >> c0 % 32;
              float4 d[W / 4];
              if (off || mild) {
#pragma unroll
                for (int j = 0; j < W / 4; ++j) d[j] = *reinterpret_cast<const float4*>(&sh.row[c0 % 32 + 4 * j]);
              } else {  // (a load for every lane: no branch)
#pragma unroll
                for (int j = 0; j < W / 4; ++j) {
                  const int at = rev ? c0 % 32 + 4 * j - lane : lane - c0 % 32 - 4 * j, up = rev ? 1 : -1;
                  d[j] = make_float4(ps.fp * sh.pw[at & 31], ps.fp * sh.pw[(at + up) & 31], ps.fp * sh.pw[(at + 2 * up) & 31], ps.fp * sh.pw[(at + 3 * up) & 31]);
                }
              }
              // a^|i-j| = a^(distance to the block's near column) times a^(distance inside); on the diagonal the first is a^-x
              const float base = off ? sh.pw[rev ? cb * 32 - i : i - cb * 32 - 31] : near;
              const f2 base2 = pk(base, base);
              tmem_wait_ld();
              float v[W];
#pragma unroll
              for (int j = 0; j < W; j += 4) {
                upk(mul2(pk(__uint_as_float(s[j]), __uint_as_float(s[j + 1])), mul2(base2, pk(d[j / 4].x, d[j / 4].y))), v[j], v[j + 1]);
                upk(mul2(pk(__uint_as_float(s[j + 2]), __uint_as_float(s[j + 3])), mul2(base2, pk(d[j / 4].z, d[j / 4].w))), v[j + 2], v[j + 3]);
              }
              if (off == 0 || n < C) {
#pragma unroll
                for (int j = 0; j < W; ++j) v[j] = mask >> j & 1 ? v[j] : 0.f;
              }
#pragma unroll
              for (int j = 0; j < W; j += 2) r[j / 2] = pack_bf16(v[j], v[j + 1]);
            }
            tmem_st(tmem + lanes + c0 / 2, r);
          }
        } else {
#pragma unroll 1
          for (int c0 = 0; c0 < C; c0 += W) {
            uint32_t r[W / 2];
            const int cb = c0 / 32, off = rev ? cb - warp : warp - cb;  // blocks of 32 columns off the diagonal
            if (off < 0) {
#pragma unroll
              for (int j = 0; j < W / 2; ++j) r[j] = 0;
            } else {
              uint32_t s[W];
              tmem_ld(tmem + lanes + c0, s);
              float4 d[W / 4];
#pragma unroll
              for (int j = 0; j < W / 4; ++j) d[j] = *reinterpret_cast<const float4*>(&sh.col[c0 + 4 * j]);
              tmem_wait_ld();
              float v[W];
#pragma unroll
              for (int j = 0; j < W; j += 4) {
                upk(mul2(pk(__uint_as_float(s[j]), __uint_as_float(s[j + 1])), pk(d[j / 4].x, d[j / 4].y)), v[j], v[j + 1]);
                upk(mul2(pk(__uint_as_float(s[j + 2]), __uint_as_float(s[j + 3])), pk(d[j / 4].z, d[j / 4].w)), v[j + 2], v[j + 3]);
              }
              if (off == 0 || n < C) {
                const uint32_t mask = sees(off, cb, n) >> c0 % 32;
#pragma unroll
                for (int j = 0; j < W; ++j) v[j] = mask >> j & 1 ? v[j] : 0.f;
              }
#pragma unroll
              for (int j = 0; j < W; j += 2) r[j / 2] = pack_bf16(v[j], v[j + 1]);
            }
            tmem_st(tmem + lanes + c0 / 2, r);
          }
        }
        tmem_wait_st();
        arrive(sh.p);
        if (!wait(sh.o, c)) break;
        fence_after();
        const float f = i < n ? ps.fo * sh.pw[rev ? (strong ? n : C) - 1 - i : i + 1] : 0.f;
        const uint32_t to = slot(PER * c);  // (x has been read: by the scores and by O2)
        auto put = [&](const float(&x)[8], int c) {
          const uint4 q = pack8(x);
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(to + c / 64 * L::BLK + swz(i, c % 64 / 8)), "r"(q.x), "r"(q.y), "r"(q.z), "r"(q.w)
                       : "memory");
        };
        if (strong) {
#pragma unroll 1
          for (int c0 = 0; c0 < DZ; c0 += 16) {
            uint32_t u[16], v[16];
            tmem_ld(tmem + lanes + L::O + c0, u);
            tmem_ld(tmem + lanes + L::O2 + c0, v);
            tmem_wait_ld();
            if (DZ == 64 && c0 == DZ - 16) arrive(sh.read);
#pragma unroll
            for (int j = 0; j < 16; j += 8) {
              float x[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = i < n ? fmaf(f, __uint_as_float(v[j + e]), __uint_as_float(u[j + e])) : 0.f;
              put(x, c0 + j);
            }
          }
        } else {
          constexpr int V = DZ == 64 && W == 16 ? 32 : 64;  // columns at a time
#pragma unroll 1
          for (int c0 = 0; c0 < DZ; c0 += V) {
            uint32_t u[V / 32][32];
#pragma unroll
            for (int k = 0; k < V / 32; ++k) tmem_ld(tmem + lanes + L::O + c0 + 32 * k, u[k]);
            tmem_wait_ld();
            if (DZ == 64 && c0 == DZ - V) arrive(sh.read);
#pragma unroll
            for (int j = 0; j < V; j += 8) {
              float x[8];
#pragma unroll
              for (int e = 0; e < 8; ++e) x[e] = i < n ? f * __uint_as_float(u[j / 32][j % 32 + e]) : 0.f;
              put(x, c0 + j);
            }
          }
        }
        fence_proxy_async();
        arrive(sh.staged);
      }
    }
  } else if (warp < 4 || (DX == 64 ? (warp & 3) >= 2 : warp >= 12)) {
    // -------------------------------------------------------------- y to K'
    const int st = (warp < 4 ? 4 + warp : DX == 64 ? (warp & 1) + (warp >= 8 ? 2 : 0) : warp - 12) * 32 + lane;  // of 32 TW threads
    for (int c = 0; c < chunks; ++c) {
      const int t0 = start(c), n = tokens(t0), ny = PER * c + IY, nz = PER * c + IZ;
      const uint32_t y = slot(ny), z = slot(nz);
      if (!wait(sh.full[ny % RING], ny / RING)) break;
      if (n < C) {
        if (!wait(sh.full[nz % RING], nz / RING)) break;
        for (int e = st; e < (C - n) * 8 * L::ZB; e += 32 * TW) {
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
      constexpr int V = 8 * L::XB / TW;  // vectors of a thread
      bool ok = true;
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        const int g = 4 * c + i;
        if (g >= 2 && !(ok = wait(sh.kfree[g & 1], (g >> 1) - 1))) break;
        const uint32_t b1 = piece(g);
        uint4 v[V];
        float f[V];
        bool on[V];
#pragma unroll
        for (int u = 0; u < V; ++u) {  // (all loads before the first store: the compiler keeps their order)
          const int e = st + u * 32 * TW, tok = i * QTR + e % 256 / 8;
          asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];"
                       : "=r"(v[u].x), "=r"(v[u].y), "=r"(v[u].z), "=r"(v[u].w)
                       : "r"(y + e / 256 * L::BLK + i * QTR * 128 + e % 256 * 16));
          on[u] = tok < n;
          const float g1 = ps.fs * sh.pw[rev ? tok + 1 : on[u] ? n - 1 - tok : 0];  // (a load for every lane: no branch)
          f[u] = on[u] ? g1 : 0.f;
        }
        const f2 minus = pk(-1.f, -1.f);
#pragma unroll
        for (int u = 0; u < V; ++u) {
          const int e = st + u * 32 * TW;
          const uint32_t at = y + e / 256 * L::BLK + i * QTR * 128 + e % 256 * 16, lo = b1 + e / 256 * QTR * 128 + e % 256 * 16;
          const f2 f2_ = pk(f[u], f[u]);
          const uint32_t in[4] = {v[u].x, v[u].y, v[u].z, v[u].w};
          uint32_t o0[4], o1[4], o2[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t live = on[u] ? in[k] : 0u;
            // the upper halves of p and of what they leave: 8 bits of it each, 24 together
            const f2 p = mul2(pk(__uint_as_float(live << 16), __uint_as_float(live & 0xffff0000u)), f2_);
            float p0, p1;
            upk(p, p0, p1);
            o0[k] = __byte_perm(__float_as_uint(p0), __float_as_uint(p1), 0x7632);
            const f2 q = fma2(pk(__uint_as_float(o0[k] << 16), __uint_as_float(o0[k] & 0xffff0000u)), minus, p);
            float q0, q1;
            upk(q, q0, q1);
            o1[k] = __byte_perm(__float_as_uint(q0), __float_as_uint(q1), 0x7632);
            const f2 r2 = fma2(pk(__uint_as_float(o1[k] << 16), __uint_as_float(o1[k] & 0xffff0000u)), minus, q);
            float r0, r1;
            upk(r2, r0, r1);
            o2[k] = __byte_perm(__float_as_uint(r0), __float_as_uint(r1), 0x7632);
          }
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(o0[0]), "r"(o0[1]), "r"(o0[2]), "r"(o0[3]) : "memory");
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(lo), "r"(o1[0]), "r"(o1[1]), "r"(o1[2]), "r"(o1[3]) : "memory");
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(lo + L::PIECE), "r"(o2[0]), "r"(o2[1]), "r"(o2[2]), "r"(o2[3]) : "memory");
        }
        fence_proxy_async();
        arrive(sh.k[g & 1]);
      }
      if (!ok) break;
    }
  } else {
    // -------------------------------------------------------------- the state
    constexpr int N = L::COLUMNS;
    const int m = (warp & 3) * 32 + lane, j0 = (warp >= 8 ? N : 0);  // this thread's row of the state, and its columns
    const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16;
    const int dx = ps.dx, dz = ps.dz;
    const int64_t area = (int64_t)dx * dz;
    float s[N];
    {
      const float* in = SUM ? nullptr : w.segments > 1 ? ps.carry + (bh * w.segments + sg) * area : ps.init ? ps.init + bh * area : nullptr;
      const bool turned = w.segments == 1 && ps.init_t;
#pragma unroll
      for (int j = 0; j < N; ++j) s[j] = in && m < dx && j0 + j < dz ? in[turned ? (int64_t)(j0 + j) * dx + m : (int64_t)m * dz + j0 + j] : 0.f;
    }
    auto show = [&](float x) {  // x S for the next chunk's product
      if (!SUM) {
#pragma unroll
        for (int j = 0; j < N; j += 8) {
          float y[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) y[e] = x * s[j + e];
          const uint4 v = pack8(y);
          const uint32_t at = sbf + (j0 + j) / 64 * L::SBLK + swz(m, (j0 + j) % 64 / 8);
          asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
        }
        fence_proxy_async();
      }
      if (!SUM) arrive(sh.state);
    };
    // (reverse rows of P and O have the decay to place 127 taken out, the state's to the last token)
    show(rev && !strong && chunks ? __fdiv_rn(1.f, sh.pw[C - tokens(start(0))]) : 1.f);
    for (int c = 0; c < chunks; ++c) {
      if (!(SUM ? wait(sh.u[c & 1], c >> 1) : wait(sh.u[0], c))) break;
      fence_after();
      const uint32_t from = lanes + (SUM && c & 1 ? tmem : tmem + L::U);
      const float pn = sh.pw[tokens(start(c))];
      const f2 pn2 = pk(pn, pn);
#pragma unroll
      for (int cb = 0; cb < N; cb += 16) {
        uint32_t u[16];
        tmem_ld(from + j0 + cb, u);
        tmem_wait_ld();
#pragma unroll
        for (int j = 0; j < 16; j += 2)
          upk(fma2(pn2, pk(s[cb + j], s[cb + j + 1]), pk(__uint_as_float(u[j]), __uint_as_float(u[j + 1]))), s[cb + j], s[cb + j + 1]);
      }
      if (SUM) arrive(sh.ufree[c & 1]);
      else show(1.f);
    }
    float* to = SUM ? ps.carry + (bh * w.segments + sg) * area : ps.end && sg == (rev ? 0 : w.segments - 1) ? ps.end + bh * area : nullptr;
    if (to && m < dx) {
#pragma unroll
      for (int j = 0; j < N; j += 4)
        if (j0 + j < dz) *reinterpret_cast<float4*>(to + (int64_t)m * dz + j0 + j) = make_float4(s[j], s[j + 1], s[j + 2], s[j + 3]);
    }
    if (!SUM && (warp & 3) == 0) {  // a column that is not finite is so in all rows
      f2 t[4] = {0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < N; j += 2) t[j / 2 % 4] = fma2(pk(s[j], s[j + 1]), 0, t[j / 2 % 4]);
      float u, v;
      upk(add2(add2(t[0], t[1]), add2(t[2], t[3])), u, v);
      if (u + v != 0.f) sh.odd = 1;  // (NaN)
    }
  }
  fence_before();
  __syncthreads();
  if (warp == L::kMma) {
    fence_after();
    tmem_dealloc(tmem, L::COLS);
  }
  static_assert((DX * DZ + kWalkMore) * 4 <= RING * L::TILE, "room for the walk");
  if (!SUM && sh.odd && !*abort_) {
    const int3 at = cta_again();
    const int pass = at.x % w.passes, head = at.x / w.passes;
    walk<bf16>(w, w.pass[pass], head / w.heads, head % w.heads, at.y, 0, w.pass[pass].dz, C, reinterpret_cast<float*>(raw));
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
  kernel<<<dim3((unsigned)(w.batch * w.heads * w.passes), (unsigned)w.segments), Shape<DX, DZ>::NT, smem, st>>>(w, maps, word);
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
  auto encode = [&](char* map, const Rows& r, const int64_t (&size)[4]) {
    const int64_t stride[3] = {size[1] > 1 ? r.h : 64, size[2] > 1 ? r.t : 64, size[3] > 1 ? r.b : 64};
    const int box[4] = {64, 1, C, 1};
    const char* why = nullptr;
    return encode_tensor_map_4d(map, r.p, size, stride, box, &why) == 0;
  };
  auto map_of = [&](const Rows& r, int d) {
    for (int i = 0; i < n; ++i)
      if (seen[i]->p == r.p && seen[i]->b == r.b && seen[i]->t == r.t && seen[i]->h == r.h && width[i] == d) return i;
    if (n == 4) return -1;
    const int64_t size[4] = {d, r.h || w.heads == 1 ? w.heads : 1, w.time, r.b || w.batch == 1 ? w.batch : 1};
    if (!encode(maps.m[n], r, size)) return -1;
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
    const int64_t size[4] = {p.dz, w.heads, w.time, w.batch};
    if (maps.x[i] < 0 || maps.y[i] < 0 || maps.z[i] < 0 || !encode(maps.out[i], p.out, size)) {
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
