// Gated linear recurrence: how a call is laid out over the GPU, the sum of a
// wide head's gate gradient, and the single-token step.
#include "recur_tile.cuh"

namespace pnn {
namespace {
using namespace recur;

__device__ int g_gave_up;  // bounded waits that expired, of all the token-sequence kernels

// A wait that runs out on purpose: its barrier expects two arrivals and gets one.
__global__ void k_seq_timeout(unsigned long long limit_ns, int* gave_up) {
  __shared__ uint64_t bar;
  __shared__ int abort_;
  if (threadIdx.x) return;
  abort_ = 0;
  mbar_init(smem_u32(&bar), 2);
  asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  mbar_arrive(smem_u32(&bar));
  if (!mbar_wait_for(smem_u32(&bar), 0, &abort_, limit_ns)) count_give_up(gave_up);
}

// dz of a head: the sum of its `parts` parts
template <typename T>
__global__ void k_recur_dz(pnn_recur_args a, const float* part, int64_t parts) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, total = a.batch * a.time * a.heads;
  if (i >= total) return;
  const int64_t k = i % a.heads, bt = i / a.heads;
  const float* p = part + i * parts;
  float s = 0.f;
  for (int64_t j = 0; j < parts; ++j) s += p[j];
  st(static_cast<T*>(a.dz) + bt / a.time * a.dz_stride_b + bt % a.time * a.dz_stride_t + k, s);
}

// the same for heads of any width that reach from one tile into the next ones
template <typename T>
__global__ void k_recur_dz_spread(pnn_recur_args a, const float* part, int tiles) {
  const int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= a.batch * a.time * (tiles - 1)) return;
  const int64_t bt = i / (tiles - 1), j = i % (tiles - 1), W = a.width, k = ((j + 1) * kTile - 1) / W;  // the head of tile j's last channel
  const int64_t last = ((k + 1) * W - 1) / kTile;
  if (k * W < j * kTile || last == j) return;  // begins in an earlier tile, or ends in this one
  const float* p = part + (bt * tiles + j) * 2;
  float s = p[1];
  for (int64_t q = j + 1; q <= last; ++q) s += p[(q - j) * 2];
  st(static_cast<T*>(a.dz) + bt / a.time * a.dz_stride_b + bt % a.time * a.dz_stride_t + k, s);
}

template <typename T>
__global__ void k_recur_step(pnn_recur_step_args a) {
  const int64_t D = a.heads * a.width, c = (int64_t)blockIdx.x * blockDim.x + threadIdx.x, i = blockIdx.y;
  if (c >= D) return;
  const int64_t k = a.slot ? (int64_t)a.slot[i] : i;
  float v = 0.f;
  if (k >= 0 && k < a.slots) {
    float* s = a.state + k * a.state_stride + c;
    const float2 f = gate1(ld(static_cast<const T*>(a.z) + i * a.z_stride + c / a.width));
    v = fmaf(f.x, *s, f.y * ld(static_cast<const T*>(a.x) + i * a.x_stride + c));
    *s = v;
  }
  st(static_cast<T*>(a.h) + i * a.h_stride + c, v);
}

// steps of a piece: the same for a forward and its backward, whatever their alignment
int piece_of(const pnn_recur_args& a) {
  if (a.width % 8 == 0) return a.dtype == PNN_DT_BF16 ? Geo<bf16, HEAD, FWD>::L : Geo<float, HEAD, FWD>::L;
  static_assert(Geo<bf16, OWN, FWD>::L == Geo<bf16, SPREAD, FWD>::L && Geo<float, OWN, FWD>::L == Geo<float, SPREAD, FWD>::L, "");
  return a.dtype == PNN_DT_BF16 ? Geo<bf16, OWN, FWD>::L : Geo<float, OWN, FWD>::L;
}
int64_t pieces_of(const pnn_recur_args& a) { return (a.time + piece_of(a) - 1) / piece_of(a); }
int64_t tiles_of(const pnn_recur_args& a) { return (a.heads * a.width + kTile - 1) / kTile; }

// HEAD: channels whose dz one CTA sums, as many as divide a head and lie in its tile.
int part_width(const pnn_recur_args& a) {
  for (int w = 64; w >= 8; w /= 2)
    if (a.width % w == 0) return w;
  return 0;
}

// Segments along time.  Measured, a CTA takes a piece in 0.85 us (backward 1.5,
// with a shared gate 2.6) alone on its SM and in 1.2 (2.1, 2.6) beside another
// one; split in segments it walks it twice, the first time in 1.0 us, with one
// launch more.
void split(const pnn_recur_args& a, bool backward, Plan& pl) {
  const int64_t pieces = pieces_of(a), chains = tiles_of(a) * a.batch, slots = 2 * (int64_t)device_sm_count();
  pl.segments = 1;
  pl.per = (int)pieces;
  if (chains * 2 > slots) return;
  const int64_t per = (pieces + slots / chains - 1) / (slots / chains), segs = (pieces + per - 1) / per;
  const bool own = a.width == 1;
  const double whole = (double)pieces * (!backward ? 0.85 : own ? 1.5 : 2.6), parts = (double)per * (!backward ? 2.2 : own ? 3.1 : 3.6) + 4.0;
  if (whole <= parts) return;
  pl.segments = (int)segs;
  pl.per = (int)per;
}

size_t sums_bytes(const pnn_recur_args& a, const Plan& pl) {
  return pl.segments > 1 ? (size_t)a.batch * pl.segments * tiles_of(a) * 32 * sizeof(ulonglong2) : 0;
}
size_t part_bytes(const pnn_recur_args& a) {
  const int pw = part_width(a);
  if (a.width == 1 || a.width == pw) return 0;
  if (!pw) return (size_t)a.batch * a.time * tiles_of(a) * 2 * 4;
  return (size_t)a.batch * a.time * (a.heads * a.width / pw) * 4;
}

// A small kernel that leaves an SM's memory divided as the large ones around it
// have it: dividing it anew each time took 30 us of a short backward pass.
cudaError_t keep_shared(const void* kernel, int which) {
  static std::atomic<uint64_t> ready[4];  // one bit a device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (e != cudaSuccess || ready[which].load(std::memory_order_acquire) & bit) return e;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributePreferredSharedMemoryCarveout, cudaSharedmemCarveoutMaxShared);
  if (e == cudaSuccess) ready[which].fetch_or(bit, std::memory_order_release);
  return e;
}

cudaError_t run(bool backward, const pnn_recur_args& a, void* ws, cudaStream_t st) {
  Plan pl{};
  split(a, backward, pl);
  pl.pw = part_width(a);
  pl.sums = static_cast<ulonglong2*>(ws);
  pl.part = backward && part_bytes(a) ? reinterpret_cast<float*>(static_cast<char*>(ws) + sums_bytes(a, pl)) : nullptr;
  int* word = seq_gave_up_word();
  if (!word) return cudaGetLastError();
  const bool half = a.dtype == PNN_DT_BF16;
  cudaError_t e = backward ? (half ? run_bwd_bf16(a, pl, word, st) : run_bwd_f32(a, pl, word, st))
                           : (half ? run_fwd_bf16(a, pl, word, st) : run_fwd_f32(a, pl, word, st));
  if (e != cudaSuccess || !pl.part) return e;
  const int tiles = (int)tiles_of(a);
  if (!pl.pw && (tiles == 1 || kTile % a.width == 0)) return e;  // no head reaches into another tile
  const int64_t total = a.batch * a.time * (pl.pw ? a.heads : tiles - 1);
  const unsigned g = (unsigned)((total + 255) / 256);
  if (pl.pw) {
    const auto kernel = half ? k_recur_dz<bf16> : k_recur_dz<float>;
    if ((e = keep_shared(reinterpret_cast<const void*>(kernel), half)) != cudaSuccess) return e;
    kernel<<<g, 256, 0, st>>>(a, pl.part, a.width / pl.pw);
  } else {
    const auto kernel = half ? k_recur_dz_spread<bf16> : k_recur_dz_spread<float>;
    if ((e = keep_shared(reinterpret_cast<const void*>(kernel), 2 + half)) != cudaSuccess) return e;
    kernel<<<g, 256, 0, st>>>(a, pl.part, tiles);
  }
  return cudaGetLastError();
}
}  // namespace

int* seq_gave_up_word() {
  static std::atomic<int*> at[64];  // of each device
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return nullptr;
  int* known = dev < 64 ? at[dev].load(std::memory_order_acquire) : nullptr;
  if (known) return known;
  void* p = nullptr;
  if (cudaGetSymbolAddress(&p, g_gave_up) != cudaSuccess) return nullptr;
  if (dev < 64) at[dev].store(static_cast<int*>(p), std::memory_order_release);
  return static_cast<int*>(p);
}

size_t recur_saved_floats(const pnn_recur_args& a) { return (size_t)a.batch * pieces_of(a) * a.heads * a.width; }
size_t recur_workspace(const pnn_recur_args& a, bool backward) {
  Plan pl{};
  split(a, backward, pl);
  return sums_bytes(a, pl) + (backward ? part_bytes(a) : 0);
}
cudaError_t launch_recur_fwd(const pnn_recur_args& a, void* ws, cudaStream_t st) { return run(false, a, ws, st); }
cudaError_t launch_recur_bwd(const pnn_recur_args& a, void* ws, cudaStream_t st) { return run(true, a, ws, st); }

cudaError_t launch_recur_step(const pnn_recur_step_args& a, cudaStream_t st) {
  const dim3 g((unsigned)((a.heads * a.width + 127) / 128), (unsigned)a.batch);
  if (a.dtype == PNN_DT_BF16) k_recur_step<bf16><<<g, 128, 0, st>>>(a);
  else k_recur_step<float><<<g, 128, 0, st>>>(a);
  return cudaGetLastError();
}

cudaError_t seq_give_ups(int* count, cudaStream_t st) {
  const cudaError_t e = cudaMemcpyFromSymbolAsync(count, g_gave_up, sizeof(int), 0, cudaMemcpyDeviceToHost, st);
  return e == cudaSuccess ? cudaStreamSynchronize(st) : e;
}

cudaError_t launch_seq_timeout(int64_t limit_ns, cudaStream_t st) {
  int* word = seq_gave_up_word();
  if (!word) return cudaGetLastError();
  k_seq_timeout<<<1, 32, 0, st>>>((unsigned long long)limit_ns, word);
  return cudaGetLastError();
}

}  // namespace pnn
