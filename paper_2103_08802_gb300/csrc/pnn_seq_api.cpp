// C entry points of the token-sequence operators: argument checks, then the
// launch.  Nothing here touches device memory or waits for the stream.
#include <cuda_runtime.h>

#include <cmath>
#include <cstdint>
#include <map>
#include <mutex>
#include <utility>

#include "../../include/pnn.h"
#include "pnn_internal.h"
#include "pnn_seq.h"

using namespace pnn;

namespace {

constexpr int64_t kMax31 = 0x7fffffffLL;

int bad(const char* msg) { return set_last_error(PNN_EINVAL, msg); }
bool dtype_ok(int32_t d) { return d == PNN_DT_F32 || d == PNN_DT_BF16; }
size_t size_of(int32_t d) { return d == PNN_DT_BF16 ? 2 : 4; }
bool aligned(const void* p, size_t a) { return (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }
int launched(cudaError_t e) { return e == cudaSuccess ? PNN_OK : set_last_error(PNN_ECUDA, cudaGetErrorString(e)); }
int workspace_ok(const void* ws, size_t have, size_t need, const char* msg) {
  if (have < need) return set_last_error(PNN_ENOMEM, msg);
  if (need && (!ws || !aligned(ws, 256))) return bad("pnn_seq: workspace must be a 256-byte aligned device pointer");
  return PNN_OK;
}

int check_embed(const pnn_embed_args* a) {
  if (!a) return bad("pnn_embed: null arguments");
  if (a->tokens < 0 || a->tokens >= kMax31 || a->vocab <= 0 || a->vocab >= kMax31 || a->width <= 0 || a->width >= kMax31)
    return bad("pnn_embed: tokens, vocab or width out of range");
  if (a->ids_bits != 32 && a->ids_bits != 64) return bad("pnn_embed: ids are int32 or int64");
  if (a->tokens && (!a->ids || !aligned(a->ids, a->ids_bits / 8))) return bad("pnn_embed: null or misaligned ids");
  return PNN_OK;
}
int check_embed_backward(const pnn_embed_args* a) {
  const int r = check_embed(a);
  if (r) return r;
  if (!dtype_ok(a->dout_dtype) || !dtype_ok(a->dtable_dtype)) return bad("pnn_embed_backward: bad dtype");
  if ((a->dout_stride && a->dout_stride < a->width) || a->dtable_stride < a->width) return bad("pnn_embed_backward: stride below the width");
  return PNN_OK;
}

int check_recur(const pnn_recur_args* a) {
  if (!a) return bad("pnn_recur: null arguments");
  if (!dtype_ok(a->dtype)) return bad("pnn_recur: bad dtype");
  if (a->batch <= 0 || a->batch > 65535 || a->time <= 0 || a->time >= kMax31 || a->heads <= 0 || a->width <= 0 ||
      a->heads > (kMax31 - 128) / a->width)
    return bad("pnn_recur: batch (1 to 65535), time, heads or width out of range");
  return PNN_OK;
}
bool rows_ok(const void* p, int64_t sb, int64_t st, size_t esz) { return p && aligned(p, esz) && sb >= 0 && st >= 0; }
// an output's rows may not overlap: a time step is at least n wide, a sequence lies apart from the next
bool out_ok(const void* p, int64_t sb, int64_t st, int64_t n, const pnn_recur_args& a, size_t esz) {
  if (!rows_ok(p, sb, st, esz)) return false;
  if (a.time > 1 && st < n) return false;
  if (a.batch == 1) return true;
  return sb >= (a.time - 1) * st + n || (sb >= n && st >= (a.batch - 1) * sb + n);
}

int check_attend(const pnn_attend_args* a) {
  if (!a) return bad("pnn_attend: null arguments");
  if (!dtype_ok(a->dtype)) return bad("pnn_attend: bad dtype");
  if (a->batch <= 0 || a->heads <= 0 || a->batch > (1ll << 29) / a->heads || a->time <= 0 || a->time > (1ll << 30))
    return bad("pnn_attend: batch, heads (together at most 2^29) or time (1 to 2^30) out of range");
  if (a->dk <= 0 || a->dk > 256 || a->dv <= 0 || a->dv > 256) return bad("pnn_attend: dk and dv are 1 to 256");
  if (!std::isfinite(a->scale)) return bad("pnn_attend: scale must be finite");
  return PNN_OK;
}
bool head_rows_ok(const pnn_head_rows& r, size_t e) { return r.p && aligned(r.p, e) && r.stride_b >= 0 && r.stride_t >= 0 && r.stride_h >= 0; }
// rows of an output of n values, over batch, time and heads, may not overlap: sorted by stride, each axis lies
// beyond all that the ones below it span
bool head_out_ok(const pnn_head_rows& r, int64_t n, const pnn_attend_args& a, size_t e) {
  if (!head_rows_ok(r, e)) return false;
  int64_t stride[3] = {r.stride_b, r.stride_t, r.stride_h}, count[3] = {a.batch, a.time, a.heads};
  for (int i = 0; i < 3; ++i)
    for (int j = i + 1; j < 3; ++j)
      if (stride[j] < stride[i]) {
        std::swap(stride[i], stride[j]);
        std::swap(count[i], count[j]);
      }
  int64_t span = n;
  for (int i = 0; i < 3; ++i) {
    if (count[i] == 1) continue;
    if (stride[i] < span) return false;
    span += (count[i] - 1) * stride[i];
  }
  return true;
}

int check_norm(const pnn_norm_args* a) {
  if (!a) return bad("pnn_norm: null arguments");
  if (!dtype_ok(a->dtype) || !dtype_ok(a->res_dtype)) return bad("pnn_norm: bad dtype");
  if (a->rows < 0 || a->rows >= kMax31 || a->width <= 0 || a->width > 16384) return bad("pnn_norm: rows or width (1 to 16384) out of range");
  if (!(a->eps > 0.f) || !std::isfinite(a->eps)) return bad("pnn_norm: eps must be positive and finite");
  if (!std::isfinite(a->scale)) return bad("pnn_norm: scale must be finite");
  if (!aligned(a->weight, 4) || !aligned(a->scales, 4) || !aligned(a->next_weight, 4)) return bad("pnn_norm: misaligned weights");
  return PNN_OK;
}
bool in_rows(const pnn_rows& r, size_t e) { return r.p && aligned(r.p, e) && r.stride >= 0; }
bool maybe_rows(const pnn_rows& r, size_t e) { return !r.p || in_rows(r, e); }
bool out_rows(const pnn_rows& r, const pnn_norm_args& a, size_t e) { return in_rows(r, e) && (a.rows <= 1 || r.stride >= a.width); }
}  // namespace

extern "C" {

int pnn_seq_sync(void* stream) {
  int dev = 0, count = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e == cudaSuccess) e = seq_give_ups(&count, static_cast<cudaStream_t>(stream));
  if (e != cudaSuccess) return launched(e);
  try {
    // A device's streams share one count; each stream has its own last sight of it.
    static std::mutex lock;
    static std::map<std::pair<int, void*>, int> seen;
    const std::lock_guard<std::mutex> hold(lock);
    int& last = seen[{dev, stream}];
    const bool more = count != last;
    last = count;
    return more ? set_last_error(PNN_ETIMEOUT, "pnn_seq_sync: a device wait timed out; outputs since this stream's last call may be incomplete") : PNN_OK;
  } catch (...) {
    return set_last_error(PNN_ENOMEM, "pnn_seq_sync: out of host memory");
  }
}

int pnn_selftest_seq_timeout(int64_t limit_ns, void* stream) {
  if (limit_ns <= 0 || limit_ns > 10000000000ll) return bad("pnn_selftest_seq_timeout: limit_ns must be in (0, 1e10]");
  return launched(launch_seq_timeout(limit_ns, static_cast<cudaStream_t>(stream)));
}

int pnn_embed_forward(const pnn_embed_args* a, void* stream) {
  const int r = check_embed(a);
  if (r) return r;
  if (!dtype_ok(a->table_dtype) || !dtype_ok(a->out_dtype)) return bad("pnn_embed_forward: bad dtype");
  if (a->tokens == 0) return PNN_OK;
  if (a->table_stride < 0 || a->out_stride < a->width) return bad("pnn_embed_forward: stride below the width");
  if (!a->table || !a->out || !aligned(a->table, size_of(a->table_dtype)) || !aligned(a->out, size_of(a->out_dtype)))
    return bad("pnn_embed_forward: null or misaligned table or output");
  return launched(launch_embed_fwd(*a, static_cast<cudaStream_t>(stream)));
}

int pnn_embed_workspace_bytes(const pnn_embed_args* a, size_t* bytes) {
  if (!bytes) return bad("pnn_embed_workspace_bytes: null output");
  const int r = check_embed_backward(a);
  if (r) return r;
  *bytes = embed_workspace(*a);
  return PNN_OK;
}

int pnn_embed_backward(const pnn_embed_args* a, void* ws, size_t ws_bytes, void* stream) {
  int r = check_embed_backward(a);
  if (r) return r;
  if (!a->dtable || !aligned(a->dtable, size_of(a->dtable_dtype)))
    return bad("pnn_embed_backward: null or misaligned dtable");
  if (a->tokens && (!a->dout || !aligned(a->dout, size_of(a->dout_dtype))))
    return bad("pnn_embed_backward: null or misaligned dout");
  if (a->tokens == 0 && a->accumulate) return PNN_OK;
  r = workspace_ok(ws, ws_bytes, embed_workspace(*a), "pnn_embed_backward: workspace too small");
  if (r) return r;
  return launched(launch_embed_bwd(*a, ws, static_cast<cudaStream_t>(stream)));
}

int pnn_recur_saved_size(const pnn_recur_args* a, size_t* floats) {
  if (!floats) return bad("pnn_recur_saved_size: null output");
  const int r = check_recur(a);
  if (r) return r;
  *floats = recur_saved_floats(*a);
  return PNN_OK;
}

int pnn_recur_workspace_bytes(const pnn_recur_args* a, int32_t backward, size_t* bytes) {
  if (!bytes) return bad("pnn_recur_workspace_bytes: null output");
  const int r = check_recur(a);
  if (r) return r;
  *bytes = recur_workspace(*a, backward != 0);
  return PNN_OK;
}

int pnn_recur_forward(const pnn_recur_args* a, void* ws, size_t ws_bytes, void* stream) {
  int r = check_recur(a);
  if (r) return r;
  const size_t e = size_of(a->dtype);
  if (!rows_ok(a->z, a->z_stride_b, a->z_stride_t, e) || !rows_ok(a->x, a->x_stride_b, a->x_stride_t, e))
    return bad("pnn_recur_forward: null or misaligned z or x, or a negative stride");
  if (!out_ok(a->h, a->h_stride_b, a->h_stride_t, a->heads * a->width, *a, e))
    return bad("pnn_recur_forward: null or misaligned h, or overlapping rows");
  if (!aligned(a->h0, 4) || !aligned(a->h_last, 4) || !aligned(a->saved, 4) || !aligned(a->lengths, 4))
    return bad("pnn_recur_forward: misaligned pointer");
  r = workspace_ok(ws, ws_bytes, recur_workspace(*a, false), "pnn_recur_forward: workspace too small");
  if (r) return r;
  return launched(launch_recur_fwd(*a, ws, static_cast<cudaStream_t>(stream)));
}

int pnn_recur_backward(const pnn_recur_args* a, void* ws, size_t ws_bytes, void* stream) {
  int r = check_recur(a);
  if (r) return r;
  const size_t e = size_of(a->dtype);
  if (!rows_ok(a->z, a->z_stride_b, a->z_stride_t, e) || !rows_ok(a->x, a->x_stride_b, a->x_stride_t, e) ||
      !rows_ok(a->dh, a->dh_stride_b, a->dh_stride_t, e))
    return bad("pnn_recur_backward: null or misaligned z, x or dh, or a negative stride");
  if (!out_ok(a->dz, a->dz_stride_b, a->dz_stride_t, a->heads, *a, e) ||
      !out_ok(a->dx, a->dx_stride_b, a->dx_stride_t, a->heads * a->width, *a, e))
    return bad("pnn_recur_backward: null or misaligned dz or dx, or overlapping rows");
  if (!a->saved || !aligned(a->saved, 4)) return bad("pnn_recur_backward: needs what the forward saved");
  if (!aligned(a->dh_last, 4) || !aligned(a->dh0, 4) || !aligned(a->lengths, 4))
    return bad("pnn_recur_backward: misaligned pointer");
  r = workspace_ok(ws, ws_bytes, recur_workspace(*a, true), "pnn_recur_backward: workspace too small");
  if (r) return r;
  return launched(launch_recur_bwd(*a, ws, static_cast<cudaStream_t>(stream)));
}

int pnn_recur_step(const pnn_recur_step_args* a, void* stream) {
  if (!a) return bad("pnn_recur_step: null arguments");
  if (!dtype_ok(a->dtype)) return bad("pnn_recur_step: bad dtype");
  if (a->batch < 0 || a->batch > 65535 || a->slots < 0 || a->slots >= kMax31 || a->heads <= 0 || a->width <= 0 ||
      a->heads > kMax31 / a->width)
    return bad("pnn_recur_step: batch (0 to 65535), slots, heads or width out of range");
  if (a->batch == 0) return PNN_OK;
  const size_t e = size_of(a->dtype);
  if (!rows_ok(a->z, 0, a->z_stride, e) || !rows_ok(a->x, 0, a->x_stride, e) || !rows_ok(a->h, 0, a->h_stride, e))
    return bad("pnn_recur_step: null or misaligned z, x or h, or a negative stride");
  if (!a->slot && a->slots < a->batch) return bad("pnn_recur_step: fewer slots than sequences and no slot list");
  if ((a->slots && !a->state) || !aligned(a->state, 4) || !aligned(a->slot, 4))
    return bad("pnn_recur_step: null or misaligned state or slot");
  if (a->state_stride < a->heads * a->width || (a->batch > 1 && a->h_stride < a->heads * a->width))
    return bad("pnn_recur_step: overlapping rows of state or h");
  return launched(launch_recur_step(*a, static_cast<cudaStream_t>(stream)));
}

int pnn_distill(const pnn_distill_args* a, void* stream) {
  if (!a) return bad("pnn_distill: null arguments");
  if (a->rows < 0 || a->rows >= kMax31 || a->vocab <= 0 || a->vocab >= kMax31) return bad("pnn_distill: rows or vocab out of range");
  if (!dtype_ok(a->dtype) || (a->k > 0 && !dtype_ok(a->teacher_dtype))) return bad("pnn_distill: bad dtype");
  if (a->k < 0 || a->k > 1024) return bad("pnn_distill: k is 0 to 1024");
  // (the kernels' factor log2(e) / tau is finite too)
  if (!(a->tau > 0.f) || !std::isfinite(a->tau) || !std::isfinite(1.5f / a->tau))
    return bad("pnn_distill: tau must be positive and finite, and so must 1.5 / tau");
  if (!(a->alpha >= 0.f && a->alpha <= 1.f)) return bad("pnn_distill: alpha is 0 to 1");
  if (a->rows == 0) return PNN_OK;
  const size_t e = size_of(a->dtype);
  if (!a->logits || !aligned(a->logits, e) || a->logits_stride < 0) return bad("pnn_distill: null or misaligned logits, or a negative stride");
  if (a->k > 0 && (!a->ids || !a->teacher || !aligned(a->ids, 4) || !aligned(a->teacher, size_of(a->teacher_dtype))))
    return bad("pnn_distill: null or misaligned ids or teacher");
  if (!a->loss || !aligned(a->loss, 4) || !aligned(a->labels, 4) || !aligned(a->weight, 4))
    return bad("pnn_distill: null loss or misaligned pointer");
  if (a->dlogits && (!aligned(a->dlogits, e) || (a->rows > 1 && a->dlogits_stride < a->vocab)))
    return bad("pnn_distill: misaligned dlogits or overlapping rows");
  if (a->dlogits == a->logits && a->dlogits && a->dlogits_stride != a->logits_stride)
    return bad("pnn_distill: a gradient in place of the logits has their stride");
  return launched(launch_distill(*a, static_cast<cudaStream_t>(stream)));
}

int pnn_attend_workspace_bytes(const pnn_attend_args* a, int32_t backward, size_t* bytes) {
  if (!bytes) return bad("pnn_attend_workspace_bytes: null output");
  const int r = check_attend(a);
  if (r) return r;
  *bytes = attend_workspace(*a, backward != 0);
  return PNN_OK;
}

int pnn_attend_forward(const pnn_attend_args* a, void* ws, size_t ws_bytes, void* stream) {
  int r = check_attend(a);
  if (r) return r;
  const size_t e = size_of(a->dtype);
  if (!head_rows_ok(a->q, e) || !head_rows_ok(a->k, e) || !head_rows_ok(a->v, e))
    return bad("pnn_attend_forward: null or misaligned q, k or v, or a negative stride");
  if (!head_out_ok(a->o, a->dv, *a, e)) return bad("pnn_attend_forward: null or misaligned o, or overlapping rows");
  if (!a->decay || !aligned(a->decay, 4) || !aligned(a->lengths, 4) || !aligned(a->s0, 4) || !aligned(a->s_last, 4))
    return bad("pnn_attend_forward: null decay or misaligned pointer");
  r = workspace_ok(ws, ws_bytes, attend_workspace(*a, false), "pnn_attend_forward: workspace too small");
  if (r) return r;
  return launched(launch_attend(*a, false, ws, static_cast<cudaStream_t>(stream)));
}

int pnn_attend_backward(const pnn_attend_args* a, void* ws, size_t ws_bytes, void* stream) {
  int r = check_attend(a);
  if (r) return r;
  const size_t e = size_of(a->dtype);
  if (!head_rows_ok(a->q, e) || !head_rows_ok(a->k, e) || !head_rows_ok(a->v, e) || !head_rows_ok(a->dout, e))
    return bad("pnn_attend_backward: null or misaligned q, k, v or dout, or a negative stride");
  if (!head_out_ok(a->dq, a->dk, *a, e) || !head_out_ok(a->dk_out, a->dk, *a, e) || !head_out_ok(a->dv_out, a->dv, *a, e))
    return bad("pnn_attend_backward: null or misaligned dq, dk or dv, or overlapping rows");
  if (!a->decay || !aligned(a->decay, 4) || !aligned(a->lengths, 4) || !aligned(a->s0, 4) || !aligned(a->ds_last, 4) || !aligned(a->ds0, 4))
    return bad("pnn_attend_backward: null decay or misaligned pointer");
  r = workspace_ok(ws, ws_bytes, attend_workspace(*a, true), "pnn_attend_backward: workspace too small");
  if (r) return r;
  return launched(launch_attend(*a, true, ws, static_cast<cudaStream_t>(stream)));
}

int pnn_attend_step(const pnn_attend_step_args* a, void* stream) {
  if (!a) return bad("pnn_attend_step: null arguments");
  if (!dtype_ok(a->dtype)) return bad("pnn_attend_step: bad dtype");
  if (a->batch < 0 || a->batch > 65535 || a->slots < 0 || a->slots >= kMax31 || a->heads <= 0 || a->heads > 32767)
    return bad("pnn_attend_step: batch (0 to 65535), slots or heads (1 to 32767) out of range");
  if (a->dk <= 0 || a->dk > 256 || a->dv <= 0 || a->dv > 256) return bad("pnn_attend_step: dk and dv are 1 to 256");
  if (!std::isfinite(a->scale)) return bad("pnn_attend_step: scale must be finite");
  if (a->batch == 0) return PNN_OK;
  const size_t e = size_of(a->dtype);
  if (!rows_ok(a->q, a->q_stride_b, a->q_stride_h, e) || !rows_ok(a->k, a->k_stride_b, a->k_stride_h, e) ||
      !rows_ok(a->v, a->v_stride_b, a->v_stride_h, e) || !rows_ok(a->o, a->o_stride_b, a->o_stride_h, e))
    return bad("pnn_attend_step: null or misaligned q, k, v or o, or a negative stride");
  if (!a->slot && a->slots < a->batch) return bad("pnn_attend_step: fewer slots than sequences and no slot list");
  if ((a->slots && !a->state) || !aligned(a->state, 4) || !aligned(a->slot, 4) || !a->decay || !aligned(a->decay, 4))
    return bad("pnn_attend_step: null or misaligned state, slot or decay");
  if (a->state_stride < a->heads * a->dk * a->dv) return bad("pnn_attend_step: overlapping states");
  if (a->heads > 1 && a->o_stride_h < a->dv) return bad("pnn_attend_step: overlapping rows of o");
  if (a->batch > 1 && a->o_stride_b < (a->heads - 1) * a->o_stride_h + a->dv && (a->o_stride_b < a->dv || a->o_stride_h < (a->batch - 1) * a->o_stride_b + a->dv))
    return bad("pnn_attend_step: overlapping rows of o");
  return launched(launch_attend_step(*a, static_cast<cudaStream_t>(stream)));
}

int pnn_norm_forward(const pnn_norm_args* a, void* stream) {
  const int r = check_norm(a);
  if (r) return r;
  if (a->rows == 0) return PNN_OK;
  const size_t e = size_of(a->dtype), f = size_of(a->res_dtype);
  if (!in_rows(a->x, e) || !maybe_rows(a->gate, e) || !maybe_rows(a->res, f)) return bad("pnn_norm_forward: null or misaligned x, gate or res, or a negative stride");
  if (!out_rows(a->h, *a, f) || (a->next_weight && !out_rows(a->n, *a, e))) return bad("pnn_norm_forward: null or misaligned h or n, or overlapping rows");
  return launched(launch_norm(*a, false, nullptr, static_cast<cudaStream_t>(stream)));
}

int pnn_norm_workspace_bytes(const pnn_norm_args* a, size_t* bytes) {
  if (!bytes) return bad("pnn_norm_workspace_bytes: null output");
  const int r = check_norm(a);
  if (r) return r;
  *bytes = norm_workspace(*a);
  return PNN_OK;
}

int pnn_norm_backward(const pnn_norm_args* a, void* ws, size_t ws_bytes, void* stream) {
  int r = check_norm(a);
  if (r) return r;
  const size_t e = size_of(a->dtype), f = size_of(a->res_dtype);
  if ((a->dweight && !a->weight) || (a->dscales && !a->scales) || (a->dnext_weight && !a->next_weight) || (a->dgate.p && !a->gate.p))
    return bad("pnn_norm_backward: the gradient of what is not there");
  if (!aligned(a->dweight, 4) || !aligned(a->dscales, 4) || !aligned(a->dnext_weight, 4)) return bad("pnn_norm_backward: misaligned gradients of the weights");
  if (a->rows) {
    if (!in_rows(a->x, e) || !maybe_rows(a->gate, e) || !maybe_rows(a->res, f) || !maybe_rows(a->dh, f) || (a->next_weight && !in_rows(a->dn, e)))
      return bad("pnn_norm_backward: null or misaligned x, gate, res, dh or dn, or a negative stride");
    if (!out_rows(a->dx, *a, e) || (a->dgate.p && !out_rows(a->dgate, *a, e)) || (a->dres.p && !out_rows(a->dres, *a, f)))
      return bad("pnn_norm_backward: null or misaligned dx, dgate or dres, or overlapping rows");
  }
  r = workspace_ok(ws, ws_bytes, norm_workspace(*a), "pnn_norm_backward: workspace too small");
  if (r) return r;
  return launched(launch_norm(*a, true, ws, static_cast<cudaStream_t>(stream)));
}

int pnn_policy(const pnn_policy_args* a, void* stream) {
  if (!a) return bad("pnn_policy: null arguments");
  if (a->rows < 0 || a->rows >= kMax31 || a->vocab <= 0 || a->vocab >= kMax31) return bad("pnn_policy: rows or vocab out of range");
  if (!dtype_ok(a->dtype)) return bad("pnn_policy: bad dtype");
  if (!(a->tau > 0.f) || !std::isfinite(a->tau) || !std::isfinite(1.5f / a->tau))
    return bad("pnn_policy: tau must be positive and finite, and so must 1.5 / tau");
  if (!(a->clip_low >= 0.f && a->clip_low <= 1.f) || !(a->clip_high >= 0.f)) return bad("pnn_policy: clip_low is 0 to 1, clip_high not negative");
  if (!(a->beta >= 0.f) || !std::isfinite(a->beta)) return bad("pnn_policy: beta must be finite and not negative");
  if (a->rows == 0) return PNN_OK;
  const size_t e = size_of(a->dtype);
  if (!a->logits || !aligned(a->logits, e) || a->logits_stride < 0) return bad("pnn_policy: null or misaligned logits, or a negative stride");
  if (!a->labels || !a->advantage || !a->loss) return bad("pnn_policy: null labels, advantage or loss");
  if (!aligned(a->labels, 4) || !aligned(a->advantage, 4) || !aligned(a->old, 4) || !aligned(a->ref, 4) || !aligned(a->weight, 4) || !aligned(a->loss, 4) ||
      !aligned(a->logp, 4))
    return bad("pnn_policy: misaligned pointer");
  if (a->dlogits && (!aligned(a->dlogits, e) || (a->rows > 1 && a->dlogits_stride < a->vocab)))
    return bad("pnn_policy: misaligned dlogits or overlapping rows");
  if (a->dlogits == a->logits && a->dlogits && a->dlogits_stride != a->logits_stride)
    return bad("pnn_policy: a gradient in place of the logits has their stride");
  return launched(launch_policy(*a, static_cast<cudaStream_t>(stream)));
}

}  // extern "C"
