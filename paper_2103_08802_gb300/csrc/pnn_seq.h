// Launchers of the token-sequence operators (embedding, gated recurrence,
// distillation, linear attention, norms, policy loss).  The arguments are checked by pnn_seq_api.cpp.
#pragma once
#include <cuda_runtime.h>

#include "../../include/pnn.h"

namespace pnn {

cudaError_t launch_embed_fwd(const pnn_embed_args& a, cudaStream_t st);
size_t embed_workspace(const pnn_embed_args& a);
cudaError_t launch_embed_bwd(const pnn_embed_args& a, void* ws, cudaStream_t st);

size_t recur_saved_floats(const pnn_recur_args& a);
size_t recur_workspace(const pnn_recur_args& a, bool backward);
cudaError_t launch_recur_fwd(const pnn_recur_args& a, void* ws, cudaStream_t st);
cudaError_t launch_recur_bwd(const pnn_recur_args& a, void* ws, cudaStream_t st);
cudaError_t launch_recur_step(const pnn_recur_step_args& a, cudaStream_t st);
// Device word that counts the bounded waits that gave up (NULL: a CUDA error);
// the count, once the stream has finished; a kernel whose wait gives up after limit_ns.
int* seq_gave_up_word();
cudaError_t seq_give_ups(int* count, cudaStream_t st);
cudaError_t launch_seq_timeout(int64_t limit_ns, cudaStream_t st);

cudaError_t launch_distill(const pnn_distill_args& a, cudaStream_t st);

size_t attend_workspace(const pnn_attend_args& a, bool back);
cudaError_t launch_attend(const pnn_attend_args& a, bool back, void* ws, cudaStream_t st);
cudaError_t launch_attend_step(const pnn_attend_step_args& a, cudaStream_t st);

size_t norm_workspace(const pnn_norm_args& a);
cudaError_t launch_norm(const pnn_norm_args& a, bool back, void* ws, cudaStream_t st);

cudaError_t launch_policy(const pnn_policy_args& a, cudaStream_t st);

}  // namespace pnn
