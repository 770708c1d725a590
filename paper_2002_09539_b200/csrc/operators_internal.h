// Launch wrappers of the operators on caller-owned tensors.  Arguments are checked by
// operators_api.cu before they get here.
#pragma once

#include "olsgd_internal.h"

namespace olsgd {

// ---- logprob_kernels.cu -------------------------------------------------------
struct LogprobArgs {
  const void* logits;
  int dtype;
  int64_t rows, V, ld;
  const int32_t* targets;
  int top;
  float *logp, *entropy, *stats, *top_logp;
  int32_t* top_ids;
  void* ws;
};
size_t logprob_workspace(int dtype, int64_t rows, int64_t V, int top);
cudaError_t launch_logprobs(const LogprobArgs& a, cudaStream_t s);
struct LogprobGradArgs {
  const void* logits;
  int dtype;
  int64_t rows, V, ld, ldd;
  const int32_t* targets;
  const float *stats, *entropy, *d_logp, *d_entropy;
  void* d_logits;
};
cudaError_t launch_logprobs_backward(const LogprobGradArgs& a, cudaStream_t s);

// ---- clip_kernels.cu ----------------------------------------------------------
size_t clip_workspace(int32_t m, int32_t n_tensors);
cudaError_t launch_clip(const olsgd_clip_tensor* t, int32_t n_tensors, int32_t m, float max_norm,
                        float* norms, void* ws, cudaStream_t s);

}  // namespace olsgd
