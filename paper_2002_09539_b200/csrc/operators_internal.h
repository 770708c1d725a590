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

// ---- gated_kernels.cu ---------------------------------------------------------
struct GatedOperand {      // [m][rows][cols], cols contiguous; strides in elements
  const void* p;
  int64_t worker_stride, row_stride;
};
struct GatedShape {
  int64_t m, T, D, F;
  int act;                 // olsgd_activation
  bool f16;
};
struct GatedForward : GatedShape {
  GatedOperand x, wg, wu;
  void *h, *ws;
  float* pre;
};
struct GatedBackward : GatedShape {
  GatedOperand dh, x, wg, wu;
  const float* pre;
  void *dx, *dwg, *dwu, *ws;
};
// Whether an operand has to be copied to rows that TMA takes.
bool gated_needs_copies(const GatedShape& d, const GatedOperand& x, const GatedOperand& wg, const GatedOperand& wu);
size_t gated_workspace(const GatedShape& d, bool backward, bool copies);
cudaError_t launch_gated_forward(GatedForward a, cudaStream_t s);
cudaError_t launch_gated_backward(GatedBackward a, cudaStream_t s);
// ---- embedding_kernels.cu -----------------------------------------------------
struct EmbeddingArgs {
  int dtype;
  int64_t m, T, V, D;
  const void* table;
  int64_t table_worker, table_row;
  const int32_t* ids;
  void* out;
  float scale;
};
cudaError_t launch_embedding_forward(const EmbeddingArgs& a, cudaStream_t s);
struct EmbeddingGradArgs {
  int dtype, out_dtype;
  int64_t m, T, V, D;
  const void* dout;
  int64_t dout_worker, dout_row;
  const int32_t* ids;
  float scale;
  void* dtable;
  int64_t dtable_worker;
  void* ws;
};
size_t embedding_workspace(int64_t m, int64_t T, int64_t D);
cudaError_t launch_embedding_backward(const EmbeddingGradArgs& a, cudaStream_t s);

// Joins the stream; *status: OLSGD_OK, or what a bounded wait left since the last call.
cudaError_t operators_status(int* status, cudaStream_t s);

}  // namespace olsgd
