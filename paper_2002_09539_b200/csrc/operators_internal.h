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

// ---- expert_kernels.cu --------------------------------------------------------
struct RouteArgs {
  int dtype;
  int64_t m, T, E;
  const void* logits;
  int64_t ld;
  int k, normalise;
  float* weights;
  int32_t *ids, *places, *tokens, *offsets;
  void* ws;
};
size_t route_workspace(int64_t m, int64_t T, int64_t E);
cudaError_t launch_route(const RouteArgs& a, cudaStream_t s);
struct RouteGradArgs {
  int dtype;
  int64_t rows;
  int E, k, normalise;
  const void* logits;
  int64_t ld;
  const int32_t* ids;
  const float *weights, *d_weights;
  void* d_logits;
};
cudaError_t launch_route_backward(const RouteGradArgs& a, cudaStream_t s);
struct CombineArgs {
  int dtype, k;
  int64_t m, T, R, D;
  const void* rows;
  int64_t rows_worker, rows_row;
  const int32_t* places;
  const float* weights;
  void* y;
  const void* rows_end;      // (set by the launch)
};
cudaError_t launch_combine(const CombineArgs& a, cudaStream_t s);
struct CombineGradArgs {
  int dtype, k;
  int64_t m, T, R, D;
  const void* d_y;
  int64_t dy_worker, dy_row;
  const void* rows;
  int64_t rows_worker, rows_row;
  const int32_t *places, *tokens;
  const float* weights;
  void* d_rows;
  float* d_weights;
  const void *rows_end, *dy_end;   // (set by the launch)
};
cudaError_t launch_combine_backward(const CombineGradArgs& a, cudaStream_t s);

// ---- product_kernels.cu -------------------------------------------------------
struct ProductShape {
  int64_t m, R, E, D, F;
  bool f16;
};
struct ExpertOperand {     // [m][E][rows][cols], cols contiguous; strides in elements
  const void* p;
  int64_t worker_stride, expert_stride, row_stride;
};
struct ProductForward : ProductShape {
  GatedOperand x;
  ExpertOperand w;
  const int32_t* offsets;
  void *y, *ws;
};
struct ProductBackward : ProductShape {
  GatedOperand dy, x;
  ExpertOperand w;
  const int32_t* offsets;
  void *dx, *dw, *ws;
};
// Whether an operand has to be copied to rows that TMA takes (dy: of the backward call).
bool product_needs_copies(const ProductShape& d, const GatedOperand& x, const ExpertOperand& w, const GatedOperand* dy);
size_t product_workspace(const ProductShape& d, bool backward, bool copies);
cudaError_t launch_product(ProductForward a, cudaStream_t s);
cudaError_t launch_product_backward(ProductBackward a, cudaStream_t s);

// ---- distill_kernels.cu -------------------------------------------------------
struct DistillArgs {
  const void* logits;
  int dtype;
  int64_t rows, V, ld;
  const int32_t* ids;
  const void* teacher;
  int teacher_dtype, K;
  float inv_t;               // 1 / temperature
  const float* d_loss;       // or null: no gradient
  float *loss, *stats;
  void* d_logits;
  int64_t ldd;
  void* ws;
  int* status;               // (set by the launch)
};
size_t distill_workspace(int dtype, int64_t rows, int64_t V, int K, bool gradient);
cudaError_t launch_distill(const DistillArgs& a, cudaStream_t s);
cudaError_t launch_distill_backward(const DistillArgs& a, cudaStream_t s);

// One word of the current device, which takes OLSGD_ETIMEOUT where a bounded wait of any operator gives up.
cudaError_t status_word(int** word);
// Joins the stream; *status: OLSGD_OK, or what a bounded wait left since the last call.
cudaError_t operators_status(int* status, cudaStream_t s);

}  // namespace olsgd
