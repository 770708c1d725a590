// C ABI of the operators on caller-owned tensors: argument checks, then one launch wrapper
// each.  Nothing is allocated, nothing is kept between calls, nothing throws.
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "operators_internal.h"

using namespace olsgd;

namespace {

olsgd_status refuse(olsgd_status st, const char* fmt, ...) {
  char buf[256];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  set_thread_error(buf);
  return st;
}

olsgd_status launched(cudaError_t e, const char* what) {
  if (e == cudaSuccess) return OLSGD_OK;
  return refuse(OLSGD_ECUDA, "%s: %s", what, cudaGetErrorString(e));
}

int elem_size(int32_t dtype) { return dtype == OLSGD_F32 ? 4 : 2; }
bool is_dtype(int32_t d) { return d == OLSGD_F32 || d == OLSGD_BF16 || d == OLSGD_F16; }
bool aligned_to(const void* p, size_t a) { return p && (reinterpret_cast<uintptr_t>(p) & (a - 1)) == 0; }

#define OLSGD_REFUSE_IF(cond, ...) \
  do {                             \
    if (cond) return refuse(OLSGD_EINVAL, __VA_ARGS__); \
  } while (0)

#define OLSGD_TRY(call)                      \
  do {                                       \
    const olsgd_status st_ = (call);         \
    if (st_ != OLSGD_OK) return st_;         \
  } while (0)

constexpr int64_t kMaxVocab = 1LL << 27;
constexpr int64_t kMaxRows = 0x7FFFFFFF;

olsgd_status check_rows(int32_t dtype, int64_t rows, int64_t V) {
  OLSGD_REFUSE_IF(!is_dtype(dtype), "unknown element type %d", (int)dtype);
  OLSGD_REFUSE_IF(rows < 0 || rows > kMaxRows, "rows must be in [0, 2^31 - 1]");
  OLSGD_REFUSE_IF(V < 1 || V > kMaxVocab, "V must be in [1, 2^27]");
  return OLSGD_OK;
}

olsgd_status check_workspace(void* ws, size_t have, size_t need) {
  if (need == 0) return OLSGD_OK;
  OLSGD_REFUSE_IF(!aligned_to(ws, 256), "workspace must be non-null and 256-byte aligned");
  if (have < need)
    return refuse(OLSGD_ENOMEM, "workspace too small: %zu bytes, %zu needed", have, need);
  return OLSGD_OK;
}

olsgd_status check_gated(int32_t m, int64_t T, int64_t D, int64_t F) {
  OLSGD_REFUSE_IF(m < 1 || m > 65535, "m must be in [1, 65535]");
  OLSGD_REFUSE_IF(T < 0 || T > (1 << 28), "T must be in [0, 2^28]");
  OLSGD_REFUSE_IF(D < 1 || D > (1 << 24) || F < 1 || F > (1 << 24), "D and F must be in [1, 2^24]");
  return OLSGD_OK;
}
olsgd_status check_gated_kind(int32_t dtype, int32_t activation) {
  OLSGD_REFUSE_IF(dtype != OLSGD_BF16 && dtype != OLSGD_F16, "the gated block takes bf16 and fp16 operands");
  OLSGD_REFUSE_IF(activation < OLSGD_ACT_SILU || activation > OLSGD_ACT_SIGMOID, "unknown activation %d", (int)activation);
  return OLSGD_OK;
}
olsgd_status check_operand(const GatedOperand& o, const char* name, int64_t m, int64_t rows, int64_t cols,
                           int size = 2) {
  OLSGD_REFUSE_IF(!aligned_to(o.p, size), "%s must be non-null and aligned to its type", name);
  OLSGD_REFUSE_IF(rows > 1 && (o.row_stride < cols || o.row_stride > (1LL << 38)), "%s: rows must not overlap", name);
  OLSGD_REFUSE_IF(m > 1 && (o.worker_stride < (rows - 1) * o.row_stride + cols || o.worker_stride > (1LL << 38)),
                  "%s: workers must not overlap", name);
  return OLSGD_OK;
}

olsgd_status check_embedding(int32_t m, int64_t T, int64_t V, int64_t D, int32_t dtype) {
  OLSGD_REFUSE_IF(m < 1 || m > 65535, "m must be in [1, 65535]");
  OLSGD_REFUSE_IF(T < 0 || T > (1 << 24), "T must be in [0, 2^24]");
  OLSGD_REFUSE_IF(V < 1 || V > (1 << 24) || D < 1 || D > (1 << 24), "V and D must be in [1, 2^24]");
  OLSGD_REFUSE_IF(!is_dtype(dtype), "unknown element type %d", (int)dtype);
  return OLSGD_OK;
}

olsgd_status check_experts(int32_t m, int64_t T, int64_t E) {
  OLSGD_REFUSE_IF(m < 1 || m > 65535, "m must be in [1, 65535]");
  OLSGD_REFUSE_IF(T < 0 || T > (1 << 24), "T must be in [0, 2^24]");
  OLSGD_REFUSE_IF(E < 1 || E > OLSGD_MAX_EXPERTS, "E must be in [1, %d]", OLSGD_MAX_EXPERTS);
  return OLSGD_OK;
}
olsgd_status check_combine(int32_t m, int64_t T, int32_t k, int64_t R, int64_t D, int32_t dtype) {
  OLSGD_REFUSE_IF(m < 1 || m > 65535, "m must be in [1, 65535]");
  OLSGD_REFUSE_IF(k < 1 || T < 0 || T > kMaxRows / k || R < 0 || R > kMaxRows, "k must be positive, T k and R at most 2^31 - 1");
  OLSGD_REFUSE_IF(D < 1 || D > (1 << 24), "D must be in [1, 2^24]");
  OLSGD_REFUSE_IF(!is_dtype(dtype), "unknown element type %d", (int)dtype);
  return OLSGD_OK;
}
olsgd_status check_product(int32_t m, int64_t R, int64_t E, int64_t D, int64_t F) {
  OLSGD_REFUSE_IF(E < 1 || E > OLSGD_MAX_EXPERTS, "E must be in [1, %d]", OLSGD_MAX_EXPERTS);
  OLSGD_REFUSE_IF(m < 1 || (int64_t)m * E > 65535, "m must be positive, m E at most 65535");
  // (4095: a tile's end, or the grid's next row, still fits 32 bits)
  OLSGD_REFUSE_IF(R < 0 || R > (kMaxRows - 4095) / m, "R must not be negative, m R at most 2^31 - 4096");
  OLSGD_REFUSE_IF(D < 1 || D > (1 << 24) || F < 1 || F > (1 << 24), "D and F must be in [1, 2^24]");
  return OLSGD_OK;
}
olsgd_status check_weights(const ExpertOperand& w, int64_t m, int64_t E, int64_t F, int64_t D) {
  OLSGD_TRY(check_operand(GatedOperand{w.p, w.expert_stride, w.row_stride}, "w", E, F, D));
  const int64_t expert = (F > 1 ? (F - 1) * w.row_stride : 0) + D;
  OLSGD_REFUSE_IF(m > 1 && (w.worker_stride < (E > 1 ? (E - 1) * w.expert_stride : 0) + expert || w.worker_stride > (1LL << 38)),
                  "w: workers must not overlap");
  return OLSGD_OK;
}
olsgd_status check_distill(int32_t dtype, int64_t rows, int64_t V, int64_t row_stride, const int32_t* ids, const void* teacher,
                           int32_t teacher_dtype, int32_t K, float temperature, const void* logits) {
  OLSGD_REFUSE_IF(!is_dtype(teacher_dtype), "unknown element type %d of the teacher", (int)teacher_dtype);
  OLSGD_REFUSE_IF(K < 1 || K > OLSGD_MAX_TEACHER, "K must be in [1, %d]", OLSGD_MAX_TEACHER);
  OLSGD_REFUSE_IF(!(temperature >= 0x1p-20f && temperature <= 0x1p20f), "temperature must be in [2^-20, 2^20]");
  if (rows == 0) return OLSGD_OK;
  OLSGD_REFUSE_IF(row_stride < V, "row_stride must be at least V");
  OLSGD_REFUSE_IF(!aligned_to(logits, elem_size(dtype)), "logits must be non-null and aligned to their type");
  OLSGD_REFUSE_IF(!aligned_to(ids, 4), "ids must be non-null and 4-byte aligned");
  OLSGD_REFUSE_IF(!aligned_to(teacher, elem_size(teacher_dtype)), "teacher must be non-null and aligned to its type");
  return OLSGD_OK;
}
olsgd_status check_distill_grad(int32_t dtype, int64_t V, int64_t row_stride, const void* logits, const float* d_loss,
                                const void* d_logits, int64_t d_row_stride) {
  OLSGD_REFUSE_IF(!aligned_to(d_loss, 4), "d_loss must be non-null and 4-byte aligned");
  OLSGD_REFUSE_IF(!aligned_to(d_logits, elem_size(dtype)) || d_row_stride < V,
                  "d_logits must be non-null and aligned to its type, d_row_stride at least V");
  OLSGD_REFUSE_IF(logits == d_logits && row_stride != d_row_stride, "d_logits in place of the logits needs the same stride");
  return OLSGD_OK;
}


}  // namespace

extern "C" {

// ------------------------------------------------------------ token log probabilities

olsgd_status olsgd_token_logprobs_workspace(int32_t dtype, int64_t rows, int64_t V, int32_t top,
                                            size_t* out_bytes) {
  OLSGD_REFUSE_IF(!out_bytes, "out_bytes is NULL");
  OLSGD_TRY(check_rows(dtype, rows, V));
  OLSGD_REFUSE_IF(top < 0 || top > OLSGD_MAX_TOP || top > V, "top must be in [0, min(V, %d)]", OLSGD_MAX_TOP);
  *out_bytes = rows == 0 ? 0 : logprob_workspace(dtype, rows, V, top);
  return OLSGD_OK;
}

olsgd_status olsgd_token_logprobs(const void* logits, int32_t dtype, int64_t rows, int64_t V,
                                  int64_t row_stride, const int32_t* targets, int32_t top,
                                  float* logp, float* entropy, float* stats, float* top_logp,
                                  int32_t* top_ids, void* workspace, size_t workspace_bytes,
                                  void* stream) {
  size_t need = 0;
  OLSGD_TRY(olsgd_token_logprobs_workspace(dtype, rows, V, top, &need));
  if (rows == 0) return OLSGD_OK;
  OLSGD_REFUSE_IF(row_stride < V, "row_stride must be at least V");
  OLSGD_REFUSE_IF(!aligned_to(logits, elem_size(dtype)), "logits must be non-null and aligned to their type");
  OLSGD_REFUSE_IF(!aligned_to(targets, 4), "targets must be non-null and 4-byte aligned");
  OLSGD_REFUSE_IF(!aligned_to(logp, 4) || !aligned_to(entropy, 4) || !aligned_to(stats, 4),
                  "logp, entropy and stats must be non-null and 4-byte aligned");
  OLSGD_REFUSE_IF(top > 0 && (!aligned_to(top_logp, 4) || !aligned_to(top_ids, 4)),
                  "top_logp and top_ids must be non-null and 4-byte aligned when top > 0");
  OLSGD_TRY(check_workspace(workspace, workspace_bytes, need));
  const LogprobArgs a{logits, dtype, rows, V, row_stride, targets, top, logp, entropy, stats, top_logp, top_ids, workspace};
  return launched(launch_logprobs(a, static_cast<cudaStream_t>(stream)), "olsgd_token_logprobs");
}

olsgd_status olsgd_token_logprobs_backward(const float* d_logp, const float* d_entropy,
                                           const void* logits, int32_t dtype, int64_t rows,
                                           int64_t V, int64_t row_stride, const int32_t* targets,
                                           const float* stats, const float* entropy,
                                           void* d_logits, int64_t d_row_stride, void* stream) {
  OLSGD_TRY(check_rows(dtype, rows, V));
  if (rows == 0) return OLSGD_OK;
  OLSGD_REFUSE_IF(row_stride < V || d_row_stride < V, "row_stride and d_row_stride must be at least V");
  OLSGD_REFUSE_IF(!aligned_to(logits, elem_size(dtype)) || !aligned_to(d_logits, elem_size(dtype)),
                  "logits and d_logits must be non-null and aligned to their type");
  OLSGD_REFUSE_IF(logits == d_logits && row_stride != d_row_stride,
                  "d_logits in place of the logits needs the same stride");
  OLSGD_REFUSE_IF(!aligned_to(targets, 4) || !aligned_to(stats, 4) || !aligned_to(entropy, 4),
                  "targets, stats and entropy must be non-null and 4-byte aligned");
  OLSGD_REFUSE_IF((d_logp && !aligned_to(d_logp, 4)) || (d_entropy && !aligned_to(d_entropy, 4)),
                  "d_logp and d_entropy must be 4-byte aligned");
  const LogprobGradArgs a{logits, dtype, rows, V, row_stride, d_row_stride, targets, stats, entropy, d_logp, d_entropy, d_logits};
  return launched(launch_logprobs_backward(a, static_cast<cudaStream_t>(stream)), "olsgd_token_logprobs_backward");
}

// --------------------------------------------------------------------- gradient clipping

olsgd_status olsgd_clip_grads_workspace(int32_t m, int32_t n_tensors, size_t* out_bytes) {
  OLSGD_REFUSE_IF(!out_bytes, "out_bytes is NULL");
  OLSGD_REFUSE_IF(m < 1 || m > 65535, "m must be in [1, 65535]");
  OLSGD_REFUSE_IF(n_tensors < 0 || n_tensors > (1 << 20), "n_tensors must be in [0, 2^20]");
  *out_bytes = clip_workspace(m, n_tensors);
  return OLSGD_OK;
}

olsgd_status olsgd_clip_grads(const olsgd_clip_tensor* tensors, int32_t n_tensors, int32_t m,
                              float max_norm, float* norms, void* workspace,
                              size_t workspace_bytes, void* stream) {
  size_t need = 0;
  OLSGD_TRY(olsgd_clip_grads_workspace(m, n_tensors, &need));
  if (n_tensors == 0) return OLSGD_OK;
  OLSGD_REFUSE_IF(!tensors, "tensors is NULL");
  OLSGD_REFUSE_IF(!(max_norm > 0.f) || std::isinf(max_norm), "max_norm must be positive and finite");
  OLSGD_REFUSE_IF(!aligned_to(norms, 4), "norms must be non-null and 4-byte aligned");
  for (int32_t i = 0; i < n_tensors; ++i) {
    const olsgd_clip_tensor& t = tensors[i];
    OLSGD_REFUSE_IF(!is_dtype(t.in_dtype) || !is_dtype(t.out_dtype), "tensor %d: unknown element type", (int)i);
    OLSGD_REFUSE_IF(t.n < 0 || t.n > (1LL << 40), "tensor %d: n must be in [0, 2^40]", (int)i);
    if (t.n == 0) continue;
    OLSGD_REFUSE_IF(!aligned_to(t.in, elem_size(t.in_dtype)) || !aligned_to(t.out, elem_size(t.out_dtype)),
                    "tensor %d: pointers must be non-null and aligned to their type", (int)i);
    OLSGD_REFUSE_IF(m > 1 && (t.in_stride < t.n || t.out_stride < t.n),
                    "tensor %d: strides must be at least n", (int)i);
    OLSGD_REFUSE_IF(t.in == t.out && (t.in_dtype != t.out_dtype || (m > 1 && t.in_stride != t.out_stride)),
                    "tensor %d: in place needs the same type and stride", (int)i);
  }
  OLSGD_TRY(check_workspace(workspace, workspace_bytes, need));
  return launched(launch_clip(tensors, n_tensors, m, max_norm, norms, workspace, static_cast<cudaStream_t>(stream)),
                  "olsgd_clip_grads");
}

// ------------------------------------------------------------------- gated feed-forward block

olsgd_status olsgd_gated_workspace(int32_t m, int64_t T, int64_t D, int64_t F, int32_t backward,
                                   int32_t aligned, size_t* out_bytes) {
  OLSGD_REFUSE_IF(!out_bytes, "out_bytes is NULL");
  OLSGD_TRY(check_gated(m, T, D, F));
  *out_bytes = T == 0 ? 0 : gated_workspace(GatedShape{m, T, D, F, 0, false}, backward != 0, aligned == 0);
  return OLSGD_OK;
}

olsgd_status olsgd_gated_forward(int32_t m, int64_t T, int64_t D, int64_t F, int32_t dtype,
                                 int32_t activation, const void* x, int64_t x_worker_stride,
                                 int64_t x_row_stride, const void* w_gate,
                                 int64_t w_gate_worker_stride, int64_t w_gate_row_stride,
                                 const void* w_up, int64_t w_up_worker_stride,
                                 int64_t w_up_row_stride, void* h, float* pre, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  OLSGD_TRY(check_gated(m, T, D, F));
  OLSGD_TRY(check_gated_kind(dtype, activation));
  if (T == 0) return OLSGD_OK;
  GatedForward a;
  static_cast<GatedShape&>(a) = GatedShape{m, T, D, F, activation, dtype == OLSGD_F16};
  a.x = GatedOperand{x, x_worker_stride, x_row_stride};
  a.wg = GatedOperand{w_gate, w_gate_worker_stride, w_gate_row_stride};
  a.wu = GatedOperand{w_up, w_up_worker_stride, w_up_row_stride};
  OLSGD_TRY(check_operand(a.x, "x", m, T, D));
  OLSGD_TRY(check_operand(a.wg, "w_gate", m, F, D));
  OLSGD_TRY(check_operand(a.wu, "w_up", m, F, D));
  OLSGD_REFUSE_IF(!aligned_to(h, 2), "h must be non-null and 2-byte aligned");
  OLSGD_REFUSE_IF(pre && !aligned_to(pre, 32), "pre must be 32-byte aligned");
  a.h = h;
  a.pre = pre;
  a.ws = workspace;
  OLSGD_TRY(check_workspace(workspace, workspace_bytes, gated_workspace(a, false, gated_needs_copies(a, a.x, a.wg, a.wu))));
  return launched(launch_gated_forward(a, static_cast<cudaStream_t>(stream)), "olsgd_gated_forward");
}

olsgd_status olsgd_gated_backward(int32_t m, int64_t T, int64_t D, int64_t F, int32_t dtype,
                                  int32_t activation, const void* d_h, int64_t d_h_worker_stride,
                                  int64_t d_h_row_stride, const void* x, int64_t x_worker_stride,
                                  int64_t x_row_stride, const void* w_gate,
                                  int64_t w_gate_worker_stride, int64_t w_gate_row_stride,
                                  const void* w_up, int64_t w_up_worker_stride,
                                  int64_t w_up_row_stride, const float* pre, void* d_x,
                                  void* d_w_gate, void* d_w_up, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  OLSGD_TRY(check_gated(m, T, D, F));
  OLSGD_TRY(check_gated_kind(dtype, activation));
  OLSGD_REFUSE_IF((d_w_gate == nullptr) != (d_w_up == nullptr), "d_w_gate and d_w_up are wanted both or neither");
  OLSGD_REFUSE_IF((d_x && !aligned_to(d_x, 2)) || (d_w_gate && (!aligned_to(d_w_gate, 2) || !aligned_to(d_w_up, 2))),
                  "d_x, d_w_gate and d_w_up must be 2-byte aligned");
  if (T == 0) {   // no tokens: the weights' gradients are zero
    if (!d_w_gate) return OLSGD_OK;
    const size_t bytes = (size_t)m * F * D * 2;
    OLSGD_TRY(launched(cudaMemsetAsync(d_w_gate, 0, bytes, static_cast<cudaStream_t>(stream)), "olsgd_gated_backward"));
    return launched(cudaMemsetAsync(d_w_up, 0, bytes, static_cast<cudaStream_t>(stream)), "olsgd_gated_backward");
  }
  GatedBackward a;
  static_cast<GatedShape&>(a) = GatedShape{m, T, D, F, activation, dtype == OLSGD_F16};
  a.dh = GatedOperand{d_h, d_h_worker_stride, d_h_row_stride};
  a.x = GatedOperand{x, x_worker_stride, x_row_stride};
  a.wg = GatedOperand{w_gate, w_gate_worker_stride, w_gate_row_stride};
  a.wu = GatedOperand{w_up, w_up_worker_stride, w_up_row_stride};
  OLSGD_TRY(check_operand(a.dh, "d_h", m, T, F));
  OLSGD_TRY(check_operand(a.x, "x", m, T, D));
  OLSGD_TRY(check_operand(a.wg, "w_gate", m, F, D));
  OLSGD_TRY(check_operand(a.wu, "w_up", m, F, D));
  OLSGD_REFUSE_IF(!aligned_to(pre, 32), "pre must be non-null and 32-byte aligned");
  if (!d_x && !d_w_gate) return OLSGD_OK;
  a.pre = pre;
  a.dx = d_x;
  a.dwg = d_w_gate;
  a.dwu = d_w_up;
  a.ws = workspace;
  OLSGD_TRY(check_workspace(workspace, workspace_bytes, gated_workspace(a, true, gated_needs_copies(a, a.x, a.wg, a.wu))));
  return launched(launch_gated_backward(a, static_cast<cudaStream_t>(stream)), "olsgd_gated_backward");
}

// -------------------------------------------------------------------------- embedding lookup

olsgd_status olsgd_embedding_forward(int32_t m, int64_t T, int64_t V, int64_t D, int32_t dtype,
                                     const void* table, int64_t table_worker_stride,
                                     int64_t table_row_stride, const int32_t* ids, float scale,
                                     void* out, void* stream) {
  OLSGD_TRY(check_embedding(m, T, V, D, dtype));
  if (T == 0) return OLSGD_OK;
  OLSGD_TRY(check_operand(GatedOperand{table, table_worker_stride, table_row_stride}, "table", m, V, D, elem_size(dtype)));
  OLSGD_REFUSE_IF(!aligned_to(ids, 4), "ids must be non-null and 4-byte aligned");
  OLSGD_REFUSE_IF(!aligned_to(out, elem_size(dtype)), "out must be non-null and aligned to its type");
  const EmbeddingArgs a{dtype, m, T, V, D, table, table_worker_stride, table_row_stride, ids, out, scale};
  return launched(launch_embedding_forward(a, static_cast<cudaStream_t>(stream)), "olsgd_embedding_forward");
}

olsgd_status olsgd_embedding_workspace(int32_t m, int64_t T, int64_t D, size_t* out_bytes) {
  OLSGD_REFUSE_IF(!out_bytes, "out_bytes is NULL");
  OLSGD_TRY(check_embedding(m, T, 1, D, OLSGD_F32));
  *out_bytes = T == 0 ? 0 : embedding_workspace(m, T, D);
  return OLSGD_OK;
}

olsgd_status olsgd_embedding_backward(int32_t m, int64_t T, int64_t V, int64_t D, int32_t dtype,
                                      const void* d_out, int64_t d_out_worker_stride,
                                      int64_t d_out_row_stride, const int32_t* ids, float scale,
                                      int32_t d_table_dtype, void* d_table,
                                      int64_t d_table_worker_stride, void* workspace,
                                      size_t workspace_bytes, void* stream) {
  OLSGD_TRY(check_embedding(m, T, V, D, dtype));
  OLSGD_REFUSE_IF(!is_dtype(d_table_dtype), "unknown element type %d of d_table", (int)d_table_dtype);
  OLSGD_REFUSE_IF(!aligned_to(d_table, elem_size(d_table_dtype)), "d_table must be non-null and aligned to its type");
  OLSGD_REFUSE_IF(m > 1 && d_table_worker_stride < V * D, "d_table: workers must not overlap");
  size_t need = 0;
  if (T > 0) {
    OLSGD_TRY(check_operand(GatedOperand{d_out, d_out_worker_stride, d_out_row_stride}, "d_out", m, T, D, elem_size(dtype)));
    OLSGD_REFUSE_IF(!aligned_to(ids, 4), "ids must be non-null and 4-byte aligned");
    need = embedding_workspace(m, T, D);
  }
  OLSGD_TRY(check_workspace(workspace, workspace_bytes, need));
  const EmbeddingGradArgs a{dtype, d_table_dtype, m, T, V, D, d_out, d_out_worker_stride, d_out_row_stride, ids, scale,
                            d_table, d_table_worker_stride, workspace};
  return launched(launch_embedding_backward(a, static_cast<cudaStream_t>(stream)), "olsgd_embedding_backward");
}

// ----------------------------------------------------------------------------------- experts

olsgd_status olsgd_expert_route_workspace(int32_t m, int64_t T, int64_t E, size_t* out_bytes) {
  OLSGD_REFUSE_IF(!out_bytes, "out_bytes is NULL");
  OLSGD_TRY(check_experts(m, T, E));
  *out_bytes = T == 0 ? 0 : route_workspace(m, T, E);
  return OLSGD_OK;
}

olsgd_status olsgd_expert_route(int32_t m, int64_t T, int64_t E, int32_t dtype, const void* logits,
                                int64_t row_stride, int32_t k, int32_t normalise, float* weights,
                                int32_t* ids, int32_t* places, int32_t* tokens, int32_t* offsets,
                                void* workspace, size_t workspace_bytes, void* stream) {
  OLSGD_TRY(check_experts(m, T, E));
  OLSGD_REFUSE_IF(!is_dtype(dtype), "unknown element type %d", (int)dtype);
  OLSGD_REFUSE_IF(k < 1 || k > OLSGD_MAX_TOP || k > E, "k must be in [1, min(E, %d)]", OLSGD_MAX_TOP);
  OLSGD_REFUSE_IF(T * k > kMaxRows, "T k must be at most 2^31 - 1");
  OLSGD_REFUSE_IF(!aligned_to(offsets, 4), "offsets must be non-null and 4-byte aligned");
  if (T == 0)
    return launched(cudaMemsetAsync(offsets, 0, (size_t)m * (E + 1) * sizeof(int32_t), static_cast<cudaStream_t>(stream)), "olsgd_expert_route");
  OLSGD_REFUSE_IF(row_stride < E, "row_stride must be at least E");
  OLSGD_REFUSE_IF(!aligned_to(logits, elem_size(dtype)), "logits must be non-null and aligned to their type");
  OLSGD_REFUSE_IF(!aligned_to(weights, 4) || !aligned_to(ids, 4) || !aligned_to(places, 4) || !aligned_to(tokens, 4),
                  "weights, ids, places and tokens must be non-null and 4-byte aligned");
  OLSGD_TRY(check_workspace(workspace, workspace_bytes, route_workspace(m, T, E)));
  const RouteArgs a{dtype, m, T, E, logits, row_stride, k, normalise != 0, weights, ids, places, tokens, offsets, workspace};
  return launched(launch_route(a, static_cast<cudaStream_t>(stream)), "olsgd_expert_route");
}

olsgd_status olsgd_expert_route_backward(int64_t rows, int64_t E, int32_t dtype, const float* d_weights,
                                         const void* logits, int64_t row_stride, int32_t k,
                                         int32_t normalise, const int32_t* ids, const float* weights,
                                         void* d_logits, void* stream) {
  OLSGD_TRY(check_experts(1, 0, E));
  OLSGD_REFUSE_IF(rows < 0 || rows > kMaxRows, "rows must be in [0, 2^31 - 1]");
  OLSGD_REFUSE_IF(!is_dtype(dtype), "unknown element type %d", (int)dtype);
  OLSGD_REFUSE_IF(k < 1 || k > OLSGD_MAX_TOP || k > E, "k must be in [1, min(E, %d)]", OLSGD_MAX_TOP);
  if (rows == 0) return OLSGD_OK;
  OLSGD_REFUSE_IF(normalise == 0 && (!aligned_to(logits, elem_size(dtype)) || row_stride < E),
                  "logits must be non-null and aligned to their type, row_stride at least E");
  OLSGD_REFUSE_IF(!aligned_to(d_weights, 4) || !aligned_to(ids, 4) || !aligned_to(weights, 4),
                  "d_weights, ids and weights must be non-null and 4-byte aligned");
  OLSGD_REFUSE_IF(!aligned_to(d_logits, elem_size(dtype)) || d_logits == logits,
                  "d_logits must be non-null, aligned to its type and apart from the logits");
  const RouteGradArgs a{dtype, rows, (int)E, k, normalise != 0, logits, row_stride, ids, weights, d_weights, d_logits};
  return launched(launch_route_backward(a, static_cast<cudaStream_t>(stream)), "olsgd_expert_route_backward");
}

olsgd_status olsgd_expert_combine(int32_t m, int64_t T, int32_t k, int64_t R, int64_t D, int32_t dtype,
                                  const void* rows, int64_t rows_worker_stride, int64_t rows_row_stride,
                                  const int32_t* places, const float* weights, void* y, void* stream) {
  OLSGD_TRY(check_combine(m, T, k, R, D, dtype));
  if (T == 0) return OLSGD_OK;
  if (R > 0) OLSGD_TRY(check_operand(GatedOperand{rows, rows_worker_stride, rows_row_stride}, "rows", m, R, D, elem_size(dtype)));
  OLSGD_REFUSE_IF(!aligned_to(places, 4) || (weights && !aligned_to(weights, 4)), "places must be non-null, places and weights 4-byte aligned");
  OLSGD_REFUSE_IF(!aligned_to(y, elem_size(dtype)), "y must be non-null and aligned to its type");
  const CombineArgs a{dtype, k, m, T, R, D, rows, rows_worker_stride, rows_row_stride, places, weights, y, nullptr};
  return launched(launch_combine(a, static_cast<cudaStream_t>(stream)), "olsgd_expert_combine");
}

olsgd_status olsgd_expert_combine_backward(int32_t m, int64_t T, int32_t k, int64_t R, int64_t D,
                                           int32_t dtype, const void* d_y, int64_t d_y_worker_stride,
                                           int64_t d_y_row_stride, const void* rows,
                                           int64_t rows_worker_stride, int64_t rows_row_stride,
                                           const int32_t* places, const int32_t* tokens,
                                           const float* weights, void* d_rows, float* d_weights,
                                           void* stream) {
  OLSGD_TRY(check_combine(m, T, k, R, D, dtype));
  if (T == 0 && R == 0) return OLSGD_OK;
  if (R > 0) {
    OLSGD_TRY(check_operand(GatedOperand{rows, rows_worker_stride, rows_row_stride}, "rows", m, R, D, elem_size(dtype)));
    OLSGD_REFUSE_IF(!aligned_to(tokens, 4), "tokens must be non-null and 4-byte aligned");
    OLSGD_REFUSE_IF(!aligned_to(d_rows, elem_size(dtype)), "d_rows must be non-null and aligned to its type");
  }
  if (T > 0) {
    OLSGD_TRY(check_operand(GatedOperand{d_y, d_y_worker_stride, d_y_row_stride}, "d_y", m, T, D, elem_size(dtype)));
    OLSGD_REFUSE_IF(!aligned_to(places, 4) || !aligned_to(weights, 4) || !aligned_to(d_weights, 4),
                    "places, weights and d_weights must be non-null and 4-byte aligned");
  }
  const CombineGradArgs a{dtype, k, m, T, R, D, d_y, d_y_worker_stride, d_y_row_stride, rows, rows_worker_stride, rows_row_stride,
                          places, tokens, weights, d_rows, d_weights, nullptr, nullptr};
  return launched(launch_combine_backward(a, static_cast<cudaStream_t>(stream)), "olsgd_expert_combine_backward");
}

olsgd_status olsgd_expert_product_workspace(int32_t m, int64_t R, int64_t E, int64_t D, int64_t F,
                                            int32_t backward, int32_t aligned, size_t* out_bytes) {
  OLSGD_REFUSE_IF(!out_bytes, "out_bytes is NULL");
  OLSGD_TRY(check_product(m, R, E, D, F));
  *out_bytes = R == 0 ? 0 : product_workspace(ProductShape{m, R, E, D, F, false}, backward != 0, aligned == 0);
  return OLSGD_OK;
}

olsgd_status olsgd_expert_product(int32_t m, int64_t R, int64_t E, int64_t D, int64_t F, int32_t dtype,
                                  const void* x, int64_t x_worker_stride, int64_t x_row_stride,
                                  const void* w, int64_t w_worker_stride,
                                  int64_t w_expert_stride, int64_t w_row_stride,
                                  const int32_t* offsets, void* y, void* workspace,
                                  size_t workspace_bytes, void* stream) {
  OLSGD_TRY(check_product(m, R, E, D, F));
  OLSGD_REFUSE_IF(dtype != OLSGD_BF16 && dtype != OLSGD_F16, "products by expert take bf16 and fp16 operands");
  if (R == 0) return OLSGD_OK;
  ProductForward a;
  static_cast<ProductShape&>(a) = ProductShape{m, R, E, D, F, dtype == OLSGD_F16};
  a.x = GatedOperand{x, x_worker_stride, x_row_stride};
  a.w = ExpertOperand{w, w_worker_stride, w_expert_stride, w_row_stride};
  OLSGD_TRY(check_operand(a.x, "x", m, R, D));
  OLSGD_TRY(check_weights(a.w, m, E, F, D));
  OLSGD_REFUSE_IF(!aligned_to(offsets, 4), "offsets must be non-null and 4-byte aligned");
  OLSGD_REFUSE_IF(!aligned_to(y, 2), "y must be non-null and 2-byte aligned");
  a.offsets = offsets;
  a.y = y;
  a.ws = workspace;
  OLSGD_TRY(check_workspace(workspace, workspace_bytes, product_workspace(a, false, product_needs_copies(a, a.x, a.w, nullptr))));
  return launched(launch_product(a, static_cast<cudaStream_t>(stream)), "olsgd_expert_product");
}

olsgd_status olsgd_expert_product_backward(int32_t m, int64_t R, int64_t E, int64_t D, int64_t F,
                                           int32_t dtype, const void* d_y, int64_t d_y_worker_stride,
                                           int64_t d_y_row_stride, const void* x, int64_t x_worker_stride,
                                           int64_t x_row_stride, const void* w, int64_t w_worker_stride,
                                           int64_t w_expert_stride, int64_t w_row_stride, const int32_t* offsets, void* d_x,
                                           void* d_w, void* workspace, size_t workspace_bytes,
                                           void* stream) {
  OLSGD_TRY(check_product(m, R, E, D, F));
  OLSGD_REFUSE_IF(dtype != OLSGD_BF16 && dtype != OLSGD_F16, "products by expert take bf16 and fp16 operands");
  OLSGD_REFUSE_IF((d_x && !aligned_to(d_x, 2)) || (d_w && !aligned_to(d_w, 2)), "d_x and d_w must be 2-byte aligned");
  if (R == 0) {   // no rows: the weights' gradients are zero
    if (!d_w) return OLSGD_OK;
    return launched(cudaMemsetAsync(d_w, 0, (size_t)m * E * F * D * 2, static_cast<cudaStream_t>(stream)), "olsgd_expert_product_backward");
  }
  ProductBackward a;
  static_cast<ProductShape&>(a) = ProductShape{m, R, E, D, F, dtype == OLSGD_F16};
  a.dy = GatedOperand{d_y, d_y_worker_stride, d_y_row_stride};
  a.x = GatedOperand{x, x_worker_stride, x_row_stride};
  a.w = ExpertOperand{w, w_worker_stride, w_expert_stride, w_row_stride};
  OLSGD_TRY(check_operand(a.dy, "d_y", m, R, F));
  OLSGD_TRY(check_operand(a.x, "x", m, R, D));
  OLSGD_TRY(check_weights(a.w, m, E, F, D));
  OLSGD_REFUSE_IF(!aligned_to(offsets, 4), "offsets must be non-null and 4-byte aligned");
  if (!d_x && !d_w) return OLSGD_OK;
  a.offsets = offsets;
  a.dx = d_x;
  a.dw = d_w;
  a.ws = workspace;
  OLSGD_TRY(check_workspace(workspace, workspace_bytes, product_workspace(a, true, product_needs_copies(a, a.x, a.w, &a.dy))));
  return launched(launch_product_backward(a, static_cast<cudaStream_t>(stream)), "olsgd_expert_product_backward");
}

// ------------------------------------------------------------------------------ distillation

olsgd_status olsgd_distill_workspace(int32_t dtype, int64_t rows, int64_t V, int32_t gradient, size_t* out_bytes) {
  OLSGD_REFUSE_IF(!out_bytes, "out_bytes is NULL");
  OLSGD_TRY(check_rows(dtype, rows, V));
  *out_bytes = rows == 0 ? 0 : distill_workspace(dtype, rows, V, OLSGD_MAX_TEACHER, gradient != 0);
  return OLSGD_OK;
}

olsgd_status olsgd_distill(const void* logits, int32_t dtype, int64_t rows, int64_t V, int64_t row_stride,
                           const int32_t* ids, const void* teacher, int32_t teacher_dtype, int32_t K,
                           float temperature, const float* d_loss, float* loss, float* stats,
                           void* d_logits, int64_t d_row_stride, void* workspace,
                           size_t workspace_bytes, void* stream) {
  OLSGD_TRY(check_rows(dtype, rows, V));
  OLSGD_TRY(check_distill(dtype, rows, V, row_stride, ids, teacher, teacher_dtype, K, temperature, logits));
  if (rows == 0) return OLSGD_OK;
  OLSGD_REFUSE_IF(!aligned_to(loss, 4) || !aligned_to(stats, 4), "loss and stats must be non-null and 4-byte aligned");
  if (d_loss) OLSGD_TRY(check_distill_grad(dtype, V, row_stride, logits, d_loss, d_logits, d_row_stride));
  OLSGD_TRY(check_workspace(workspace, workspace_bytes, distill_workspace(dtype, rows, V, K, d_loss != nullptr)));
  const DistillArgs a{logits, dtype, rows, V, row_stride, ids, teacher, teacher_dtype, K, (float)(1.0 / temperature),
                      d_loss, loss, stats, d_logits, d_row_stride, workspace, nullptr};
  return launched(launch_distill(a, static_cast<cudaStream_t>(stream)), "olsgd_distill");
}

olsgd_status olsgd_distill_backward(const float* d_loss, const void* logits, int32_t dtype, int64_t rows,
                                    int64_t V, int64_t row_stride, const int32_t* ids, const void* teacher,
                                    int32_t teacher_dtype, int32_t K, float temperature,
                                    const float* stats, void* d_logits, int64_t d_row_stride,
                                    void* stream) {
  OLSGD_TRY(check_rows(dtype, rows, V));
  OLSGD_TRY(check_distill(dtype, rows, V, row_stride, ids, teacher, teacher_dtype, K, temperature, logits));
  if (rows == 0) return OLSGD_OK;
  OLSGD_REFUSE_IF(!aligned_to(stats, 4), "stats must be non-null and 4-byte aligned");
  OLSGD_TRY(check_distill_grad(dtype, V, row_stride, logits, d_loss, d_logits, d_row_stride));
  const DistillArgs a{logits, dtype, rows, V, row_stride, ids, teacher, teacher_dtype, K, (float)(1.0 / temperature),
                      d_loss, nullptr, const_cast<float*>(stats), d_logits, d_row_stride, nullptr, nullptr};
  return launched(launch_distill_backward(a, static_cast<cudaStream_t>(stream)), "olsgd_distill_backward");
}

olsgd_status olsgd_operators_join(void* stream) {
  int status = 0;
  const olsgd_status st = launched(operators_status(&status, static_cast<cudaStream_t>(stream)), "olsgd_operators_join");
  if (st != OLSGD_OK) return st;
  if (status != 0) return refuse(OLSGD_ETIMEOUT, "a bounded device-side wait of an operator gave up: its outputs are not valid");
  return OLSGD_OK;
}

}  // extern "C"
