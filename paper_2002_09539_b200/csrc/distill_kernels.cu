// Distillation from a teacher's top logits: for a row x of V logits and K pairs (token, teacher's logit z),
//   q = softmax(z / tau) over the pairs, p = softmax(x / tau) over all tokens,
//   loss = sum q_j (log q_j - log p_id_j),    d_x = (d_loss / tau) (p - q at the pairs' tokens).
// With m = max x: log p = (x - m) / tau - log sum exp((x - m) / tau); the difference is formed before it is
// scaled.  Sums and statistics are held in fp32.
//
// Bound by the logits' way in and, for a gradient, its way out (4096 x 32768 bf16 with gradient: 122 us, 537 MB, 4.4 TB/s; loss
// of 1021 x 50021 fp32: 39 us, 204 MB, 5.2 TB/s).  Where the rows' weights are known when
// the loss is formed, both come from one read: a row lies in the registers of a CTA as exp(x - the warp's own max), 32 or 40
// values a thread, until the whole row's sum is known.  Longer rows take two passes; so do losses alone and gradients that are asked for
// later, one each, unless the row is short (4096 x 32768 bf16: 55 and 91 us).  Rows of up to 1024 logits belong to a warp.
//
// A gradient at the pairs' tokens is formed apart from the others, from the logit and the sum of the q of
// all pairs with that token, and stored behind them, so that it is rounded once.
#include "operator_common.cuh"
#include "operators_internal.h"

namespace olsgd {
namespace {

using namespace op;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kChunkElems = 256;     // of a warp's turn: eight elements a lane
constexpr int kWarpRowMax = 1024;    // longest row that stays in a warp's registers
constexpr int kMaxSplit = 64;
constexpr int kGradPieces = 4;       // of a thread's turn
constexpr int64_t kGradCtas = 148 * 16, kKeepBytes = 64 << 20;
constexpr int kMaxPairs = OLSGD_MAX_TEACHER;
static_assert(kMaxPairs <= kThreads, "a thread for each pair");

struct Sum {
  float m, s;   // maximum; sum of exp((x - m) / tau)
};
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }
// c = log2(e) / tau
__device__ __forceinline__ Sum join(const Sum& a, const Sum& b, float c) {
  Sum r;
  r.m = fmaxf(a.m, b.m);
  const float base = base_of(r.m);
  // (a part of nothing but -inf has the sum 0, or NaN)
  r.s = a.s * (a.m == -INFINITY ? 1.f : ex2((a.m - base) * c)) + b.s * (b.m == -INFINITY ? 1.f : ex2((b.m - base) * c));
  return r;
}
__device__ __forceinline__ Sum shfl_join(Sum v, float c) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    Sum w;
    w.m = __shfl_xor_sync(0xffffffffu, v.m, o);
    w.s = __shfl_xor_sync(0xffffffffu, v.s, o);
    v = join(v, w, c);
  }
  return v;
}
__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
// A row of nothing but -inf has no distribution: log p = -inf, no gradient.
__device__ __forceinline__ bool empty(const Sum& v) { return v.m == -INFINITY && v.s == 0.f; }
__device__ __forceinline__ float log_sum(const Sum& v) { return empty(v) ? 0.f : logf(v.s); }

template <typename T>
__host__ __device__ constexpr uint32_t minus_inf() {
  return sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00u : 0xFF80u;
}
__device__ __forceinline__ float load_any(const void* p, int dtype, int64_t i) {
  if (dtype == OLSGD_F32) return static_cast<const float*>(p)[i];
  if (dtype == OLSGD_BF16) return Elem<__nv_bfloat16>::to_float(static_cast<const __nv_bfloat16*>(p)[i]);
  return Elem<__half>::to_float(static_cast<const __half*>(p)[i]);
}

// A pair as its thread holds it.  A token outside [0, V) is no pair.
struct Pair {
  int32_t id;
  float z, x;   // the teacher's logit, the student's
};
template <typename T>
__device__ __forceinline__ Pair fetch_pair(const DistillArgs& a, const T* row, int64_t r, int j) {
  Pair p{-1, -INFINITY, 0.f};
  if (j < a.K) {
    p.id = a.ids[r * a.K + j];
    if (p.id < 0 || p.id >= a.V) {
      p.id = -1;
    } else {
      p.z = load_any(a.teacher, a.teacher_dtype, r * a.K + j);
      p.x = Elem<T>::to_float(row[p.id]);
    }
  }
  return p;
}

// The teacher's side of a row: maximum and sum of its logits as the student's.  A maximum that passes over
// NaN is followed by a sum that does not.
struct PairTerm {
  float q, loss;
};
__device__ __forceinline__ PairTerm pair_term(const Pair& p, const Sum& teacher, float log_teacher, const Sum& row, float log_s,
                                              float inv_t, float c) {
  PairTerm t{0.f, 0.f};
  if (p.id < 0 || empty(teacher)) return t;
  const float z = (p.z - base_of(teacher.m)) * inv_t;
  t.q = ex2((p.z - base_of(teacher.m)) * c) / teacher.s;
  if (t.q == 0.f) return t;
  const float lp = empty(row) ? -INFINITY : (p.x - base_of(row.m)) * inv_t - log_s;
  t.loss = t.q * ((z - log_teacher) - lp);
  return t;
}

// What a gradient takes from a row.  Rows that nothing is asked of (no teacher, a weight of 0) and rows without
// a distribution have a gradient of 0 whatever they hold.
struct GradRow {
  float base, scale;   // gradient of an ordinary token: scale exp((x - base) / tau)
  float g;             // d_loss / tau
  bool zero;
  __device__ __forceinline__ float at(float x, float c) const { return zero ? 0.f : scale * ex2((x - base) * c); }
};

// ------------------------------------------------------------ rows in a warp's registers
// LOSS: loss and statistics are written; GRAD: the gradient (from `stats` where LOSS is false).
template <typename T, int NL, bool LOSS, bool GRAD>
__global__ void __launch_bounds__(kThreads) distill_warp_kernel(const DistillArgs a) {
  __shared__ float q_of[kWarps][kMaxPairs];
  __shared__ float x_of[kWarps][kMaxPairs];
  __shared__ int32_t id_of[kWarps][kMaxPairs];
  launch_gate();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t r = (int64_t)blockIdx.x * kWarps + warp;
  if (r >= a.rows) return;
  const T* row = static_cast<const T*>(a.logits) + r * a.ld;
  const int V = (int)a.V;
  const float c = a.inv_t * kLog2e;
  float v[NL], mx = -INFINITY;
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int j = i * 32 + lane;
    v[i] = j < V ? Elem<T>::to_float(row[j]) : -INFINITY;
    mx = fmaxf(mx, v[i]);
  }
  Sum student, teacher{-INFINITY, 0.f};
  float log_s;
  if (LOSS) {
    student.m = warp_max(mx);
    student.s = 0.f;
    const float base = base_of(student.m);
#pragma unroll
    for (int i = 0; i < NL; ++i) student.s += ex2((v[i] - base) * c);
    student.s = warp_sum(student.s);
    log_s = log_sum(student);
  } else {
    student.m = a.stats[2 * r];
    log_s = a.stats[2 * r + 1];
    student.s = student.m == -INFINITY && log_s == 0.f ? 0.f : ex2(log_s * kLog2e);
  }
  for (int j = lane; j < a.K; j += 32) teacher.m = fmaxf(teacher.m, fetch_pair<T>(a, row, r, j).z);
  teacher.m = warp_max(teacher.m);
  for (int j = lane; j < a.K; j += 32) teacher.s += ex2((fetch_pair<T>(a, row, r, j).z - base_of(teacher.m)) * c);
  teacher.s = warp_sum(teacher.s);
  const float log_teacher = log_sum(teacher);
  float loss = 0.f;
  for (int j = lane; j < a.K; j += 32) {
    const Pair p = fetch_pair<T>(a, row, r, j);
    const PairTerm t = pair_term(p, teacher, log_teacher, student, log_s, a.inv_t, c);
    loss += t.loss;
    q_of[warp][j] = t.q;
    x_of[warp][j] = p.x;
    id_of[warp][j] = p.id;
  }
  if (LOSS) {
    loss = warp_sum(loss);
    if (lane == 0) {
      a.loss[r] = loss;
      a.stats[2 * r] = student.m;
      a.stats[2 * r + 1] = log_s;
    }
  }
  if (GRAD) {
    __syncwarp();
    T* out = static_cast<T*>(a.d_logits) + r * a.ldd;
    const float weight = a.d_loss[r];
    GradRow g;
    g.zero = weight == 0.f || empty(teacher) || empty(student);
    g.g = weight * a.inv_t;
    g.base = base_of(student.m);
    g.scale = g.g / student.s;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int j = i * 32 + lane;
      if (j < V) out[j] = Elem<T>::from_float(g.at(v[i], c));
    }
    if (g.zero) return;
    __syncwarp();
    // the pairs' tokens; the first of the pairs with a token adds up all of them
    for (int j = lane; j < a.K; j += 32) {
      const int32_t id = id_of[warp][j];
      float q = 0.f;
      int first = j;
      for (int e = 0; e < a.K; ++e)
        if (id_of[warp][e] == id) {
          q += q_of[warp][e];
          first = min(first, e);
        }
      if (id >= 0 && first == j) out[id] = Elem<T>::from_float(fmaf(-g.g, q, g.at(x_of[warp][j], c)));
    }
  }
}

// -------------------------------------------------------------------------- long rows
// Sums over a CTA's threads, every thread gets them.
template <int NT>
__device__ __forceinline__ Sum block_join(Sum v, float c, Sum* sh) {
  v = shfl_join(v, c);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
  v = (threadIdx.x & 31) < NT / 32 ? sh[threadIdx.x & 31] : Sum{-INFINITY, 0.f};
  v = shfl_join(v, c);
  __syncthreads();
  return v;
}

// The loss of a row whose statistics are known, by a whole CTA.
template <typename T, int NT>
__device__ __forceinline__ void write_loss(const DistillArgs& a, const T* row, int64_t r, const Sum& student, Sum* sh, float* sums) {
  const float c = a.inv_t * kLog2e;
  const Pair p = fetch_pair<T>(a, row, r, threadIdx.x);
  // (a thread's own term: relative to itself 1, or NaN, or nothing)
  const Sum teacher = block_join<NT>(Sum{p.z == p.z ? p.z : -INFINITY, p.z == -INFINITY ? 0.f : p.z == p.z ? ex2((p.z - p.z) * c) : p.z}, c, sh);
  const float log_s = log_sum(student);
  const PairTerm t = pair_term(p, teacher, log_sum(teacher), student, log_s, a.inv_t, c);
  const float loss = warp_sum(t.loss);
  if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = loss;
  __syncthreads();
  if (threadIdx.x == 0) {
    float all = 0.f;
    for (int i = 0; i < NT / 32; ++i) all += sums[i];
    a.loss[r] = all;
    a.stats[2 * r] = student.m;
    a.stats[2 * r + 1] = log_s;
  }
}

// CTA (r, split): chunks [split * cps, (split + 1) * cps) of row r, dealt to the warps in turn.
template <typename T>
__global__ void __launch_bounds__(kThreads) distill_row_kernel(const DistillArgs a, int nchunks, int cps, float2* __restrict__ part) {
  constexpr int VEC = Elem<T>::kVec;
  constexpr int Q = kChunkElems / 32 / VEC;   // pieces of a chunk per lane
  constexpr int U = 4;                        // chunks a turn
  __shared__ Sum sh[kWarps];
  __shared__ float sums[kWarps];
  launch_gate();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, V = (int)a.V;
  const int64_t r = blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + r * a.ld;
  const int shift = row_shift(row);
  const float c = a.inv_t * kLog2e;
  const f32x2 c2 = pack2f(c, c);
  const int c_end = min(nchunks, (int)(blockIdx.y + 1) * cps);
  float m = -INFINITY;
  f32x2 s = 0;
  for (int c0 = blockIdx.y * cps + warp; c0 < c_end; c0 += kWarps * U) {
    uint4 w[U][Q];
    const int first = c0 * kChunkElems - shift, last = (c0 + (U - 1) * kWarps) * kChunkElems - shift;
    if (first >= 0 && c0 + (U - 1) * kWarps < c_end && last + kChunkElems <= V) {
      const uint4* p = reinterpret_cast<const uint4*>(row + first) + lane;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < Q; ++q) w[u][q] = ld16_stream(p + u * (kWarps * 32 * Q) + q * 32);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          const int at = c0 + u * kWarps;
          w[u][q] = load_raw<T>(row, at < c_end ? at * kChunkElems + (q * 32 + lane) * VEC - shift : V, V, minus_inf<T>());
        }
    }
    float mx = m;
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < Q; ++q) mx = fmaxf(mx, raw_max<T, false>(w[u][q]));
    if (mx > m) {   // (each lane has a maximum of its own)
      if (m > -INFINITY) {
        const float f = ex2((m - mx) * c);
        s = mul2(s, pack2f(f, f));
      }
      m = mx;
    }
    const float base = -base_of(m);
    const f32x2 minus_base = pack2f(base, base);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) {
          float lo, hi;
          unpack2f(mul2(add2(raw_pair<T>(w[u][q], i), minus_base), c2), lo, hi);
          s = add2(s, pack2f(ex2(lo), ex2(hi)));
        }
  }
  float lo, hi;
  unpack2f(s, lo, hi);
  const Sum whole = block_join<kThreads>(Sum{m, lo + hi}, c, sh);
  if (part) {
    if (threadIdx.x == 0) part[r * gridDim.y + blockIdx.y] = make_float2(whole.m, whole.s);
  } else {
    write_loss<T, kThreads>(a, row, r, whole, sh, sums);
  }
}

// Joins a row's parts.
template <typename T>
__global__ void __launch_bounds__(kThreads) distill_finish_kernel(const DistillArgs a, int nsplit, const float2* __restrict__ part) {
  __shared__ Sum sh[kWarps];
  __shared__ float sums[kWarps];
  launch_gate();
  const int64_t r = blockIdx.x;
  Sum v{-INFINITY, 0.f};
  if ((int)threadIdx.x < nsplit) {
    const float2 p = part[r * nsplit + threadIdx.x];
    v = Sum{p.x, p.y};
  }
  v = block_join<kThreads>(v, a.inv_t * kLog2e, sh);
  write_loss<T, kThreads>(a, static_cast<const T*>(a.logits) + r * a.ld, r, v, sh, sums);
}

// The pairs of a row in shared memory, for its gradient.
struct PairTable {
  float q[kMaxPairs];
  int32_t id[kMaxPairs];
};
// After the CTA's stores of the elements [begin, end): those of them that are the pairs' tokens.  The first of
// the pairs with a token adds up all of them.
template <typename T>
__device__ __forceinline__ void store_pairs(const DistillArgs& a, const PairTable& t, const Pair& p, const GradRow& g, int begin, int end,
                                            float c, T* out) {
  __syncthreads();
  if (p.id >= 0 && p.id >= begin && p.id < end) {   // (-1: no pair; a segment may begin ahead of the row)
    float q = 0.f;
    int first = kMaxPairs;
    for (int e = 0; e < a.K; ++e)
      if (t.id[e] == p.id) {
        q += t.q[e];
        first = min(first, e);
      }
    if (first == (int)threadIdx.x) out[p.id] = Elem<T>::from_float(fmaf(-g.g, q, g.at(p.x, c)));
  }
}

// CTA (r, segment): `turns` times kThreads * U pieces of row r, the next on their way while the last leave.  What the pairs cost is
// paid once a segment, so that these are as long as leave the GPU full.
template <typename T, bool STREAM>
__global__ void __launch_bounds__(kThreads, 4) distill_grad_kernel(const DistillArgs a, int turns) {
  constexpr int VEC = Elem<T>::kVec, U = kGradPieces, kTurn = kThreads * U * VEC;
  __shared__ Sum sh[kWarps];
  __shared__ PairTable table;
  launch_gate();
  const int64_t r = a.rows - 1 - blockIdx.x;   // from the row that was read last
  const int V = (int)a.V;
  const T* row = static_cast<const T*>(a.logits) + r * a.ld;
  T* out = static_cast<T*>(a.d_logits) + r * a.ldd;
  const int shift = row_shift(row);
  const bool aligned = row_shift(out) == shift;
  const float c = a.inv_t * kLog2e;
  const int begin = (int)blockIdx.y * turns * kTurn - shift, end = min(V, begin + turns * kTurn);
  int j0 = begin + (int)threadIdx.x * VEC;
  uint4 w[U];
#pragma unroll
  for (int u = 0; u < U; ++u) w[u] = load_raw<T>(row, j0 + u * kThreads * VEC, V, 0);
  const Pair p = fetch_pair<T>(a, row, r, threadIdx.x);
  const Sum teacher = block_join<kThreads>(Sum{p.z == p.z ? p.z : -INFINITY, p.z == -INFINITY ? 0.f : p.z == p.z ? ex2((p.z - p.z) * c) : p.z}, c, sh);
  const float m = a.stats[2 * r], log_s = a.stats[2 * r + 1], weight = a.d_loss[r];
  const Sum student{m, m == -INFINITY && log_s == 0.f ? 0.f : ex2(log_s * kLog2e)};
  GradRow g;
  g.zero = weight == 0.f || empty(teacher) || empty(student);
  g.g = weight * a.inv_t;
  g.base = base_of(m);
  g.scale = g.g / student.s;
  if ((int)threadIdx.x < a.K) {
    table.q[threadIdx.x] = p.id < 0 || empty(teacher) ? 0.f : ex2((p.z - base_of(teacher.m)) * c) / teacher.s;
    table.id[threadIdx.x] = p.id;
  }
  for (; j0 < end; j0 += kTurn) {
    uint4 next[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + kTurn + u * kThreads * VEC;
      if (j < end) next[u] = load_raw<T>(row, j, V, 0);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kThreads * VEC;
      if (j >= end) break;
      float d[VEC];
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) {
        float lo, hi;
        unpack2f(raw_pair<T>(w[u], i), lo, hi);
        d[2 * i] = g.at(lo, c);
        d[2 * i + 1] = g.at(hi, c);
      }
      store_floats<T, VEC, STREAM>(out, j, V, aligned, d);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) w[u] = next[u];
  }
  if (!g.zero) store_pairs<T>(a, table, p, g, begin, end, c, out);
}

// -------------------------------------------------------- loss and gradient from one read
// CTAs that stay, a row at a time, 32 or 40 elements a thread, counted from the 16-byte boundary at or before the row.  The warps
// have the row's elements: each takes its own maximum and sum, and joins them all behind the row's one barrier.
// One more warp brings the rows in (bulk copies of the whole 16-byte pieces, two buffers), has the pairs and writes
// the loss; it stores the gradients at the pairs' tokens a row later, when the others' stores of their row are done.
// 4096 x 32768 bf16, 32 pairs: 200 us with a row's loss and gradient behind one another in all warps, 117 like this.
constexpr int kStages = 2;
constexpr int kMostWarps = 31;
struct StreamShared {
  uint64_t full[kStages];                  // copies
  Sum stats[2][kMostWarps];                // of the warps, of rows in turn
  int teacher[2];                          // whether the row has one
  int gave_up, asked;                      // whether a wait for a copy did; rows, from the CTA's first on, that were asked for
  uint32_t seen[kMostWarps * 40];          // a bit for each element
  int32_t id[kMaxPairs];                   // where a token occurs twice
  float q[kMaxPairs];
};
__device__ __forceinline__ uint32_t shared_address(const void* p) { return static_cast<uint32_t>(__cvta_generic_to_shared(p)); }
__device__ __forceinline__ void expect_bytes(uint32_t bar, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void bulk_load(uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  expect_bytes(bar, bytes);
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst), "l"(src), "r"(bytes), "r"(bar)
               : "memory");
}

// Waits for a phase of a barrier, a second at most.
__device__ __forceinline__ bool phase_done(uint32_t bar, uint32_t parity) {
  uint64_t t0 = 0;
  for (uint32_t it = 1;; ++it) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n\tselp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok)
                 : "r"(bar), "r"(parity), "r"(100000)
                 : "memory");
    if (ok) return true;
    if (it % 8 == 0) {
      uint64_t now;
      asm volatile("mov.u64 %0, %%globaltimer;" : "=l"(now));
      if (t0 == 0) t0 = now;
      else if (now - t0 > 1000000000ull) return false;
    }
  }
}
__device__ __forceinline__ float redux_max(float v) {
  asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(v));
  return v;
}

// Waits for the last copy to each buffer of the rows that were asked for; a copy's parity is that of its turn of the buffer.  (A
// function of its own: inlined, it took registers from the rows' loop, 4096 x 32768 with 64 pairs 121 and 129 us.)
__device__ __noinline__ void copies_end(uint32_t full, int asked) {
  for (int i = max(0, asked - kStages); i < asked; ++i) phase_done(full + i % kStages * 8, i / kStages & 1);
}

// blockDim.x: 32 threads for every warp with elements, and 32.  KP: pairs of a lane of the last warp (4: of short rows alone,
// which have registers for them).
template <int KP, int kValues>
constexpr int kStreamThreads = KP == 4 ? 192 : (kValues == 32 ? 16 : kMostWarps) * 32 + 32;
template <typename T, int KP, int kValues>
__global__ void __launch_bounds__(kStreamThreads<KP, kValues>, KP == 4 ? 5 : kValues == 32 ? 2 : 1) distill_stream_kernel(const DistillArgs a) {
  constexpr int VEC = Elem<T>::kVec, U = kValues / VEC;
  extern __shared__ __align__(16) uint8_t stage_memory[];   // [kStages][part] elements
  __shared__ StreamShared sh;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int warps = blockDim.x / 32 - 1, NT = warps * 32, part = NT * kValues;
  const int64_t first = blockIdx.x, step = gridDim.x;
  const int V = (int)a.V;
  const float c = a.inv_t * kLog2e;
  // Of a row: its first element; where what the threads hold begins (ahead of the row by up to a piece); its
  // whole pieces, which are copied (partial ones are loaded by the threads that have them).
  const auto row_at = [&](int64_t r) { return static_cast<const T*>(a.logits) + r * a.ld; };
  const auto begin_of = [&](const T* row) { return -row_shift(row); };
  const auto first_whole = [&](int begin) { return begin < 0 ? 1 : 0; };
  const auto whole_bytes = [&](int begin) {
    const int last = min(part / VEC, max(0, V - begin) / VEC);
    return (uint32_t)max(0, last - first_whole(begin)) * 16u;
  };
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i)
      asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(&sh.full[i])));
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  for (int i = threadIdx.x; i < kMostWarps * 40; i += blockDim.x) sh.seen[i] = 0;
  if (threadIdx.x == 0) sh.gave_up = 0;
  launch_gate();
  __syncthreads();
  // The one barrier of a row.  (Nobody is a whole row ahead of it: two buffers for the statistics do.)
  const auto meet = [&] {
    __syncwarp();
    __syncthreads();
  };
  // Statistics of row n, behind its barrier, by a warp.
  const auto joined = [&](int n) {
    float m = -INFINITY;
    for (int i = lane; i < warps; i += 32) m = fmaxf(m, sh.stats[n & 1][i].m);
    Sum r;
    r.m = redux_max(m);
    r.s = 0.f;
    for (int i = lane; i < warps; i += 32) {
      const Sum v = sh.stats[n & 1][i];
      r.s += v.m == -INFINITY ? v.s : v.s * ex2((v.m - base_of(r.m)) * c);
    }
    r.s = warp_sum(r.s);
    return r;
  };
  bool gave_up = false;
  // (one lane waits for its warp: of all lanes' polling the other warps would feel.)  A warp that gives up waits no more, and says so
  // ahead of its row's barrier.  The last warp, behind it, asks for no more copies then, so that no barrier sees more turns than have
  // ended, and at its end waits for those that are on their way, before the CTA gives their memory back.
  const auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (lane == 0 && !gave_up && !phase_done(shared_address(bar), parity)) sh.gave_up = gave_up = true;
    __syncwarp();
  };

  if (warp < warps) {
    uint32_t copies = 0;   // bit i: parity of the next copy to buffer i
    int n = 0;
    for (int64_t r = first; r < a.rows; r += step, ++n) {
      const T* row = row_at(r);
      const int begin = begin_of(row);
      const float weight = a.d_loss ? a.d_loss[r] : 0.f;   // (used behind the wait)
      if (whole_bytes(begin)) {
        wait(&sh.full[n % kStages], copies >> (n % kStages) & 1);
        copies ^= 1u << (n % kStages);
      }
      const T* part_row = reinterpret_cast<const T*>(stage_memory) + (n % kStages) * part;
      uint4 w[U];
      float mx = -INFINITY;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int at = (u * NT + (int)threadIdx.x) * VEC, j = begin + at;
        if (j >= 0 && j + VEC <= V) w[u] = *reinterpret_cast<const uint4*>(part_row + at);
        else w[u] = load_raw<T>(row, j, V, minus_inf<T>());
        mx = fmaxf(mx, raw_max<T, false>(w[u]));
      }
      const float m = redux_max(mx);
      f32x2 e[U][VEC / 2];
      f32x2 s2 = 0;
      {
        const float base = -base_of(m);
        const f32x2 minus_base = pack2f(base, base), c2 = pack2f(c, c);
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
          for (int i = 0; i < VEC / 2; ++i) {
            float lo, hi;
            unpack2f(mul2(add2(raw_pair<T>(w[u], i), minus_base), c2), lo, hi);
            e[u][i] = pack2f(ex2(lo), ex2(hi));
            s2 = add2(s2, e[u][i]);
          }
      }
      float lo, hi;
      unpack2f(s2, lo, hi);
      const float s = warp_sum(lo + hi);
      if (lane == 0) sh.stats[n & 1][warp] = Sum{m, s};
      // (behind this the last warp reuses the row's buffer, and stores where this warp stored for the row before)
      meet();
      if (!a.d_loss) continue;   // the loss alone
      const Sum student = joined(n);
      T* out = static_cast<T*>(a.d_logits) + r * a.ldd;
      const bool aligned = row_shift(out) == row_shift(row);
      if (weight == 0.f || empty(student) || !sh.teacher[n & 1]) {
        const float none[VEC] = {};
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int j = begin + (u * NT + (int)threadIdx.x) * VEC;
          if (j < V) store_floats<T, VEC, true>(out, j, V, aligned, none);
        }
      } else {
        // (values relative to the warp's own maximum)
        const float scale = weight * a.inv_t / student.s * (m == -INFINITY ? 1.f : ex2((m - base_of(student.m)) * c));
        const f32x2 scale2 = pack2f(scale, scale);
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int j = begin + (u * NT + (int)threadIdx.x) * VEC;
          float d[VEC];
#pragma unroll
          for (int i = 0; i < VEC / 2; ++i) unpack2f(mul2(e[u][i], scale2), d[2 * i], d[2 * i + 1]);
          if (j < V) store_floats<T, VEC, true>(out, j, V, aligned, d);
        }
      }
    }
    meet();   // the last row's stores are done
  } else {
    const auto request = [&](int64_t r, int n) {
      if (lane != 0 || r >= a.rows) return;
      sh.asked = n + 1;
      const T* row = row_at(r);
      const int begin = begin_of(row), skip = first_whole(begin) * VEC;
      const uint32_t bytes = whole_bytes(begin);
      if (bytes)
        bulk_load(shared_address(stage_memory) + ((n % kStages) * part + skip) * (int)sizeof(T), row + begin + skip, bytes,
                  shared_address(&sh.full[n % kStages]));
    };
    // Three loads deep (the id, the logits there): the ids come two rows ahead, the rest one.
    const auto fetch_ids = [&](int64_t r, int32_t* id) {
#pragma unroll
      for (int i = 0; i < KP; ++i) id[i] = r < a.rows && i * 32 + lane < a.K ? a.ids[r * a.K + i * 32 + lane] : -1;
    };
    const auto fetch_pairs = [&](int64_t r, const int32_t* id, Pair* p) {
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        p[i] = Pair{-1, -INFINITY, 0.f};
        if (id[i] >= 0 && id[i] < V) {
          p[i].id = id[i];
          p[i].z = load_any(a.teacher, a.teacher_dtype, r * a.K + i * 32 + lane);
          p[i].x = Elem<T>::to_float(row_at(r)[id[i]]);
        }
      }
    };
    for (int i = 0; i < kStages; ++i) request(first + i * step, i);
    int32_t ids[KP];
    Pair now[KP], next[KP];
    fetch_ids(first, ids);
    fetch_pairs(first, ids, next);
    fetch_ids(first + step, ids);
    int32_t old_id[KP];   // the last row's tokens, and their gradients
    float old_d[KP];
    T* old_out = nullptr;
    const auto store_old = [&] {
      if (!old_out) return;
#pragma unroll
      for (int i = 0; i < KP; ++i)
        if (old_id[i] >= 0) old_out[old_id[i]] = Elem<T>::from_float(old_d[i]);
    };
    int n = 0;
    for (int64_t r = first; r < a.rows; r += step, ++n) {
      const float weight = a.d_loss ? a.d_loss[r] : 0.f;
#pragma unroll
      for (int i = 0; i < KP; ++i) now[i] = next[i];
      if (r + step < a.rows) fetch_pairs(r + step, ids, next);
      fetch_ids(r + 2 * step, ids);
      // the teacher's side
      Sum teacher{-INFINITY, 0.f};
#pragma unroll
      for (int i = 0; i < KP; ++i) teacher.m = fmaxf(teacher.m, now[i].z);
      teacher.m = redux_max(teacher.m);
#pragma unroll
      for (int i = 0; i < KP; ++i) teacher.s += ex2((now[i].z - base_of(teacher.m)) * c);
      teacher.s = warp_sum(teacher.s);
      const bool none = empty(teacher);
      const float log_teacher = log_sum(teacher);
      if (lane == 0) sh.teacher[n & 1] = !none;
      // Whether a token occurs twice: a bit for each (cleared at once: one warp's own).
      const int begin = begin_of(row_at(r));
      uint32_t twice = 0;
      const auto in_part = [&](int32_t id) { return id >= 0 && id >= begin && id < begin + part; };
#pragma unroll
      for (int i = 0; i < KP; ++i)
        if (in_part(now[i].id)) {
          const int at = now[i].id - begin;
          twice |= atomicOr(&sh.seen[at >> 5], 1u << (at & 31)) >> (at & 31) & 1u;
        }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < KP; ++i)
        if (in_part(now[i].id)) sh.seen[(now[i].id - begin) >> 5] = 0;
      const bool any_twice = __any_sync(0xffffffffu, twice != 0);
      meet();
      store_old();
      if (!sh.gave_up) request(r + kStages * step, n + kStages);
      const Sum student = joined(n);
      const float log_s = log_sum(student);
      float loss = 0.f, q[KP];
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const PairTerm t = pair_term(now[i], teacher, log_teacher, student, log_s, a.inv_t, c);
        q[i] = t.q;
        loss += t.loss;
      }
      loss = warp_sum(loss);
      if (lane == 0 && a.loss) {   // (none: a gradient that is asked for later)
        a.loss[r] = loss;
        a.stats[2 * r] = student.m;
        a.stats[2 * r + 1] = log_s;
      }
      old_out = weight == 0.f || none || empty(student) ? nullptr : static_cast<T*>(a.d_logits) + r * a.ldd;
#pragma unroll
      for (int i = 0; i < KP; ++i) old_id[i] = in_part(now[i].id) ? now[i].id : -1;
      if (any_twice) {
        // the first of the pairs with a token has the sum of all of them
#pragma unroll
        for (int i = 0; i < KP; ++i) {
          sh.id[i * 32 + lane] = now[i].id;
          sh.q[i * 32 + lane] = q[i];
        }
        __syncwarp();
#pragma unroll
        for (int i = 0; i < KP; ++i) {
          q[i] = 0.f;
          for (int e = 0; e < a.K; ++e)
            if (sh.id[e] == now[i].id) {
              q[i] += sh.q[e];
              if (e < i * 32 + lane) old_id[i] = -1;
            }
        }
        __syncwarp();
      }
      const float g = weight * a.inv_t, base = base_of(student.m), scale = g / student.s;
#pragma unroll
      for (int i = 0; i < KP; ++i) old_d[i] = fmaf(-g, q[i], scale * ex2((now[i].x - base) * c));
    }
    meet();
    store_old();
    if (sh.gave_up) copies_end(shared_address(sh.full), sh.asked);
  }
  if (gave_up) atomicExch(a.status, (int)OLSGD_ETIMEOUT);
}

// ------------------------------------------------------------------------------ host
int64_t chunk_count(int64_t V, int dtype) {
  return (V + (dtype == OLSGD_F32 ? 3 : 7) + kChunkElems - 1) / kChunkElems;
}
struct Plan {
  int nchunks, cps, nsplit;   // chunks of a row; chunks per part; parts
};
// Parts of a row: as many as give every multiprocessor four CTAs, none shorter than a turn of a CTA's warps.
Plan plan(int64_t rows, int64_t V, int dtype) {
  Plan p;
  p.nchunks = (int)chunk_count(V, dtype);
  const int64_t want = (4LL * 148 + rows - 1) / rows, most = (p.nchunks + kWarps * 4 - 1) / (kWarps * 4);
  int64_t n = want < most ? want : most;
  if (n > kMaxSplit) n = kMaxSplit;
  if (n < 1) n = 1;
  p.cps = (int)((p.nchunks + n - 1) / n);
  p.nsplit = (p.nchunks + p.cps - 1) / p.cps;
  return p;
}
// Loss and gradient from one read, by a CTA that holds the row: its warps with elements and a thread's elements; no warps where two
// passes are taken.  Up to 16384 elements of 32 a thread, of which a multiprocessor holds several CTAs; above, 40 a thread, one CTA.
// Longer rows take two passes: by clusters of two to eight CTAs they took 146 to 175 us (2048 x 65536 to 837 x 160001 bf16), by
// two passes 145 to 148.  So do more pairs than the one warp deals with beside the row: one read and two passes, us, bf16, 96M
// logits: 64 pairs, V = 4000 97 and 315, 16000 87 and 128, 38000 88 and 110; 128 pairs, V = 1500 252 and 909, 4000 152 and 354.
// (Past kManyPairsMax, 128 pairs: 8000 128 and 195, 16000 127 and 142, of a kernel that has become faster since the bound was
// set by 271 and 212.)  256 pairs took 1330 and more by one read, by two passes 134 (38000) to 1360 (1500).
// A loss alone takes a CTA that stays where the row is short, which else costs a CTA's start and its barriers each: like
// this and a CTA a row, us, 96M logits (fp32 48M): 32 pairs, bf16, V = 1500 107 and 369, 4000 62 and 147, 8000 56 and 68,
// 16000 59 and 50; fp32 4000 48 and 76, 8000 44 and 39; 64 pairs, bf16, 4000 77 and 150, 8000 90 and 70.  So does a
// gradient that is asked for later: bf16, V = 1500 154 and 403, 4000 92 and 153, 8000 81 and 92, 16000 83 and 76.
// aligned: all rows start on a 16-byte boundary.
struct Held {
  int warps, values;
};
constexpr int kManyPairsMax = 4096;   // longest row that is held with more than 64 pairs
static_assert((kManyPairsMax + 7 + 1023) / 1024 * 32 + 32 <= kStreamThreads<4, 32>, "threads of a row with many pairs");
bool is_short(int64_t V, int K, int dtype) { return K <= 64 && V * (dtype == OLSGD_F32 ? 4 : 2) <= (K <= 32 ? 16384 : 8192); }
Held held_by(int64_t V, int K, int dtype, bool aligned, bool gradient) {
  const int64_t n = V + (aligned ? 0 : dtype == OLSGD_F32 ? 3 : 7);
  const int most = (dtype == OLSGD_F32 ? 19 : kMostWarps) * 1280;   // (two buffers of 97 or 78 KB)
  if (!gradient && !is_short(V, K, dtype)) return Held{0, 0};
  if (n > most || K > 128 || (K > 64 && V > kManyPairsMax)) return Held{0, 0};
  return n <= 16 * 1024 ? Held{(int)((n + 1023) / 1024), 32} : Held{(int)((n + 1279) / 1280), 40};
}
template <typename T>
bool rows_aligned(const DistillArgs& a) {
  return ((reinterpret_cast<uintptr_t>(a.logits) | (uintptr_t)(a.ld * sizeof(T))) & 15) == 0;
}

template <typename T, bool LOSS, bool GRAD>
cudaError_t warp_rows(const DistillArgs& a, cudaStream_t s) {
  const dim3 grid((unsigned)((a.rows + kWarps - 1) / kWarps));
  auto k = a.V <= 32    ? distill_warp_kernel<T, 1, LOSS, GRAD>
           : a.V <= 256 ? distill_warp_kernel<T, 8, LOSS, GRAD>
                        : distill_warp_kernel<T, 32, LOSS, GRAD>;
  return launch_chained(k, grid, dim3(kThreads), 0, s, a);
}

// As many CTAs as the GPU holds at once.
template <typename T, int KP, int kValues>
cudaError_t stream_as(DistillArgs a, const Held& h, cudaStream_t s) {
  const int threads = h.warps * 32 + 32;
  const size_t smem = (size_t)kStages * h.warps * 32 * kValues * sizeof(T);
  static PerDeviceSmem configured;
  auto kern = distill_stream_kernel<T, KP, kValues>;
  cudaError_t e = ensure_dynamic_smem(configured, kern, 200 * 1024);
  if (e == cudaSuccess) e = status_word(&a.status);
  if (e != cudaSuccess) return e;
  // (registers, and 227 KB a multiprocessor)
  int64_t resident = 65536 / ((kValues == 40 || KP == 4 ? 64 : 56) * threads), by_memory = 227 * 1024 / (smem + sizeof(StreamShared) + 1024);
  resident = resident < by_memory ? resident : by_memory;
  const int64_t room = sm_count() * (resident < 1 ? 1 : resident);
  return launch_chained(kern, dim3((unsigned)(a.rows < room ? a.rows : room)), dim3(threads), smem, s, a);
}
template <typename T, int kValues>
cudaError_t stream_pairs(const DistillArgs& a, const Held& h, cudaStream_t s) {
  if (a.K <= 32) return stream_as<T, 1, kValues>(a, h, s);
  if constexpr (kValues == 32)
    if (a.K > 64) return stream_as<T, 4, kValues>(a, h, s);
  return stream_as<T, 2, kValues>(a, h, s);
}
template <typename T>
cudaError_t stream_rows(const DistillArgs& a, const Held& h, cudaStream_t s) {
  return h.values == 40 ? stream_pairs<T, 40>(a, h, s) : stream_pairs<T, 32>(a, h, s);
}

template <typename T>
cudaError_t gradient(const DistillArgs& a, cudaStream_t s) {
  if (a.V <= kWarpRowMax) return warp_rows<T, false, true>(a, s);
  // (of short rows the statistics are formed again: a CTA for each row and its barriers take longer)
  const Held h = held_by(a.V, a.K, a.dtype, rows_aligned<T>(a), true);
  if (h.warps > 0 && is_short(a.V, a.K, a.dtype)) return stream_rows<T>(a, h, s);
  const int64_t pieces = (a.V + (rows_aligned<T>(a) ? 1 : 2) * (Elem<T>::kVec - 1)) / Elem<T>::kVec, per = kThreads * kGradPieces;
  const int64_t whole = (pieces + per - 1) / per, want = (kGradCtas + a.rows - 1) / a.rows;   // turns of a row; segments
  const int64_t turns = want >= whole ? 1 : (whole + want - 1) / want;
  const bool large = a.rows * a.V * (int64_t)sizeof(T) > kKeepBytes;   // a gradient that L2 would not hold anyway
  return launch_chained(large ? distill_grad_kernel<T, true> : distill_grad_kernel<T, false>,
                        dim3((unsigned)a.rows, (unsigned)((whole + turns - 1) / turns)), dim3(kThreads), 0, s, a, (int)turns);
}

template <typename T>
cudaError_t forward(const DistillArgs& a, cudaStream_t s) {
  if (a.V <= kWarpRowMax) return a.d_loss ? warp_rows<T, true, true>(a, s) : warp_rows<T, true, false>(a, s);
  const Held h = held_by(a.V, a.K, a.dtype, rows_aligned<T>(a), a.d_loss != nullptr);
  if (h.warps > 0) return stream_rows<T>(a, h, s);
  const Plan p = plan(a.rows, a.V, a.dtype);
  float2* part = p.nsplit > 1 ? static_cast<float2*>(a.ws) : nullptr;
  cudaError_t e = launch_chained(distill_row_kernel<T>, dim3((unsigned)a.rows, (unsigned)p.nsplit), dim3(kThreads), 0, s, a, p.nchunks, p.cps, part);
  if (e == cudaSuccess && part)
    e = launch_chained(distill_finish_kernel<T>, dim3((unsigned)a.rows), dim3(kThreads), 0, s, a, p.nsplit, (const float2*)part);
  return e == cudaSuccess && a.d_loss ? gradient<T>(a, s) : e;
}

}  // namespace

size_t distill_workspace(int dtype, int64_t rows, int64_t V, int K, bool gradient) {
  if (V <= kWarpRowMax || held_by(V, K, dtype, false, gradient).warps > 0) return 0;   // (whatever the alignment)
  const Plan p = plan(rows, V, dtype);
  return p.nsplit == 1 ? 0 : (size_t)rows * p.nsplit * sizeof(float2);
}

cudaError_t launch_distill(const DistillArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case OLSGD_F32: return forward<float>(a, s);
    case OLSGD_BF16: return forward<__nv_bfloat16>(a, s);
    default: return forward<__half>(a, s);
  }
}
cudaError_t launch_distill_backward(const DistillArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case OLSGD_F32: return gradient<float>(a, s);
    case OLSGD_BF16: return gradient<__nv_bfloat16>(a, s);
    default: return gradient<__half>(a, s);
  }
}

}  // namespace olsgd
