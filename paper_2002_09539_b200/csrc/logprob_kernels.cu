// Log probabilities of given tokens, entropy, the most likely alternatives, and the gradient.
//
// For a row x of V logits, m = max x, S = sum exp(x - m):
//   log p_j = (x_j - m) - log S,   H = log S - (1/S) sum exp(x_j - m) (x_j - m).
// One pass keeps a running maximum and, relative to it, s = sum e^d and t = sum e^d d
// (d = x - m, in units of log2): when the maximum rises from m to m', both are carried over
// by s' = s f, t' = (t + s delta) f with delta = (m - m') log2 e, f = 2^delta.  The
// difference x - m is formed before it is scaled, so rows of the type's lowest value, or far
// from zero, keep their probabilities.  All of it is held in fp32.
//
// Alternatives: a warp reads 32 consecutive 16-byte pieces (a chunk) at a time and needs the
// chunk's maximum for the running maximum anyway, so it also stores it.  The k largest
// elements (ties to the lowest index) lie in the k chunks that come first by (maximum, lowest
// index): if an element's chunk is not among them, each of those k chunks holds an element
// that comes before it.  The finishing kernel therefore reads k chunks again and nothing else.
//
// Rows of up to 1024 logits stay in a warp's registers (one launch, no second read).  Longer
// ones are bound by reading the logits once; a row is split over several CTAs when there are
// fewer rows than the GPU has room for, and the parts are joined by the finishing kernel.
#include "operator_common.cuh"
#include "operators_internal.h"

namespace olsgd {
namespace {

using namespace op;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kUnrollChunks = 4;      // 16-byte loads a lane has in flight
constexpr int kWarpRowMax = 1024;     // longest row that stays in a warp's registers
constexpr int kMaxTop = OLSGD_MAX_TOP;
static_assert(kMaxTop == 32, "a lane holds one candidate of each warp");
constexpr int kMaxSplit = 64;

struct RowState {
  float m, s, t;   // running maximum; sums relative to it (t in log2 units)
};

// e^(x - m) and its product with the exponent.  The clamp keeps 0 * -inf out of t (e is zero
// long before); a NaN stays in e and reaches both sums.
__device__ __forceinline__ void accumulate(float x, float base, float& s, float& t) {
  const float d = (x - base) * kLog2e;
  const float e = ex2(d);
  s += e;
  t = fmaf(e, fmaxf(d, -1000.f), t);
}

// Carries (s, t) from maximum `from` to the larger maximum `to`.
__device__ __forceinline__ void rebase(float from, float to, float& s, float& t) {
  if (from == -INFINITY) return;   // nothing but zeros (or a NaN) so far
  const float delta = fmaxf((from - to) * kLog2e, -1000.f);
  const float f = ex2(delta);
  t = fmaf(s, delta, t) * f;
  s *= f;
}

__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.f : m; }

__device__ __forceinline__ RowState join(const RowState& a, const RowState& b) {
  RowState r;
  r.m = fmaxf(a.m, b.m);
  float sa = a.s, ta = a.t, sb = b.s, tb = b.t;
  rebase(a.m, r.m, sa, ta);
  rebase(b.m, r.m, sb, tb);
  r.s = sa + sb;
  r.t = ta + tb;
  return r;
}

__device__ __forceinline__ RowState shfl_join(RowState v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) {
    RowState w;
    w.m = __shfl_xor_sync(0xffffffffu, v.m, o);
    w.s = __shfl_xor_sync(0xffffffffu, v.s, o);
    w.t = __shfl_xor_sync(0xffffffffu, v.t, o);
    v = join(v, w);
  }
  return v;
}

// ---- alternatives: keys that order by (value, lowest index), NaN first, -0 equal to +0
// (every key is below ~0, the first limit of a selection, and above 0, "none")
constexpr uint32_t kNanOrder = 0xFFFFFFFEu;
__device__ __forceinline__ uint32_t order_of(float v) {
  uint32_t u = __float_as_uint(v);
  if (u == 0x80000000u) u = 0;
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return kNanOrder;
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t o) {
  if (o == kNanOrder) return __uint_as_float(0x7FFFFFFFu);
  return __uint_as_float((o >> 31) ? (o & 0x7FFFFFFFu) : ~o);
}
__device__ __forceinline__ uint64_t key_of(uint32_t order, int64_t index) {
  return ((uint64_t)order << 32) | (uint32_t)(0xFFFFFFFFu - (uint32_t)index);
}
__device__ __forceinline__ int32_t index_of(uint64_t key) { return (int32_t)(0xFFFFFFFFu - (uint32_t)key); }
__device__ __forceinline__ uint64_t warp_max_key(uint64_t k) {
  const uint32_t hi = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32));
  const uint32_t lo = __reduce_max_sync(0xffffffffu, (uint32_t)(k >> 32) == hi ? (uint32_t)k : 0u);
  return ((uint64_t)hi << 32) | lo;
}

// The up-to-k largest keys of a set whose members each lane can rescan: own_max(limit) gives
// the lane's largest key below `limit` (0: none).  emit(r, key) is called by lane 0.  Stops
// early at keys below `floor_key`.
template <typename OwnMax, typename Emit>
__device__ __forceinline__ int warp_select(int k, uint64_t floor_key, OwnMax own_max, Emit emit) {
  const int lane = threadIdx.x & 31;
  uint64_t best = own_max(~0ull);
  int r = 0;
  for (; r < k; ++r) {
    const uint64_t w = warp_max_key(best);
    if (w == 0 || w < floor_key) break;
    if (lane == 0) emit(r, w);
    if (best == w) best = own_max(w);
  }
  return r;
}

struct RowOut {
  const int32_t* targets;
  float *logp, *entropy, *stats;
};

// A row whose logits are all -inf has no distribution: log p = -inf, entropy 0, and a zero
// gradient (its statistics are (-inf, 0)).
__device__ __forceinline__ float log_sum(const RowState& v) {
  return (v.m == -INFINITY && v.s == 0.f) ? 0.f : logf(v.s);
}
__device__ __forceinline__ float log_prob(float x, const RowState& v, float log_s) {
  return (v.m == -INFINITY && v.s == 0.f) ? -INFINITY : (x - base_of(v.m)) - log_s;
}

template <typename T>
__device__ __forceinline__ void write_row(const RowOut& o, const T* row, int64_t r, int64_t V,
                                          const RowState& v) {
  const float log_s = log_sum(v);
  const int32_t t = o.targets[r];
  const bool empty = v.m == -INFINITY && v.s == 0.f;
  float h = empty ? 0.f : log_s - 0.6931471805599453f * (v.t / v.s);
  if (h < 0.f) h = 0.f;   // rounding of a row that is certain; a NaN stays
  o.entropy[r] = h;
  o.stats[2 * r] = v.m;
  o.stats[2 * r + 1] = log_s;
  // a target outside [0, V) marks a row without a token
  o.logp[r] = (t >= 0 && t < V) ? log_prob(Elem<T>::to_float(row[t]), v, log_s) : 0.f;
}

// ------------------------------------------------------------ rows in a warp's registers
template <typename T, int NL>
__global__ void __launch_bounds__(kThreads)
logprob_warp_kernel(const T* __restrict__ x, int64_t rows, int V, int64_t ld, RowOut o, int top,
                    float* __restrict__ top_logp, int32_t* __restrict__ top_ids) {
  launch_gate();
  const int lane = threadIdx.x & 31;
  const int64_t r = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (r >= rows) return;
  const T* row = x + r * ld;
  float v[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) {
    const int j = i * 32 + lane;
    v[i] = j < V ? Elem<T>::to_float(row[j]) : -INFINITY;
  }
  RowState st;
  float mx = v[0];
#pragma unroll
  for (int i = 1; i < NL; ++i) mx = fmaxf(mx, v[i]);
#pragma unroll
  for (int off = 16; off; off >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, off));
  st.m = mx;
  if (!(mx > -INFINITY)) st.m = -INFINITY;   // all -inf, or nothing but NaN
  const float base = base_of(st.m);
  st.s = st.t = 0.f;
#pragma unroll
  for (int i = 0; i < NL; ++i) accumulate(v[i], base, st.s, st.t);
  st.s = warp_sum(st.s);
  st.t = warp_sum(st.t);
  if (lane == 0) write_row<T>(o, row, r, V, st);
  if (top > 0) {
    const float log_s = log_sum(st);
    warp_select(
        top, 0,
        [&](uint64_t limit) {
          uint64_t b = 0;
#pragma unroll
          for (int i = 0; i < NL; ++i) {
            const int j = i * 32 + lane;
            const uint64_t key = key_of(order_of(v[i]), j);
            if (j < V && key < limit && key > b) b = key;
          }
          return b;
        },
        [&](int q, uint64_t key) {
          top_ids[r * top + q] = index_of(key);
          top_logp[r * top + q] = log_prob(value_of((uint32_t)(key >> 32)), st, log_s);
        });
  }
}

// -------------------------------------------------------------------------- long rows
// CTA (r, split): chunks [split * cps, (split + 1) * cps) of row r, dealt to the warps in turn.
template <typename T, bool TOP, bool WHOLE>
__global__ void __launch_bounds__(kThreads)
logprob_row_kernel(const T* __restrict__ x, int64_t V, int64_t ld, int nchunks, int cps, RowOut o,
                   float4* __restrict__ part, uint32_t* __restrict__ chunk_max) {
  constexpr int VEC = Elem<T>::kVec;
  constexpr int U = kUnrollChunks;
  launch_gate();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t r = blockIdx.x;
  const T* row = x + r * ld;
  const int shift = row_shift(row);
  const int c_begin = blockIdx.y * cps, c_end = min(nchunks, c_begin + cps);

  RowState st{-INFINITY, 0.f, 0.f};
  for (int c0 = c_begin + warp; c0 < c_end; c0 += kWarps * U) {
    float v[U][VEC];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int c = c0 + u * kWarps;
      if (c < c_end) {
        load_piece<T>(row, ((int64_t)c * 32 + lane) * VEC - shift, V, -INFINITY, v[u]);
      } else {
#pragma unroll
        for (int e = 0; e < VEC; ++e) v[u][e] = -INFINITY;
      }
    }
    float mx = st.m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float cm = v[u][0];
      if (TOP) {
#pragma unroll
        for (int e = 1; e < VEC; ++e) cm = max_nan(cm, v[u][e]);
        // over the warp as an ordered integer, in which a NaN comes first
        const uint32_t order = __reduce_max_sync(0xffffffffu, order_of(cm));
        const int c = c0 + u * kWarps;
        if (lane == 0 && c < c_end) chunk_max[r * nchunks + c] = order;
        cm = value_of(order);   // (a NaN does not move the running maximum)
      } else {
#pragma unroll
        for (int e = 1; e < VEC; ++e) cm = fmaxf(cm, v[u][e]);
      }
      mx = fmaxf(mx, cm);
    }
    if (!TOP) {
      float w;
      asm volatile("redux.sync.max.f32 %0, %1, 0xffffffff;" : "=f"(w) : "f"(mx));
      mx = w;
    }
    if (mx > st.m) {
      rebase(st.m, mx, st.s, st.t);
      st.m = mx;
    }
    const float base = base_of(st.m);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < VEC; ++e) accumulate(v[u][e], base, st.s, st.t);
  }
  st.s = warp_sum(st.s);
  st.t = warp_sum(st.t);
  __shared__ RowState sh[kWarps];
  if (lane == 0) sh[warp] = st;
  __syncthreads();
  if (threadIdx.x == 0) {
    RowState a = sh[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) a = join(a, sh[w]);
    if (WHOLE)
      write_row<T>(o, row, r, V, a);
    else
      part[r * gridDim.y + blockIdx.y] = make_float4(a.m, a.s, a.t, 0.f);
  }
}

// Joins a row's parts and finds its alternatives; one CTA per row.
template <typename T>
__global__ void __launch_bounds__(kThreads)
logprob_finish_kernel(const T* __restrict__ x, int64_t V, int64_t ld, int nchunks, int nsplit, RowOut o,
                      const float4* __restrict__ part, const uint32_t* __restrict__ chunk_max, int top,
                      float* __restrict__ top_logp, int32_t* __restrict__ top_ids) {
  constexpr int VEC = Elem<T>::kVec;
  __shared__ uint64_t cand[kWarps * kMaxTop];
  __shared__ int32_t chosen[kMaxTop];
  __shared__ uint64_t found[kMaxTop * kMaxTop];
  __shared__ int n_found, n_chosen;
  __shared__ uint32_t threshold;
  launch_gate();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t r = blockIdx.x;
  const T* row = x + r * ld;
  const int shift = row_shift(row);

  RowState st{-INFINITY, 0.f, 0.f};
  if (warp == 0) {
    for (int i = lane; i < nsplit; i += 32) {
      const float4 p = part[r * nsplit + i];
      st = join(st, RowState{p.x, p.y, p.z});
    }
    st = shfl_join(st);
    if (lane == 0) write_row<T>(o, row, r, V, st);
  }
  if (top == 0) return;
  // 1. each warp: the best chunks of its share; then warp 0: the best of those
  if (threadIdx.x == 0) n_found = 0;
  const uint32_t* cm = chunk_max + r * nchunks;
  {
    int got = warp_select(
        top, 0,
        [&](uint64_t limit) {
          uint64_t b = 0;
          for (int c = warp * 32 + lane; c < nchunks; c += kThreads) {
            const uint64_t key = key_of(cm[c], c);
            if (key < limit && key > b) b = key;
          }
          return b;
        },
        [&](int q, uint64_t key) { cand[warp * kMaxTop + q] = key; });
    for (int q = got + lane; q < kMaxTop; q += 32) cand[warp * kMaxTop + q] = 0;
  }
  __syncthreads();
  if (warp == 0) {
    uint64_t last = 0;
    const int got = warp_select(
        top, 0,
        [&](uint64_t limit) {
          uint64_t b = 0;
#pragma unroll
          for (int w = 0; w < kWarps; ++w) {
            const uint64_t key = cand[w * kMaxTop + lane];
            if (key < limit && key > b) b = key;
          }
          return b;
        },
        [&](int q, uint64_t key) {
          chosen[q] = index_of(key);
          last = key;
        });
    if (lane == 0) {
      n_chosen = got;
      // with k chunks chosen, k elements are at least as large as the last one's maximum
      threshold = got == top ? (uint32_t)(last >> 32) : 0u;
    }
  }
  __syncthreads();
  // 2. the elements of the chosen chunks that can be among the k largest
  const uint64_t floor_key = (uint64_t)threshold << 32;
  for (int i = warp; i < n_chosen; i += kWarps) {
    const int64_t j0 = ((int64_t)chosen[i] * 32 + lane) * VEC - shift;
    float v[VEC];
    load_piece<T>(row, j0, V, -INFINITY, v);
    warp_select(
        top, floor_key,
        [&](uint64_t limit) {
          uint64_t b = 0;
#pragma unroll
          for (int e = 0; e < VEC; ++e) {
            const int64_t j = j0 + e;
            const uint64_t key = key_of(order_of(v[e]), j);
            if (j >= 0 && j < V && key < limit && key > b) b = key;
          }
          return b;
        },
        [&](int, uint64_t key) { found[atomicAdd(&n_found, 1)] = key; });
  }
  __syncthreads();
  // 3. the k largest of those, in order (the list's own order does not matter: keys differ)
  if (warp == 0) {
    const float log_s = log_sum(st);
    const int n = n_found;
    warp_select(
        top, 0,
        [&](uint64_t limit) {
          uint64_t b = 0;
          for (int i = lane; i < n; i += 32) {
            const uint64_t key = found[i];
            if (key < limit && key > b) b = key;
          }
          return b;
        },
        [&](int q, uint64_t key) {
          top_ids[r * top + q] = index_of(key);
          top_logp[r * top + q] = log_prob(value_of((uint32_t)(key >> 32)), st, log_s);
        });
  }
}

// ---------------------------------------------------------------------------- gradient
// dx_j = dlp (1[j = t] - p_j) - dH p_j (log p_j + H): reads the logits once, writes once.
struct GradRow {
  float base, log_s, d_lp, d_h, h;
  int32_t target;
  bool empty;
  __device__ __forceinline__ float operator()(float x, int64_t j) const {
    if (empty) return 0.f;
    const float lp = fmaxf((x - base) - log_s, -1.0e4f);   // p is zero there; a NaN is put back below
    const float p = ex2(((x - base) - log_s) * kLog2e);
    float d = -p * fmaf(d_h, lp + h, d_lp);
    if (j == target) d += d_lp;
    return d;
  }
};

__device__ __forceinline__ GradRow grad_row(const LogprobGradArgs& a, int64_t r) {
  GradRow g;
  const float m = a.stats[2 * r];
  g.log_s = a.stats[2 * r + 1];
  g.empty = m == -INFINITY && g.log_s == 0.f;
  g.base = base_of(m);
  const int32_t t = a.targets[r];
  const bool has = t >= 0 && t < a.V;
  g.target = has ? t : -1;
  g.d_lp = has && a.d_logp ? a.d_logp[r] : 0.f;
  g.d_h = a.d_entropy ? a.d_entropy[r] : 0.f;
  g.h = a.entropy[r];
  return g;
}

template <typename T>
__global__ void __launch_bounds__(kThreads) logprob_grad_warp_kernel(LogprobGradArgs a) {
  launch_gate();
  const int lane = threadIdx.x & 31;
  const int64_t r = (int64_t)blockIdx.x * kWarps + (threadIdx.x >> 5);
  if (r >= a.rows) return;
  const T* row = static_cast<const T*>(a.logits) + r * a.ld;
  T* out = static_cast<T*>(a.d_logits) + r * a.ldd;
  const GradRow g = grad_row(a, r);
  for (int64_t j = lane; j < a.V; j += 32) out[j] = Elem<T>::from_float(g(Elem<T>::to_float(row[j]), j));
}

// CTA (r, segment): kThreads * kUnrollChunks pieces of row r.
template <typename T>
__global__ void __launch_bounds__(kThreads) logprob_grad_kernel(LogprobGradArgs a) {
  constexpr int VEC = Elem<T>::kVec;
  constexpr int U = kUnrollChunks;
  launch_gate();
  const int64_t r = blockIdx.x;
  const T* row = static_cast<const T*>(a.logits) + r * a.ld;
  T* out = static_cast<T*>(a.d_logits) + r * a.ldd;
  const int shift = row_shift(row);
  const bool aligned = row_shift(out) == shift;
  const GradRow g = grad_row(a, r);
  const int64_t q0 = (int64_t)blockIdx.y * (kThreads * U) + threadIdx.x;
  float v[U][VEC];
#pragma unroll
  for (int u = 0; u < U; ++u) load_piece<T>(row, (q0 + u * kThreads) * VEC - shift, a.V, 0.f, v[u]);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t j = (q0 + u * kThreads) * VEC - shift;
    float d[VEC];
#pragma unroll
    for (int e = 0; e < VEC; ++e) d[e] = g(v[u][e], j + e);
    store_floats<T, VEC>(out, j, a.V, aligned, d);
  }
}

// ------------------------------------------------------------------------------ host
int chunk_elems(int dtype) { return 32 * (dtype == OLSGD_F32 ? 4 : 8); }
// upper bound over every alignment of a row
int64_t chunk_count(int64_t V, int dtype) {
  const int64_t ce = chunk_elems(dtype);
  return (V + ce / 32 - 1 + ce - 1) / ce;
}
// Parts a row is split into.  One part per row once the rows alone give every multiprocessor
// four CTAs; before that as many parts as fill the GPU that often, none shorter than one
// unrolled turn of a CTA's warps (32 chunks).
int split_count(int64_t rows, int64_t nchunks) {
  const int64_t want = (4LL * 148 + rows - 1) / rows;
  const int64_t most = (nchunks + kWarps * kUnrollChunks - 1) / (kWarps * kUnrollChunks);
  int64_t n = want < most ? want : most;
  if (n > kMaxSplit) n = kMaxSplit;
  return n < 1 ? 1 : (int)n;
}

struct Plan {
  int nchunks, cps, nsplit;   // chunks of a row; chunks per part; parts
};
Plan plan(int64_t rows, int64_t V, int dtype) {
  Plan p;
  p.nchunks = (int)chunk_count(V, dtype);
  const int want = split_count(rows, p.nchunks);
  p.cps = (p.nchunks + want - 1) / want;
  p.nsplit = (p.nchunks + p.cps - 1) / p.cps;
  return p;
}

template <typename T>
cudaError_t forward(const LogprobArgs& a, cudaStream_t s) {
  const T* x = static_cast<const T*>(a.logits);
  const RowOut o{a.targets, a.logp, a.entropy, a.stats};
  if (a.V <= kWarpRowMax) {
    const dim3 grid((unsigned)((a.rows + kWarps - 1) / kWarps));
    auto k = a.V <= 32 ? logprob_warp_kernel<T, 1> : a.V <= 256 ? logprob_warp_kernel<T, 8> : logprob_warp_kernel<T, 32>;
    return launch_chained(k, grid, dim3(kThreads), 0, s, x, a.rows, (int)a.V, a.ld, o, a.top, a.top_logp, a.top_ids);
  }
  const Plan p = plan(a.rows, a.V, a.dtype);
  const int nchunks = p.nchunks, cps = p.cps, nsplit = p.nsplit;
  float4* part = static_cast<float4*>(a.ws);
  uint32_t* cmax = reinterpret_cast<uint32_t*>(part + a.rows * nsplit);
  const dim3 grid((unsigned)a.rows, (unsigned)nsplit);
  const bool whole = nsplit == 1 && a.top == 0;
  auto k = a.top > 0 ? logprob_row_kernel<T, true, false>
           : whole   ? logprob_row_kernel<T, false, true>
                     : logprob_row_kernel<T, false, false>;
  const cudaError_t e = launch_chained(k, grid, dim3(kThreads), 0, s, x, a.V, a.ld, nchunks, cps, o, part, cmax);
  if (e != cudaSuccess || whole) return e;
  return launch_chained(logprob_finish_kernel<T>, dim3((unsigned)a.rows), dim3(kThreads), 0, s, x, a.V, a.ld, nchunks,
                        nsplit, o, (const float4*)part, (const uint32_t*)cmax, a.top, a.top_logp, a.top_ids);
}

template <typename T>
cudaError_t backward(const LogprobGradArgs& a, cudaStream_t s) {
  if (a.V <= kWarpRowMax)
    return launch_chained(logprob_grad_warp_kernel<T>, dim3((unsigned)((a.rows + kWarps - 1) / kWarps)), dim3(kThreads),
                          0, s, a);
  const int64_t pieces = (a.V + 2 * Elem<T>::kVec - 2) / Elem<T>::kVec;
  const int64_t per = kThreads * kUnrollChunks;
  return launch_chained(logprob_grad_kernel<T>, dim3((unsigned)a.rows, (unsigned)((pieces + per - 1) / per)),
                        dim3(kThreads), 0, s, a);
}

}  // namespace

size_t logprob_workspace(int dtype, int64_t rows, int64_t V, int top) {
  if (V <= kWarpRowMax) return 0;
  const Plan p = plan(rows, V, dtype);
  if (p.nsplit == 1 && top == 0) return 0;
  // the parts of every row, and the chunk maxima
  return (size_t)rows * p.nsplit * sizeof(float4) + (top > 0 ? (size_t)rows * p.nchunks * sizeof(uint32_t) : 0);
}

cudaError_t launch_logprobs(const LogprobArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case OLSGD_F32: return forward<float>(a, s);
    case OLSGD_BF16: return forward<__nv_bfloat16>(a, s);
    default: return forward<__half>(a, s);
  }
}

cudaError_t launch_logprobs_backward(const LogprobGradArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case OLSGD_F32: return backward<float>(a, s);
    case OLSGD_BF16: return backward<__nv_bfloat16>(a, s);
    default: return backward<__half>(a, s);
  }
}

}  // namespace olsgd
