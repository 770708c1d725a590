// Routing of tokens to experts, and the experts' results on their way back, worker-batched.
//
// Route: the k largest of a token's E logits (ties to the lowest expert; -inf is never chosen), their
// softmax, and a stable counting sort of the slots (token, j) by expert: slots of expert e are the
// rows offsets[e] .. offsets[e + 1] - 1, tokens in order.
//   w_j = exp(l_j - l_0) / sum over the chosen, or over all experts, of exp(l - l_0)
//   d_l = w_j (dw_j - sum w dw) at the chosen, or p_e (G_e - sum w dw) everywhere (G: dw at the chosen)
// A warp holds a token's logits in registers, NL consecutive ones a lane, so that the lowest lane
// has the lowest index among equals and a round of the selection is one reduction and one
// ballot.  A warp walks over consecutive tokens; a token's experts differ, so the lanes that hold
// its slots count them without a conflict, and the count before is the slot's rank.  Counts of the
// warps of a CTA are added up there, those of the CTAs by the placing kernel, each of whose CTAs reads
// them all: where one CTA holds all tokens of a worker there is one launch.  No order depends on timing.
//
// Combine: y_t = sum_j w_tj rows[place_tj], in order of j in fp32; its gradient is a product and a dot
// product for each slot.  Both are bound by reading (and writing) each row once.
#include "operator_common.cuh"
#include "operators_internal.h"

namespace olsgd {
namespace {

using namespace op;

constexpr int kSms = 148;
constexpr int kRouteWarps = 32;
constexpr int kRouteThreads = 32 * kRouteWarps;
static_assert(OLSGD_MAX_EXPERTS <= kRouteThreads, "a thread for each expert");
static_assert(OLSGD_MAX_TOP <= 32, "a lane for each slot of a token");

// Values that order as the logits do: 0 for -inf (never chosen), NaN above all.
constexpr uint32_t kNanKey = 0xFFFFFFFEu;
__device__ __forceinline__ uint32_t key_of(float v) {
  uint32_t u = __float_as_uint(v);
  if (u == 0x80000000u) u = 0;
  if ((u & 0x7FFFFFFFu) > 0x7F800000u) return kNanKey;
  if (u == 0xFF800000u) return 0;
  return (u >> 31) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float value_of(uint32_t key) {
  if (key == kNanKey) return __uint_as_float(0x7FFFFFFFu);
  if (key == 0) return -INFINITY;
  return __uint_as_float((key >> 31) ? (key & 0x7FFFFFFFu) : ~key);
}

// A lane's NL consecutive elements of a row of n; those past it are `fill`.  vec: E is a multiple of NL and rows start on
// boundaries of the NL elements (or of 16 bytes).
template <typename T, int NL>
__device__ __forceinline__ void load_lane(const T* row, int n, bool vec, float fill, float* v) {
  const int j0 = (threadIdx.x & 31) * NL;
  constexpr int kBytes = NL * (int)sizeof(T), V = Elem<T>::kVec;
  if (vec) {
    if (j0 < n) {
      if constexpr (kBytes >= 16) {
#pragma unroll
        for (int i = 0; i < NL; i += V) Elem<T>::unpack(ld16(row + j0 + i), v + i);
      } else {
        T raw[NL];
        if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(raw) = *reinterpret_cast<const uint2*>(row + j0);
        else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t*>(raw) = *reinterpret_cast<const uint32_t*>(row + j0);
        else raw[0] = row[j0];
#pragma unroll
        for (int i = 0; i < NL; ++i) v[i] = Elem<T>::to_float(raw[i]);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NL; ++i) v[i] = fill;
    }
  } else {
#pragma unroll
    for (int i = 0; i < NL; ++i) v[i] = j0 + i < n ? Elem<T>::to_float(row[j0 + i]) : fill;
  }
}

struct RouteKernelArgs {
  const void* logits;
  int64_t ld;
  int T, E, k, per_warp;     // tokens of a worker, experts, slots of a token, tokens of a warp
  int normalise, vec;
  float* weights;
  int32_t *ids, *places, *tokens, *offsets;
  int32_t* counts;           // [m][tiles][E], where a worker's tokens take several CTAs
};

// Exclusive sums of v over the CTA's threads.
__device__ __forceinline__ int block_before(int v, int* warp_sums) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  int scan = v;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, scan, off);
    if (lane >= off) scan += up;
  }
  if (lane == 31) warp_sums[warp] = scan;
  __syncthreads();
  if (warp == 0) {
    int s = warp_sums[lane];
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
      const int up = __shfl_up_sync(0xffffffffu, s, off);
      if (lane >= off) s += up;
    }
    warp_sums[lane] = s;
  }
  __syncthreads();
  return scan - v + (warp ? warp_sums[warp - 1] : 0);
}

// CTA (tile, worker): tokens tile * 32 * per_warp and up.
template <typename T, int NL, bool ONE>
__global__ void __launch_bounds__(kRouteThreads, 1) route_kernel(const RouteKernelArgs a) {
  extern __shared__ int count[];   // [kRouteWarps][E]
  __shared__ int warp_sums[32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = a.E, k = a.k;
  const int64_t worker = blockIdx.y;
  int* mine = count + warp * E;
  for (int e = lane; e < E; e += 32) mine[e] = 0;
  __syncwarp();
  launch_gate();
  const int64_t first = ((int64_t)blockIdx.x * kRouteWarps + warp) * a.per_warp;
  const int64_t last = min((int64_t)a.T, first + a.per_warp);
  const T* rows = static_cast<const T*>(a.logits) + worker * a.T * a.ld;
  constexpr bool kAhead = NL <= 8;   // the next token's logits are on their way (registers for 64 a thread)
  float x[NL];
  if (kAhead && first < last) load_lane<T, NL>(rows + first * a.ld, E, a.vec, -INFINITY, x);
  for (int64_t t = first; t < last; ++t) {
    uint32_t key[NL];
    uint32_t best = 0;
    if (!kAhead) load_lane<T, NL>(rows + t * a.ld, E, a.vec, -INFINITY, x);
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      key[i] = key_of(x[i]);
      best = max(best, key[i]);
    }
    if (kAhead && t + 1 < last) load_lane<T, NL>(rows + (t + 1) * a.ld, E, a.vec, -INFINITY, x);
    int id = -1;
    uint32_t chosen = 0, top = 0;
    for (int j = 0; j < k; ++j) {
      const uint32_t most = __reduce_max_sync(0xffffffffu, best);
      if (most == 0) break;
      if (j == 0) top = most;
      const int winner = __ffs(__ballot_sync(0xffffffffu, best == most)) - 1;
      int at = 0;
      if (lane == winner) {
        // the lowest of this lane's that equal it leaves
        bool gone = false;
        best = 0;
#pragma unroll
        for (int i = 0; i < NL; ++i) {
          if (!gone && key[i] == most) {
            gone = true;
            at = i;
            key[i] = 0;
          }
          best = max(best, key[i]);
        }
      }
      at = __shfl_sync(0xffffffffu, at, winner) + winner * NL;
      if (lane == j) {
        id = at;
        chosen = most;
      }
    }
    const float base = value_of(top);
    float e = id >= 0 ? expf(value_of(chosen) - base) : 0.f, total = e;
    if (!a.normalise) {
      // the others, too (those chosen have left)
#pragma unroll
      for (int i = 0; i < NL; ++i)
        if (key[i]) total += expf(value_of(key[i]) - base);
    }
    total = warp_sum(total);
    if (lane < k) {
      const int64_t slot = (worker * a.T + t) * k + lane;
      a.ids[slot] = id;
      a.weights[slot] = id >= 0 ? e / total : 0.f;
      a.places[slot] = id >= 0 ? mine[id]++ : -1;   // (for now: its rank among the warp's slots of this expert)
    }
    __syncwarp();
  }
  __syncthreads();
  // Counts of the warps before, then (one CTA) of the experts before
  int sum = 0;
  if (threadIdx.x < E) {
#pragma unroll 8
    for (int w = 0; w < kRouteWarps; ++w) {
      const int c = count[w * E + threadIdx.x];
      count[w * E + threadIdx.x] = sum;
      sum += c;
    }
  }
  if constexpr (ONE) {
    const int before = block_before(threadIdx.x < E ? sum : 0, warp_sums);
    if (threadIdx.x < E) {
#pragma unroll 8
      for (int w = 0; w < kRouteWarps; ++w) count[w * E + threadIdx.x] += before;
      a.offsets[worker * (E + 1) + threadIdx.x] = before;
    }
    const int all = warp_sums[31];
    if (threadIdx.x == 0) a.offsets[worker * (E + 1) + E] = all;
    for (int64_t r = all + threadIdx.x; r < (int64_t)a.T * k; r += kRouteThreads) a.tokens[worker * a.T * k + r] = -1;
  } else if (threadIdx.x < E) {
    a.counts[(worker * gridDim.x + blockIdx.x) * E + threadIdx.x] = sum;
  }
  __syncthreads();
  // (each lane reads what it has written)
  for (int64_t t = first; t < last; ++t) {
    const int64_t slot = (worker * a.T + t) * k + lane;
    if (lane < k) {
      const int id = a.ids[slot];
      if (id >= 0) {
        const int place = a.places[slot] + mine[id];
        a.places[slot] = place;
        if (ONE) a.tokens[worker * a.T * k + place] = (int32_t)t;
      }
    }
  }
}

// CTA (tile, worker): ranks within the tile become places.
__global__ void __launch_bounds__(kRouteThreads, 1) place_kernel(const RouteKernelArgs a) {
  __shared__ int totals[kRouteThreads], befores[kRouteThreads];
  __shared__ int warp_sums[32];
  launch_gate();
  const int E = a.E, tiles = gridDim.x;
  const int64_t worker = blockIdx.y;
  // threads (part, expert): every part adds up its share of the tiles
  const int parts = kRouteThreads / E, part = threadIdx.x / E, e = threadIdx.x - part * E;
  int total = 0, before = 0;
  if (part < parts) {
    const int32_t* c = a.counts + worker * tiles * E + e;
#pragma unroll 8
    for (int i = part; i < tiles; i += parts) {
      const int n = c[(int64_t)i * E];
      total += n;
      before += i < (int)blockIdx.x ? n : 0;
    }
  }
  totals[threadIdx.x] = total;
  befores[threadIdx.x] = before;
  __syncthreads();
  total = before = 0;
  if (threadIdx.x < E) {
    for (int p = 0; p < parts; ++p) {
      total += totals[p * E + threadIdx.x];
      before += befores[p * E + threadIdx.x];
    }
  }
  __syncthreads();
  const int start = block_before(total, warp_sums);
  if (threadIdx.x < E) {
    befores[threadIdx.x] = start + before;
    if (blockIdx.x == 0) a.offsets[worker * (E + 1) + threadIdx.x] = start;
  }
  const int all = warp_sums[31];
  if (blockIdx.x == 0 && threadIdx.x == 0) a.offsets[worker * (E + 1) + E] = all;
  __syncthreads();
  const int64_t slots = (int64_t)a.T * a.k, per_tile = (int64_t)kRouteWarps * a.per_warp * a.k;
  const int64_t end = min(slots, (blockIdx.x + 1) * per_tile);
  int32_t *places = a.places + worker * slots, *tokens = a.tokens + worker * slots;
  const int32_t* ids = a.ids + worker * slots;
  for (int64_t s = blockIdx.x * per_tile + threadIdx.x; s < end; s += kRouteThreads) {
    const int id = ids[s];
    if (id >= 0) {
      const int place = places[s] + befores[id];
      places[s] = place;
      tokens[place] = (int32_t)(s / a.k);
    }
  }
  for (int64_t r = all + (int64_t)blockIdx.x * kRouteThreads + threadIdx.x; r < slots; r += (int64_t)tiles * kRouteThreads) tokens[r] = -1;
}

// The gradient of a token's logits, by a warp.
template <typename T, int NL>
__global__ void __launch_bounds__(256) route_backward_kernel(const RouteGradArgs a, int vec_in, int vec_out) {
  launch_gate();
  const int lane = threadIdx.x & 31, k = a.k, E = a.E;
  const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (r >= a.rows) return;
  int id = -1;
  float w = 0.f, dw = 0.f;
  if (lane < k) {
    id = a.ids[r * k + lane];
    if (id >= E) id = -1;
    if (id >= 0) {
      w = a.weights[r * k + lane];
      dw = a.d_weights[r * k + lane];
    }
  }
  const float mean = warp_sum(w * dw);
  float d[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) d[i] = 0.f;
  const float at_chosen = a.normalise ? w * (dw - mean) : dw;
  for (int j = 0; j < k; ++j) {
    const int e = __shfl_sync(0xffffffffu, id, j) - lane * NL;
    const float g = __shfl_sync(0xffffffffu, at_chosen, j);
#pragma unroll
    for (int i = 0; i < NL; ++i)
      if (e == i) d[i] += g;
  }
  if (!a.normalise) {
    float x[NL], most = -INFINITY, total = 0.f;
    load_lane<T, NL>(static_cast<const T*>(a.logits) + r * a.ld, E, vec_in, -INFINITY, x);
#pragma unroll
    for (int i = 0; i < NL; ++i) most = fmaxf(most, x[i]);
#pragma unroll
    for (int off = 16; off; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
    // nothing was chosen: nothing is asked of this row (padding: all -inf)
    const bool empty = __ballot_sync(0xffffffffu, id >= 0) == 0;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      x[i] = empty ? 0.f : expf(x[i] - most);
      total += x[i];
    }
    total = empty ? 1.f : warp_sum(total);
#pragma unroll
    for (int i = 0; i < NL; ++i) d[i] = x[i] / total * (d[i] - mean);
  }
  T* out = static_cast<T*>(a.d_logits) + r * E;
  const int j0 = lane * NL;
  constexpr int kBytes = NL * (int)sizeof(T), V = Elem<T>::kVec;
  if (vec_out) {
    if (j0 < E) {
      if constexpr (kBytes >= 16) {
#pragma unroll
        for (int i = 0; i < NL; i += V) *reinterpret_cast<uint4*>(out + j0 + i) = Elem<T>::pack(d + i);
      } else {
        T raw[NL];
#pragma unroll
        for (int i = 0; i < NL; ++i) raw[i] = Elem<T>::from_float(d[i]);
        if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(out + j0) = *reinterpret_cast<uint2*>(raw);
        else if constexpr (kBytes == 4) *reinterpret_cast<uint32_t*>(out + j0) = *reinterpret_cast<uint32_t*>(raw);
        else out[j0] = raw[0];
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < NL; ++i)
      if (j0 + i < E) out[j0 + i] = Elem<T>::from_float(d[i]);
  }
}

// ------------------------------------------------------------------------------ combine

// V elements at p as they lie in memory, to floats and back.  (V == 1: rows of any alignment.)
template <typename T, int V>
__device__ __forceinline__ void load_some(const T* p, float* v) {
  if constexpr (V == 1) v[0] = Elem<T>::to_float(*p);
  else Elem<T>::unpack(ld16(p), v);
}
template <typename T, int V>
__device__ __forceinline__ void store_some(T* p, const float* v) {
  if constexpr (V == 1) *p = Elem<T>::from_float(v[0]);
  else *reinterpret_cast<uint4*>(p) = Elem<T>::pack(v);
}

// Thread: V elements of a token.
template <typename T, int V>
__global__ void __launch_bounds__(256) combine_kernel(const CombineArgs a) {
  launch_gate();
  const int64_t pieces = a.D / V, at = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t token = at / pieces, c = (at - token * pieces) * V;
  if (token >= a.m * a.T) return;
  const int64_t worker = token / a.T;
  const T* rows = static_cast<const T*>(a.rows) + worker * a.rows_worker + c;
  const int32_t* places = a.places + token * a.k;
  const float* weights = a.weights ? a.weights + token * a.k : nullptr;
  float y[V];
#pragma unroll
  for (int e = 0; e < V; ++e) y[e] = 0.f;
  constexpr int U = 4;
  for (int j0 = 0; j0 < a.k; j0 += U) {
    int32_t p[U];
    float w[U], v[U][V];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      p[u] = j0 + u < a.k ? places[j0 + u] : -1;
      if (p[u] >= a.R) p[u] = -1;
      w[u] = weights && j0 + u < a.k ? weights[j0 + u] : 1.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p[u] >= 0) load_some<T, V>(rows + p[u] * a.rows_row, v[u]);
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p[u] >= 0)
#pragma unroll
        for (int e = 0; e < V; ++e) y[e] = fmaf(w[u], v[u][e], y[e]);
  }
  store_some<T, V>(static_cast<T*>(a.y) + token * a.D + c, y);
}

// NT threads for each slot: the row's gradient, and the weight's.  Slots of a token follow one another, so
// that its gradient comes from L1 after the first.  The same threads zero the row of their own number if no
// token has it.
template <typename T, int V, int NT>
__global__ void __launch_bounds__(256) combine_backward_kernel(const CombineGradArgs a) {
  launch_gate();
  const int64_t slots = a.T * a.k, per = slots > a.R ? slots : a.R;
  const int64_t at = (int64_t)blockIdx.x * (256 / NT) + threadIdx.x / NT, worker = blockIdx.y;
  const int t0 = threadIdx.x % NT;
  float dot = 0.f;
  bool has = false;
  if (at < per) {
    T* d_rows = static_cast<T*>(a.d_rows) + worker * a.R * a.D;
    if (at < a.R && a.tokens[worker * a.R + at] < 0) {
      float zero[V];
#pragma unroll
      for (int e = 0; e < V; ++e) zero[e] = 0.f;
      for (int64_t c = (int64_t)t0 * V; c < a.D; c += NT * V) store_some<T, V>(d_rows + at * a.D + c, zero);
    }
    has = at < slots;
    if (has) {
      const int32_t p = a.places[worker * slots + at];
      if (p >= 0 && p < a.R) {
        const float w = a.weights[worker * slots + at];
        const T* dy = static_cast<const T*>(a.d_y) + worker * a.dy_worker + at / a.k * a.dy_row;
        const T* row = static_cast<const T*>(a.rows) + worker * a.rows_worker + p * a.rows_row;
        T* out = d_rows + (int64_t)p * a.D;
        constexpr int U = V == 1 ? 8 : 4;
        for (int64_t c0 = (int64_t)t0 * V; c0 < a.D; c0 += NT * V * U) {
          float g[U][V], x[U][V];
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int64_t c = c0 + u * NT * V;
            if (c < a.D) {
              load_some<T, V>(dy + c, g[u]);
              load_some<T, V>(row + c, x[u]);
            }
          }
#pragma unroll
          for (int u = 0; u < U; ++u) {
            const int64_t c = c0 + u * NT * V;
            if (c < a.D) {
              float d[V];
#pragma unroll
              for (int e = 0; e < V; ++e) {
                dot = fmaf(g[u][e], x[u][e], dot);
                d[e] = w * g[u][e];
              }
              store_some<T, V>(out + c, d);
            }
          }
        }
      }
    }
  }
  dot = warp_sum(dot);
  if constexpr (NT > 32) {
    __shared__ float sums[8];
    if ((threadIdx.x & 31) == 0) sums[threadIdx.x >> 5] = dot;
    __syncthreads();
    if (threadIdx.x == 0) {
      dot = 0.f;
#pragma unroll
      for (int i = 0; i < NT / 32; ++i) dot += sums[i];
    }
  }
  if (t0 == 0 && has) a.d_weights[worker * slots + at] = dot;
}

// ---------------------------------------------------------------------------------- host

// Tokens of a warp: as few as the GPU has room for at once.
int route_per_warp(int64_t m, int64_t T) {
  const int64_t tiles = m < kSms ? kSms / m : 1;
  const int64_t n = (T + kRouteWarps * tiles - 1) / (kRouteWarps * tiles);
  return (int)(n < 1 ? 1 : n);
}
int64_t route_tiles(int64_t m, int64_t T) {
  const int64_t per = (int64_t)kRouteWarps * route_per_warp(m, T);
  return (T + per - 1) / per;
}

int lane_elements(int64_t E) {
  int nl = 1;
  while (nl * 32 < E) nl *= 2;
  return nl;
}
// Whether lanes may load (or store) their elements of every row at once.
bool lanes_aligned(const void* p, int64_t ld, int64_t E, int nl, int size) {
  const int bytes = nl * size < 16 ? nl * size : 16;
  return E % nl == 0 && (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(ld * size)) % bytes == 0;
}

template <typename T, int NL>
cudaError_t route_as(const RouteArgs& r, cudaStream_t s) {
  RouteKernelArgs a{r.logits, r.ld, (int)r.T, (int)r.E, r.k, route_per_warp(r.m, r.T), r.normalise,
                    lanes_aligned(r.logits, r.ld, r.E, NL, sizeof(T)), r.weights, r.ids, r.places, r.tokens, r.offsets,
                    static_cast<int32_t*>(r.ws)};
  const int64_t tiles = route_tiles(r.m, r.T);
  const size_t smem = (size_t)kRouteWarps * r.E * sizeof(int);
  static PerDeviceSmem configured[2];
  auto kern = tiles == 1 ? route_kernel<T, NL, true> : route_kernel<T, NL, false>;
  cudaError_t e = ensure_dynamic_smem(configured[tiles == 1], kern, (size_t)kRouteWarps * 32 * NL * sizeof(int));
  if (e != cudaSuccess) return e;
  const dim3 grid((unsigned)tiles, (unsigned)r.m);
  e = launch_chained(kern, grid, dim3(kRouteThreads), smem, s, a);
  if (e != cudaSuccess || tiles == 1) return e;
  return launch_chained(place_kernel, grid, dim3(kRouteThreads), 0, s, a);
}
template <typename T>
cudaError_t route_of(const RouteArgs& r, cudaStream_t s) {
  switch (lane_elements(r.E)) {
    case 1: return route_as<T, 1>(r, s);
    case 2: return route_as<T, 2>(r, s);
    case 4: return route_as<T, 4>(r, s);
    case 8: return route_as<T, 8>(r, s);
    case 16: return route_as<T, 16>(r, s);
    default: return route_as<T, 32>(r, s);
  }
}

template <typename T, int NL>
cudaError_t route_backward_as(const RouteGradArgs& a, cudaStream_t s) {
  return launch_chained(route_backward_kernel<T, NL>, dim3((unsigned)((a.rows + 7) / 8)), dim3(256), 0, s, a,
                        (int)lanes_aligned(a.logits, a.ld, a.E, NL, sizeof(T)), (int)lanes_aligned(a.d_logits, a.E, a.E, NL, sizeof(T)));
}
template <typename T>
cudaError_t route_backward_of(const RouteGradArgs& a, cudaStream_t s) {
  switch (lane_elements(a.E)) {
    case 1: return route_backward_as<T, 1>(a, s);
    case 2: return route_backward_as<T, 2>(a, s);
    case 4: return route_backward_as<T, 4>(a, s);
    case 8: return route_backward_as<T, 8>(a, s);
    case 16: return route_backward_as<T, 16>(a, s);
    default: return route_backward_as<T, 32>(a, s);
  }
}

bool whole_pieces(const void* p, int64_t worker, int64_t row, int size) {
  return (reinterpret_cast<uintptr_t>(p) | (uintptr_t)(worker * size) | (uintptr_t)(row * size)) % 16 == 0;
}

template <typename T>
cudaError_t combine_of(const CombineArgs& a, cudaStream_t s) {
  constexpr int V = Elem<T>::kVec;
  const bool vec = a.D % V == 0 && whole_pieces(a.rows, a.rows_worker, a.rows_row, sizeof(T)) && whole_pieces(a.y, 0, a.D, sizeof(T));
  const int64_t threads = a.m * a.T * (vec ? a.D / V : a.D);
  return launch_chained(vec ? combine_kernel<T, V> : combine_kernel<T, 1>, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a);
}

template <typename T, int V>
cudaError_t combine_backward_as(const CombineGradArgs& a, cudaStream_t s) {
  const int64_t slots = a.T * a.k, per = slots > a.R ? slots : a.R;
  // a CTA for a slot where its row is long enough to keep all threads busy
  const bool wide = a.D >= 256 * V * 2;
  const int64_t ctas = wide ? per : (per + 7) / 8;
  return launch_chained(wide ? combine_backward_kernel<T, V, 256> : combine_backward_kernel<T, V, 32>, dim3((unsigned)ctas, (unsigned)a.m),
                        dim3(256), 0, s, a);
}
template <typename T>
cudaError_t combine_backward_of(const CombineGradArgs& a, cudaStream_t s) {
  constexpr int V = Elem<T>::kVec;
  const bool vec = a.D % V == 0 && whole_pieces(a.rows, a.rows_worker, a.rows_row, sizeof(T)) &&
                   whole_pieces(a.d_y, a.dy_worker, a.dy_row, sizeof(T)) && whole_pieces(a.d_rows, 0, a.D, sizeof(T));
  return vec ? combine_backward_as<T, V>(a, s) : combine_backward_as<T, 1>(a, s);
}

}  // namespace

size_t route_workspace(int64_t m, int64_t T, int64_t E) {
  const int64_t tiles = route_tiles(m, T);
  return tiles == 1 ? 0 : (size_t)m * tiles * E * sizeof(int32_t);
}

cudaError_t launch_route(const RouteArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case OLSGD_F32: return route_of<float>(a, s);
    case OLSGD_BF16: return route_of<__nv_bfloat16>(a, s);
    default: return route_of<__half>(a, s);
  }
}
cudaError_t launch_route_backward(const RouteGradArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case OLSGD_F32: return route_backward_of<float>(a, s);
    case OLSGD_BF16: return route_backward_of<__nv_bfloat16>(a, s);
    default: return route_backward_of<__half>(a, s);
  }
}
cudaError_t launch_combine(const CombineArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case OLSGD_F32: return combine_of<float>(a, s);
    case OLSGD_BF16: return combine_of<__nv_bfloat16>(a, s);
    default: return combine_of<__half>(a, s);
  }
}
cudaError_t launch_combine_backward(const CombineGradArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case OLSGD_F32: return combine_backward_of<float>(a, s);
    case OLSGD_BF16: return combine_backward_of<__nv_bfloat16>(a, s);
    default: return combine_backward_of<__half>(a, s);
  }
}

}  // namespace olsgd
