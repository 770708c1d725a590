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
// Bound by the instructions of the selection (8 of 128, 2 x 16384 tokens, fp32: 20 us and 7 for the placing, 25 MB); a few
// tokens by their one CTA's way through its barriers (8 tokens: 6 us).  Gradient: 11 us for 37 MB.
//
// Combine: y_t = sum_j w_tj rows[place_tj], in order of j in fp32; its gradient is a product and a dot
// product for each slot.  Both are bound by reading (and writing) each row once (16384 tokens x 2 x 1024 bf16: 19 us for
// 101 MB, 5.2 TB/s, and 25 for 168 MB, part of them still in L2); rows of any alignment by the instructions that shift them
// (16 x 333 x 3 x 1021 fp16: 21 us for 43 MB, 27 for 76).
#include "operator_common.cuh"
#include "operators_internal.h"

namespace olsgd {
namespace {

using namespace op;

constexpr int kSms = 148;
constexpr int kRouteWarps = 32;
constexpr int kRouteThreads = 32 * kRouteWarps;
constexpr int kKeptSlots = 64 * 1024;
constexpr int kSorted = 4;   // elements of a lane that are sorted ahead of the rounds
static_assert(OLSGD_MAX_EXPERTS <= kRouteThreads, "a thread for each expert");
static_assert(OLSGD_MAX_TOP <= 32, "a lane for each slot of a token");
static_assert(OLSGD_MAX_EXPERTS <= 1024, "ten bits");

// Values that order as the logits do: 0 for -inf (never chosen), NaN above all.  (Adding 0 makes -0 +0, and any NaN the one
// with sign 0.)
constexpr uint32_t kLowest = 0x007FFFFFu;   // of -inf before it is moved to 0
__device__ __forceinline__ uint32_t key_of(float v) {
  const uint32_t u = __float_as_uint(v + 0.f);
  return (u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u)) - kLowest;
}
__device__ __forceinline__ float value_of(uint32_t key) {
  const uint32_t o = key + kLowest;
  return __uint_as_float((o >> 31) ? (o ^ 0x80000000u) : ~o);
}
// e^d by the hardware's power of two: off by 2 steps and the rounding of d log2 e.
__device__ __forceinline__ float power(float d) { return ex2(d * kLog2e); }

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
  int keep;                  // whether a CTA's slots have room in shared memory
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
  extern __shared__ int count[];   // [kRouteWarps][E]; then (keep) the slots' experts and ranks, [kRouteWarps][per_warp][k]
  __shared__ int warp_sums[32];
  __shared__ int2 picked[kRouteWarps][32];   // expert and key of a token's slots (NL <= kSorted)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = a.E, k = a.k;
  const int64_t worker = blockIdx.y;
  int* mine = count + warp * E;
  uint32_t* slots = reinterpret_cast<uint32_t*>(count + kRouteWarps * E) + (int64_t)warp * a.per_warp * k;
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
    if constexpr (NL <= kSorted) {
      // Each lane's keys in falling order (equal ones stay as they are), so that what a round takes is a head.
      int at[NL], found = 0;
      uint32_t own[NL];
#pragma unroll
      for (int i = 0; i < NL; ++i) {
        own[i] = key[i];
        at[i] = lane * NL + i;
      }
#pragma unroll
      for (int pass = NL - 1; pass > 0; --pass)
#pragma unroll
        for (int i = 0; i < pass; ++i) {
          const bool swap = own[i + 1] > own[i];
          const uint32_t big = swap ? own[i + 1] : own[i], small = swap ? own[i] : own[i + 1];
          const int big_at = swap ? at[i + 1] : at[i], small_at = swap ? at[i] : at[i + 1];
          own[i] = big;
          own[i + 1] = small;
          at[i] = big_at;
          at[i + 1] = small_at;
        }
      for (int j = 0; j < k; ++j) {
        const uint32_t most = __reduce_max_sync(0xffffffffu, own[0]);
        if (most == 0) break;
        if (j == 0) top = most;
        const uint32_t equal = __ballot_sync(0xffffffffu, own[0] == most);
        if ((equal & (0u - equal)) == 1u << lane) {   // the lowest of the lanes that have it: its head leaves
          picked[warp][j] = make_int2(at[0], (int)most);
#pragma unroll
          for (int i = 0; i + 1 < NL; ++i) {
            own[i] = own[i + 1];
            at[i] = at[i + 1];
          }
          own[NL - 1] = 0;
        }
        found = j + 1;
      }
      __syncwarp();
      if (lane < found) {
        const int2 p = picked[warp][lane];
        id = p.x;
        chosen = (uint32_t)p.y;
      }
      __syncwarp();
    } else {
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
    }
    const float base = value_of(top);
    float e = id >= 0 ? power(value_of(chosen) - base) : 0.f, total = e;
    if (!a.normalise) {
      // all of them (NL > kSorted: those chosen have left, and count already)
      if (NL <= kSorted) total = 0.f;
#pragma unroll
      for (int i = 0; i < NL; ++i) total += key[i] ? power(value_of(key[i]) - base) : 0.f;
    }
    total = warp_sum(total);
    if (lane < k) {
      const int64_t slot = (worker * a.T + t) * k + lane;
      a.ids[slot] = id;
      a.weights[slot] = id >= 0 ? e / total : 0.f;
      // its rank among the warp's slots of this expert
      const int rank = id >= 0 ? mine[id]++ : -1;
      if (a.keep) slots[(t - first) * k + lane] = id >= 0 ? (uint32_t)rank << 10 | (uint32_t)id : ~0u;
      else a.places[slot] = rank;
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
  // (each lane reads what it has written; not kept: in global memory)
  for (int64_t t = first; t < last; ++t) {
    const int64_t slot = (worker * a.T + t) * k + lane;
    if (lane < k) {
      int id, rank;
      if (a.keep) {
        const uint32_t s = slots[(t - first) * k + lane];
        id = s == ~0u ? -1 : (int)(s & 1023u);
        rank = (int)(s >> 10);
      } else {
        id = a.ids[slot];
        rank = a.places[slot];
      }
      const int place = id >= 0 ? rank + mine[id] : -1;
      a.places[slot] = place;
      if (ONE && id >= 0) a.tokens[worker * a.T * k + place] = (int32_t)t;
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
  const int64_t slots = (int64_t)a.T * a.k, per_tile = (int64_t)kRouteWarps * a.per_warp * a.k;
  const int64_t first = blockIdx.x * per_tile + threadIdx.x, end = min(slots, (blockIdx.x + 1) * per_tile);
  int32_t *places = a.places + worker * slots, *tokens = a.tokens + worker * slots;
  const int32_t* ids = a.ids + worker * slots;
  // the first slots are on their way while the counts are added up
  constexpr int kAhead = 2;
  int ids_ahead[kAhead], ranks_ahead[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) {
    const int64_t s = first + u * kRouteThreads;
    ids_ahead[u] = s < end ? ids[s] : -1;
    ranks_ahead[u] = s < end ? places[s] : 0;
  }
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
  const auto put = [&](int64_t s, int id, int rank) {
    if (id < 0) return;
    const int place = rank + befores[id];
    places[s] = place;
    tokens[place] = (int32_t)((uint32_t)s / (uint32_t)a.k);
  };
#pragma unroll
  for (int u = 0; u < kAhead; ++u) put(first + u * kRouteThreads, ids_ahead[u], ranks_ahead[u]);
  for (int64_t s = first + kAhead * kRouteThreads; s < end; s += kRouteThreads) put(s, ids[s], places[s]);
  for (int64_t r = all + (int64_t)blockIdx.x * kRouteThreads + threadIdx.x; r < slots; r += (int64_t)tiles * kRouteThreads) tokens[r] = -1;
}

// The gradient of a token's logits, by a warp: what is asked at the chosen goes through shared memory to the lanes
// that hold them.
template <typename T, int NL>
__global__ void __launch_bounds__(256) route_backward_kernel(const RouteGradArgs a, int vec_in, int vec_out) {
  extern __shared__ float asked[];   // [8][32 NL]
  launch_gate();
  const int lane = threadIdx.x & 31, k = a.k, E = a.E;
  const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  if (r >= a.rows) return;
  float* mine = asked + (threadIdx.x >> 5) * 32 * NL;
  float x[NL];
  if (!a.normalise) load_lane<T, NL>(static_cast<const T*>(a.logits) + r * a.ld, E, vec_in, -INFINITY, x);
  int id = -1;
  float w = 0.f, dw = 0.f;
  if (lane < k) {
    id = a.ids[r * k + lane];
    w = a.weights[r * k + lane];
    dw = a.d_weights[r * k + lane];
  }
#pragma unroll
  for (int i = 0; i < NL; ++i) mine[i * 32 + lane] = 0.f;
  if (id < 0 || id >= E) {   // no expert: whatever its gradient holds
    id = -1;
    w = dw = 0.f;
  }
  const float mean = warp_sum(w * dw);
  __syncwarp();
  if (id >= 0) atomicAdd(mine + id, a.normalise ? w * (dw - mean) : dw);   // (a token's experts differ)
  __syncwarp();
  float d[NL];
#pragma unroll
  for (int i = 0; i < NL; ++i) d[i] = mine[lane * NL + i];
  if (!a.normalise) {
    float most = -INFINITY, total = 0.f;
#pragma unroll
    for (int i = 0; i < NL; ++i) most = fmaxf(most, x[i]);
#pragma unroll
    for (int off = 16; off; off >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, off));
    // nothing was chosen: nothing is asked of this row (padding: all -inf)
    const bool empty = __ballot_sync(0xffffffffu, id >= 0) == 0;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      x[i] = empty ? 0.f : power(x[i] - most);
      total += x[i];
    }
    const float share = empty ? 0.f : 1.f / warp_sum(total);
#pragma unroll
    for (int i = 0; i < NL; ++i) d[i] = x[i] * share * (d[i] - mean);
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

// 16 bytes of a row from element j on.  SHIFTED: rows start anywhere.
template <typename T, bool SHIFTED>
__device__ __forceinline__ uint4 load_sixteen(const T* row, int64_t j, int64_t n, const T* begin, const T* end) {
  if (SHIFTED) return load_shifted<T>(row, j, n, begin, end);
  return ld16_stream(row + j);
}
// Pieces of a result's row, counted from the boundary at or before it.
template <typename T>
int64_t row_pieces(int64_t D, bool shifted) {
  constexpr int V = Elem<T>::kVec;
  return shifted ? (D + 2 * V - 2) / V : D / V;
}

// Thread: 16 bytes of each of a token's row's P parts.  U: rows on their way at a time.
template <typename T, bool SHIFTED, int U, int P>
__global__ void __launch_bounds__(256, U > 2 && P > 1 ? 3 : SHIFTED || U > 2 || P > 1 ? 4 : 6) combine_kernel(const CombineArgs a, int64_t pieces, bool narrow) {
  constexpr int V = Elem<T>::kVec;
  launch_gate();
  const int64_t at = (int64_t)blockIdx.x * 256 + threadIdx.x, share = pieces / P;
  // (narrow: the launch's threads fit 32 bits; a division of 64 takes a hundred instructions)
  const int64_t token = narrow ? (uint32_t)at / (uint32_t)share : at / share;
  if (token >= a.m * a.T) return;
  T* y = static_cast<T*>(a.y) + token * a.D;
  const int64_t j = (at - token * share) * V - (SHIFTED ? row_shift(y) : 0), part = share * V;
  if (SHIFTED && j >= a.D) return;
  const int64_t worker = narrow ? (uint32_t)token / (uint32_t)a.T : token / a.T;
  const T* rows = static_cast<const T*>(a.rows) + worker * a.rows_worker;
  const T *begin = static_cast<const T*>(a.rows), *end = static_cast<const T*>(a.rows_end);
  const int32_t* places = a.places + token * a.k;
  const float* weights = a.weights ? a.weights + token * a.k : nullptr;
  float sum[P][V];
#pragma unroll
  for (int q = 0; q < P; ++q)
#pragma unroll
    for (int e = 0; e < V; ++e) sum[q][e] = 0.f;
  for (int s0 = 0; s0 < a.k; s0 += U) {
    int32_t p[U];
    float w[U];
    uint4 raw[U][P];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      p[u] = s0 + u < a.k ? places[s0 + u] : -1;
      w[u] = weights && s0 + u < a.k ? weights[s0 + u] : 1.f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p[u] >= 0 && p[u] < a.R) {
#pragma unroll
        for (int q = 0; q < P; ++q) raw[u][q] = load_sixteen<T, SHIFTED>(rows + p[u] * a.rows_row, j + q * part, a.D, begin, end);
      }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (p[u] >= 0 && p[u] < a.R) {
#pragma unroll
        for (int q = 0; q < P; ++q) {
          float v[V];
          Elem<T>::unpack(raw[u][q], v);
#pragma unroll
          for (int e = 0; e < V; ++e) sum[q][e] = fmaf(w[u], v[e], sum[q][e]);
        }
      }
  }
#pragma unroll
  for (int q = 0; q < P; ++q) store_floats<T, V>(y, j + q * part, a.D, true, sum[q]);
}

// NT threads for each slot: the row's gradient, and the weight's.  Slots of a token follow one another, so
// that its gradient comes from L1 after the first.  The same threads zero the row of their own number if no
// token has it.
template <typename T, bool SHIFTED, int NT>
__global__ void __launch_bounds__(256, 4) combine_backward_kernel(const CombineGradArgs a, int pieces) {
  constexpr int V = Elem<T>::kVec, U = SHIFTED ? 2 : 4;
  launch_gate();
  const int64_t slots = a.T * a.k;
  const int64_t at = (int64_t)blockIdx.x * (256 / NT) + threadIdx.x / NT, worker = blockIdx.y;
  const int t0 = threadIdx.x % NT;
  float dot = 0.f;
  const bool has = at < slots;
  T* d_rows = static_cast<T*>(a.d_rows) + worker * a.R * a.D;
  const bool zero = at < a.R && a.tokens[worker * a.R + at] < 0;
  const int32_t p = has ? a.places[worker * slots + at] : -1;
  const float w = has ? a.weights[worker * slots + at] : 0.f;
  if (zero) {
    T* out = d_rows + at * a.D;
    const int shift = SHIFTED ? row_shift(out) : 0;
    float none[V];
#pragma unroll
    for (int e = 0; e < V; ++e) none[e] = 0.f;
    for (int q = t0; q < pieces; q += NT) store_floats<T, V>(out, (int64_t)q * V - shift, a.D, true, none);
  }
  if (p >= 0 && p < a.R) {
    const T *dy_all = static_cast<const T*>(a.d_y), *rows_all = static_cast<const T*>(a.rows);
    const T* dy = dy_all + worker * a.dy_worker + (int64_t)((uint32_t)at / (uint32_t)a.k) * a.dy_row;
    const T* row = rows_all + worker * a.rows_worker + p * a.rows_row;
    T* out = d_rows + (int64_t)p * a.D;
    const int shift = SHIFTED ? row_shift(out) : 0;
    // (not SHIFTED: unused)
    const ShiftedRow<T> dy_at(dy, -shift, a.D, pieces, dy_all, static_cast<const T*>(a.dy_end));
    const ShiftedRow<T> row_at(row, -shift, a.D, pieces, rows_all, static_cast<const T*>(a.rows_end));
    f32x2 sum = 0;
    const f32x2 w2 = pack2f(w, w);
    for (int q0 = t0; q0 < pieces; q0 += NT * U) {
      uint4 g[U], x[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t j = (int64_t)(q0 + u * NT) * V - shift;
        const bool live = q0 + u * NT < pieces && j < a.D;
        g[u] = x[u] = make_uint4(0, 0, 0, 0);
        if (live) {
          // (the token's gradient is read again by its other slots)
          g[u] = SHIFTED ? dy_at.load(q0 + u * NT) : ld16(dy + j);
          x[u] = SHIFTED ? row_at.load(q0 + u * NT) : ld16_stream(row + j);
        }
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t j = (int64_t)(q0 + u * NT) * V - shift;
        if (q0 + u * NT >= pieces || j >= a.D) continue;
        float d[V];
        if (!SHIFTED || (j >= 0 && j + V <= a.D)) {
#pragma unroll
          for (int i = 0; i < V / 2; ++i) {
            const f32x2 gi = raw_pair<T>(g[u], i);
            sum = fma2(gi, raw_pair<T>(x[u], i), sum);
            unpack2f(mul2(w2, gi), d[2 * i], d[2 * i + 1]);
          }
        } else {   // an end of the row
          float gf[V], xf[V];
          Elem<T>::unpack(g[u], gf);
          Elem<T>::unpack(x[u], xf);
#pragma unroll
          for (int e = 0; e < V; ++e) {
            if (j + e >= 0 && j + e < a.D) dot = fmaf(gf[e], xf[e], dot);
            d[e] = w * gf[e];
          }
        }
        store_floats<T, V>(out, j, a.D, true, d);
      }
    }
    float lo, hi;
    unpack2f(sum, lo, hi);
    dot += lo + hi;
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
  const int per_warp = route_per_warp(r.m, r.T);
  const int64_t tiles = route_tiles(r.m, r.T), slots = (int64_t)kRouteWarps * per_warp * r.k * sizeof(int);
  const bool keep = slots <= kKeptSlots;
  RouteKernelArgs a{r.logits, r.ld, (int)r.T, (int)r.E, r.k, per_warp, r.normalise,
                    lanes_aligned(r.logits, r.ld, r.E, NL, sizeof(T)), keep, r.weights, r.ids, r.places, r.tokens, r.offsets,
                    static_cast<int32_t*>(r.ws)};
  const size_t smem = (size_t)kRouteWarps * r.E * sizeof(int) + (keep ? slots : 0);
  static PerDeviceSmem configured[2];
  auto kern = tiles == 1 ? route_kernel<T, NL, true> : route_kernel<T, NL, false>;
  cudaError_t e = ensure_dynamic_smem(configured[tiles == 1], kern, (size_t)kRouteWarps * 32 * NL * sizeof(int) + kKeptSlots);
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
  return launch_chained(route_backward_kernel<T, NL>, dim3((unsigned)((a.rows + 7) / 8)), dim3(256), 8 * 32 * NL * sizeof(float), s, a,
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

// One past the last element of [m][rows][cols].
template <typename T>
const void* tensor_end(const void* p, int64_t m, int64_t worker, int64_t rows, int64_t row, int64_t cols) {
  if (!p || rows == 0) return p;
  return static_cast<const T*>(p) + (m > 1 ? (m - 1) * worker : 0) + (rows - 1) * row + cols;
}

template <typename T, bool SHIFTED>
cudaError_t combine_as(const CombineArgs& a, cudaStream_t s) {
  const int64_t pieces = row_pieces<T>(a.D, SHIFTED);
  // More pieces a thread, hence more bytes on their way, where enough threads remain: two, or four where a token has one row.  us with
  // one and with these: bf16, 16384 tokens x 2 x 1024: 18 and 17, 8192 x 4 x 1024: 16 and 14; fp32, 2 x 8192 x 4 x 512: 37 and 27,
  // 8192 x 6 x 1024: 49 and 39.  (Of rows of any alignment, 16 x 333 x 3 x 1021: 15.5 and 18.)
  const int64_t all = a.m * a.T * pieces;
  const int share = SHIFTED || all < kSms * 4096 ? 1 : a.k == 1 && pieces % 4 == 0 ? 4 : pieces % 2 == 0 ? 2 : 1;
  const int64_t threads = all / share;
  auto k = a.k == 1 ? combine_kernel<T, SHIFTED, 1, 1> : a.k == 2 ? combine_kernel<T, SHIFTED, 2, 1> : combine_kernel<T, SHIFTED, 4, 1>;
  if constexpr (!SHIFTED) {
    if (share == 4) k = combine_kernel<T, false, 1, 4>;
    if (share == 2) k = a.k == 1 ? combine_kernel<T, false, 1, 2> : a.k == 2 ? combine_kernel<T, false, 2, 2> : combine_kernel<T, false, 4, 2>;
  }
  return launch_chained(k, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, s, a, pieces, threads <= 0xffffffffll);
}
template <typename T>
cudaError_t combine_of(CombineArgs a, cudaStream_t s) {
  const bool whole = a.D % Elem<T>::kVec == 0 && whole_pieces(a.rows, a.rows_worker, a.rows_row, sizeof(T)) && whole_pieces(a.y, 0, a.D, sizeof(T));
  a.rows_end = tensor_end<T>(a.rows, a.m, a.rows_worker, a.R, a.rows_row, a.D);
  return whole ? combine_as<T, false>(a, s) : combine_as<T, true>(a, s);
}

template <typename T, bool SHIFTED>
cudaError_t combine_backward_as(const CombineGradArgs& a, cudaStream_t s) {
  const int64_t slots = a.T * a.k, per = slots > a.R ? slots : a.R, pieces = row_pieces<T>(a.D, SHIFTED);
  // a CTA for a slot where its row is long enough to keep all threads busy
  const bool wide = pieces >= 512;
  const int64_t ctas = wide ? per : (per + 7) / 8;
  return launch_chained(wide ? combine_backward_kernel<T, SHIFTED, 256> : combine_backward_kernel<T, SHIFTED, 32>,
                        dim3((unsigned)ctas, (unsigned)a.m), dim3(256), 0, s, a, (int)pieces);
}
template <typename T>
cudaError_t combine_backward_of(CombineGradArgs a, cudaStream_t s) {
  const bool whole = a.D % Elem<T>::kVec == 0 && whole_pieces(a.rows, a.rows_worker, a.rows_row, sizeof(T)) &&
                     whole_pieces(a.d_y, a.dy_worker, a.dy_row, sizeof(T)) && whole_pieces(a.d_rows, 0, a.D, sizeof(T));
  a.rows_end = tensor_end<T>(a.rows, a.m, a.rows_worker, a.R, a.rows_row, a.D);
  a.dy_end = tensor_end<T>(a.d_y, a.m, a.dy_worker, a.T, a.dy_row, a.D);
  return whole ? combine_backward_as<T, false>(a, s) : combine_backward_as<T, true>(a, s);
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
