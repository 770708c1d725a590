// Log probabilities of given tokens, entropy, the most likely alternatives, and the gradient.
//
// For a row x of V logits, m = max x, S = sum exp(x - m):
//   log p_j = (x_j - m) - log S,   H = log S - (1/S) sum exp(x_j - m) (x_j - m).
// One pass keeps a running maximum and, relative to it, s = sum e^d and t = sum e^d d
// (d = x - m): when the maximum rises from m to m', both are carried over by s' = s f,
// t' = (t + s delta) f with delta = m - m', f = e^delta.  The difference x - m is formed before it
// is scaled, so rows of the type's lowest value, or far from zero, keep their probabilities.
// All of it is held in fp32.
//
// Alternatives: a warp reads 256 consecutive logits (a chunk) at a time and needs the chunk's
// maximum for the running maximum anyway, so it also stores it.  The k largest elements (ties to
// the lowest index) lie in the k chunks that come first by (maximum, lowest index): if an
// element's chunk is not among them, each of those k chunks holds an element that comes before
// it.  So k chunks, and few more, are read again and nothing else (find_top).
//
// Rows of up to 1024 logits stay in a warp's registers (one launch, no second read).  Longer
// ones are bound by reading the logits once; a row is split over several CTAs when there are
// fewer rows than the GPU has room for, and the parts are joined by a finishing kernel.
#include "operator_common.cuh"
#include "operators_internal.h"

namespace olsgd {
namespace {

using namespace op;

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;
constexpr int kUnroll = 4;            // chunks, or pieces of the gradient, in flight
constexpr int kChunkElems = 256;      // eight elements per lane: one 16-byte piece, or two of fp32
constexpr int kWarpRowMax = 1024;     // longest row that stays in a warp's registers
constexpr int kWarpList = 160;        // candidates that a warp lists
constexpr int kMaxTop = OLSGD_MAX_TOP;
static_assert(kMaxTop <= 32, "a lane for each chunk of a row that has no more than k");
constexpr int kMaxSplit = 64;
// Unsplit rows that are this short, or whose alternatives are wanted, get CTAs of half the threads:
// twice as many rows are on their way while others begin and end (3684 x 10549 bf16: 18.7 us against
// 26.5, with five alternatives 34 against 46; 4096 x 32768 without: 3 % slower, hence the bound).
constexpr int kNarrowRow = 16384;
// The last rows that the forward kernel reads (this many bytes of them) are loaded at normal priority
// and stay in L2; the gradient, which usually follows, starts from them.
constexpr int64_t kKeepBytes = 64LL << 20;

struct RowState {
  float m, s, t;   // running maximum; sums relative to it
};

// Differences are clamped here: e^d is zero long before, and 0 * -inf stays out of t.
constexpr float kFarBelow = -1.0e9f;

// e^(x - m) and its product with the exponent; a NaN reaches both sums.
__device__ __forceinline__ void accumulate(float x, float base, float& s, float& t) {
  const float d = max_nan(x - base, kFarBelow);
  const float e = ex2(d * kLog2e);
  s += e;
  t = fmaf(e, d, t);
}
// The same for two elements at a time.
__device__ __forceinline__ void accumulate2(f32x2 x, f32x2 minus_base, f32x2& s, f32x2& t) {
  float lo, hi;
  unpack2f(add2(x, minus_base), lo, hi);
  lo = max_nan(lo, kFarBelow);
  hi = max_nan(hi, kFarBelow);
  const f32x2 d = pack2f(lo, hi);
  unpack2f(mul2(d, pack2f(kLog2e, kLog2e)), lo, hi);
  const f32x2 e = pack2f(ex2(lo), ex2(hi));
  s = add2(s, e);
  t = fma2(e, d, t);
}

// Carries (s, t) from maximum `from` to the larger maximum `to`.
__device__ __forceinline__ void rebase(float from, float to, float& s, float& t) {
  if (from == -INFINITY) return;   // nothing but zeros (or a NaN) so far
  const float delta = fmaxf(from - to, kFarBelow);
  const float f = ex2(delta * kLog2e);
  t = fmaf(s, delta, t) * f;
  s *= f;
}
__device__ __forceinline__ void rebase2(float from, float to, f32x2& s, f32x2& t) {
  if (from == -INFINITY) return;
  const float delta = fmaxf(from - to, kFarBelow);
  const float f = ex2(delta * kLog2e);
  t = mul2(fma2(s, pack2f(delta, delta), t), pack2f(f, f));
  s = mul2(s, pack2f(f, f));
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

// The target's logit, fetched ahead of the sums: two dependent loads that nothing waits for then.
struct Target {
  float x;
  bool has;
};
template <typename T>
__device__ __forceinline__ Target fetch_target(const RowOut& o, const T* row, int64_t r, int64_t V) {
  const int32_t t = o.targets[r];
  Target g;
  g.has = t >= 0 && t < V;   // a target outside [0, V) marks a row without a token
  g.x = g.has ? Elem<T>::to_float(row[t]) : 0.f;
  return g;
}
__device__ __forceinline__ void write_row(const RowOut& o, const Target& g, int64_t r, const RowState& v) {
  const float log_s = log_sum(v);
  const bool empty = v.m == -INFINITY && v.s == 0.f;
  float h = empty ? 0.f : log_s - v.t / v.s;
  if (h < 0.f) h = 0.f;   // rounding of a row that is certain; a NaN stays
  o.entropy[r] = h;
  o.stats[2 * r] = v.m;
  o.stats[2 * r + 1] = log_s;
  o.logp[r] = g.has ? log_prob(g.x, v, log_s) : 0.f;
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
  const Target target = fetch_target<T>(o, row, r, V);
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
  if (lane == 0) write_row(o, target, r, st);
  if (top > 0) {
    // As for long rows (find_top): the k-th best of the groups' maxima is a floor; what reaches it is
    // listed, and takes its place by counting.  Should the list overflow: rounds of a maximum.
    __shared__ uint64_t lists[kWarps][kWarpList];
    uint64_t* list = lists[threadIdx.x >> 5];
    const float log_s = log_sum(st);
    const auto put = [&](int q, uint64_t key) {
      top_ids[r * top + q] = index_of(key);
      top_logp[r * top + q] = log_prob(value_of((uint32_t)(key >> 32)), st, log_s);
    };
    uint32_t ord[NL];   // of an element past the row: 0, below every other
#pragma unroll
    for (int i = 0; i < NL; ++i) ord[i] = i * 32 + lane < V ? order_of(v[i]) : 0u;
    const auto key_at = [&](int i) { return ord[i] ? key_of(ord[i], i * 32 + lane) : 0ull; };
    if (NL == 1) {
      const uint64_t mine = key_at(0);
      int larger = 0;
#pragma unroll
      for (int i = 0; i < 32; ++i) larger += __shfl_sync(0xffffffffu, mine, i) > mine;
      if (mine && larger < top) put(larger, mine);
      return;
    }
    // 64 groups: the halves of the lanes' elements (the lower index comes first among equals)
    uint64_t best[2];
    int larger[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      uint32_t o = 0;
      int at = 0;
#pragma unroll
      for (int i = h * (NL / 2); i < (h + 1) * (NL / 2); ++i) {
        if (ord[i] > o) {
          o = ord[i];
          at = i;
        }
      }
      best[h] = o ? key_of(o, at * 32 + lane) : 0ull;
    }
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const uint64_t a = __shfl_sync(0xffffffffu, best[0], i), b = __shfl_sync(0xffffffffu, best[1], i);
#pragma unroll
      for (int h = 0; h < 2; ++h) larger[h] += (a > best[h]) + (b > best[h]);
    }
    uint64_t floor_key = 1;   // fewer groups than k: all are candidates
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const uint32_t here = __ballot_sync(0xffffffffu, best[h] && larger[h] == top - 1);
      if (here) floor_key = __shfl_sync(0xffffffffu, best[h], __ffs(here) - 1);
    }
    const uint32_t floor_order = (uint32_t)(floor_key >> 32);
    const int floor_at = floor_key == 1 ? V : index_of(floor_key);
    int n = 0;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const bool reaches = ord[i] > floor_order || (ord[i] == floor_order && ord[i] && i * 32 + lane <= floor_at);
      const uint32_t in = __ballot_sync(0xffffffffu, reaches);
      const int at = n + __popc(in & ((1u << lane) - 1));
      if (reaches && at < kWarpList) list[at] = key_of(ord[i], i * 32 + lane);
      n += __popc(in);
    }
    __syncwarp();
    if (n <= kWarpList) {
      for (int i = lane; i < n; i += 32) {
        const uint64_t mine = list[i];
        int above = 0;
#pragma unroll 4
        for (int q = 0; q < n; ++q) above += list[q] > mine;
        if (above < top) put(above, mine);
      }
    } else {
      warp_select(
          top, 0,
          [&](uint64_t limit) {
            uint64_t b = 0;
#pragma unroll
            for (int i = 0; i < NL; ++i) {
              const uint64_t key = key_at(i);
              if (key < limit && key > b) b = key;
            }
            return b;
          },
          put);
    }
  }
}

// -------------------------------------------------------------------------- long rows
template <typename T>
__host__ __device__ constexpr uint32_t minus_inf() {
  return sizeof(T) == 4 ? 0xFF800000u : std::is_same<T, __half>::value ? 0xFC00u : 0xFF80u;
}

// Finds a row's alternatives; by a whole CTA.
//
// The chunks' maxima are dealt to 64 groups.  The k-th best of the groups' maxima is a floor: k
// chunks, so k elements, reach it, and what is below it is dropped.  Little more than k chunks are
// left; their elements that reach the floor, little more than k again, go to a list, and each counts
// how many are larger: its place in the order.  Rows of no more chunks than alternatives deal out their
// elements instead.  Should the list overflow all the same (a chunk full of larger elements than
// others have), each of the k best chunks gives its k best elements in k rounds of a maximum.
constexpr int kList = 1024;
constexpr int kGroups = 64;
static_assert(kGroups > kMaxTop, "k groups have a chunk where there are more chunks than k");
static_assert(kMaxTop * kMaxTop <= kList, "k of each of k chunks");
struct TopShared {
  uint64_t group_best[kGroups];
  uint64_t list[kList];
  int32_t chunk[kList];
  uint64_t floor_key;
  int n_chunks, n_list;
};

template <typename T, int NT>
__device__ __forceinline__ void find_top(TopShared& sh, const T* row, int64_t r, int V, int nchunks, float* cm, const RowState& st,
                                         int top, float* top_logp, int32_t* top_ids) {
  constexpr int VEC = Elem<T>::kVec;
  constexpr int Q = kChunkElems / 32 / VEC;
  constexpr int kWarps = NT / 32, kGroupThreads = NT / kGroups;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int shift = row_shift(row);
  if (st.s != st.s) {
    // a NaN (or +inf) in the row: the maxima passed over it, and are formed again
    for (int c = warp; c < nchunks; c += kWarps) {
      float v = raw_max<T, true>(load_raw<T>(row, c * kChunkElems + lane * VEC - shift, V, minus_inf<T>()));
      if (Q == 2) v = max_nan(v, raw_max<T, true>(load_raw<T>(row, c * kChunkElems + (32 + lane) * VEC - shift, V, minus_inf<T>())));
      const uint32_t order = __reduce_max_sync(0xffffffffu, order_of(v));
      if (lane == 0) cm[c] = value_of(order);
    }
    __syncthreads();
  }
  const bool few = nchunks <= top;
  const int n_dealt = few ? V : nchunks;
  const auto dealt_key = [&](int c) { return key_of(order_of(few ? Elem<T>::to_float(row[c]) : cm[c]), c); };

  // the floor
  uint64_t best = 0;
#pragma unroll 4
  for (int c = threadIdx.x / kGroupThreads + kGroups * (threadIdx.x % kGroupThreads); c < n_dealt; c += NT) {
    const uint64_t key = dealt_key(c);
    best = key > best ? key : best;
  }
#pragma unroll
  for (int off = 1; off < kGroupThreads; off <<= 1) {
    const uint64_t other = __shfl_xor_sync(0xffffffffu, best, off);
    best = other > best ? other : best;
  }
  if (threadIdx.x % kGroupThreads == 0) sh.group_best[threadIdx.x / kGroupThreads] = best;
  if (threadIdx.x == 0) sh.n_chunks = sh.n_list = 0;
  __syncthreads();
  if (threadIdx.x < kGroups) {
    const uint64_t mine = sh.group_best[threadIdx.x];
    int larger = 0;
#pragma unroll 16
    for (int i = 0; i < kGroups; ++i) larger += sh.group_best[i] > mine;
    if (larger == top - 1) sh.floor_key = mine;   // (keys differ: one group is the k-th best)
  }
  __syncthreads();
  const uint64_t floor_key = sh.floor_key;
  const uint64_t elem_floor = few ? floor_key : floor_key & 0xFFFFFFFF00000000ull;   // at a chunk's floor any index will do
  const auto list_element = [&](uint64_t key) {
    const int at = atomicAdd(&sh.n_list, 1);
    if (at < kList) sh.list[at] = key;
  };

  // what reaches it
  for (int c = threadIdx.x; c < n_dealt; c += NT) {
    const uint64_t key = dealt_key(c);
    if (key >= floor_key) {
      if (few) {
        list_element(key);
      } else {
        const int at = atomicAdd(&sh.n_chunks, 1);
        if (at < kList) sh.chunk[at] = c;
      }
    }
  }
  __syncthreads();
  int nc = few ? 0 : sh.n_chunks;
  const bool many_chunks = nc > kList;
  const uint32_t floor_order = (uint32_t)(elem_floor >> 32);
  for (int i = warp; i < (many_chunks ? 0 : nc); i += kWarps) {
    const int j0 = sh.chunk[i] * kChunkElems + lane * VEC - shift;
    uint32_t ord[Q][VEC];   // past the row: 0
    int equal = 0;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      const uint4 w = load_raw<T>(row, j0 + q * 32 * VEC, V, minus_inf<T>());
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const int j = j0 + q * 32 * VEC + e;
        float v, other;
        unpack2f(raw_pair<T>(w, e / 2), v, other);
        ord[q][e] = j >= 0 && j < V ? order_of(e % 2 ? other : v) : 0u;
        equal += ord[q][e] == floor_order;
      }
    }
    // of the elements that tie with the floor, the first k of the chunk will do
    const bool tied = __reduce_add_sync(0xffffffffu, equal) > top;
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      int before = 0;   // in this half of the chunk (Q == 2: k of each half)
      if (tied) {
        int mine = 0;
#pragma unroll
        for (int e = 0; e < VEC; ++e) mine += ord[q][e] == floor_order;
        int scan = mine;
#pragma unroll
        for (int off = 1; off < 32; off <<= 1) {
          const int up = __shfl_up_sync(0xffffffffu, scan, off);
          if (lane >= off) scan += up;
        }
        before = scan - mine;
      }
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const bool ties = ord[q][e] == floor_order;
        if (ord[q][e] > floor_order || (ties && (!tied || before < top))) list_element(key_of(ord[q][e], j0 + q * 32 * VEC + e));
        before += tied && ties;
      }
    }
  }
  __syncthreads();
  int n = sh.n_list;
  if (many_chunks || n > kList) {
    // the k best chunks (all of them, where there are no more), then the k best of each
    __syncthreads();
    if (threadIdx.x == 0) sh.n_list = 0;
    nc = min(top, nchunks);
    if (warp == 0) {
      if (few) {
        if (lane < nchunks) sh.chunk[lane] = lane;
      } else {
        warp_select(
            top, 0,
            [&](uint64_t limit) {
              uint64_t b = 0;
              for (int c = lane; c < nchunks; c += 32) {
                const uint64_t key = dealt_key(c);
                if (key < limit && key > b) b = key;
              }
              return b;
            },
            [&](int q, uint64_t key) { sh.chunk[q] = index_of(key); });
      }
    }
    __syncthreads();
    for (int i = warp; i < nc; i += kWarps) {
      const int j0 = sh.chunk[i] * kChunkElems + lane * VEC - shift;
      float v[Q][VEC];
#pragma unroll
      for (int q = 0; q < Q; ++q) load_piece<T>(row, j0 + q * 32 * VEC, V, -INFINITY, v[q]);
      warp_select(
          top, elem_floor,
          [&](uint64_t limit) {
            uint64_t b = 0;
#pragma unroll
            for (int q = 0; q < Q; ++q)
#pragma unroll
              for (int e = 0; e < VEC; ++e) {
                const int j = j0 + q * 32 * VEC + e;
                const uint64_t key = key_of(order_of(v[q][e]), j);
                if (j >= 0 && j < V && key < limit && key > b) b = key;
              }
            return b;
          },
          [&](int, uint64_t key) { list_element(key); });
    }
    __syncthreads();
    n = sh.n_list;
  }
  // each takes its place (the list's own order does not matter: keys differ)
  const float log_s = log_sum(st);
  for (int i = threadIdx.x; i < n; i += NT) {
    const uint64_t mine = sh.list[i];
    int larger = 0;
#pragma unroll 4
    for (int q = 0; q < n; ++q) larger += sh.list[q] > mine;
    if (larger < top) {
      top_ids[r * top + larger] = index_of(mine);
      top_logp[r * top + larger] = log_prob(value_of((uint32_t)(mine >> 32)), st, log_s);
    }
  }
}

// CTA (r, split): chunks [split * cps, (split + 1) * cps) of row r, dealt to the warps in turn.
// Per element the loop spends about six instructions (packed fp32 for the difference, the product
// and both sums; the maximum in the element's own type).  An unsplit row is finished here: while
// one CTA looks for its alternatives the others of the multiprocessor go on reading.
// NT: threads of the CTA.
template <typename T, bool TOP, bool WHOLE, int NT>
__global__ void __launch_bounds__(NT)
logprob_row_kernel(const T* __restrict__ x, int V, int64_t ld, int nchunks, int cps, RowOut o,
                   float4* __restrict__ part, float* chunk_max, int top, float* __restrict__ top_logp,
                   int32_t* __restrict__ top_ids) {
  constexpr int VEC = Elem<T>::kVec;
  constexpr int Q = kChunkElems / 32 / VEC;   // pieces of a chunk per lane
  constexpr int U = 4;                  // chunks per turn: four 16-byte loads a lane, eight of fp32 (1021 x 50021
                                        // fp32: 39 us against 43 with four; 4096 x 32768 bf16 loses 3 % with eight)
  constexpr int kWarps = NT / 32;
  launch_gate();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t r = blockIdx.x;
  const T* row = x + r * ld;
  const int shift = row_shift(row);
  const int c_begin = blockIdx.y * cps, c_end = min(nchunks, c_begin + cps);
  const bool again = gridDim.x - r <= kKeepBytes / ((int64_t)V * (int)sizeof(T));

  Target target{0.f, false};
  if (WHOLE && threadIdx.x == 0) target = fetch_target<T>(o, row, r, V);

  float m = -INFINITY;
  f32x2 s = 0, t = 0;
  for (int c0 = c_begin + warp; c0 < c_end; c0 += kWarps * U) {
    uint4 w[U][Q];
    const int first = c0 * kChunkElems - shift, last = (c0 + (U - 1) * kWarps) * kChunkElems - shift;
    if (first >= 0 && c0 + (U - 1) * kWarps < c_end && last + kChunkElems <= V) {
      // every piece of this turn is whole: one address, constant distances
      const uint4* p = reinterpret_cast<const uint4*>(row + first) + lane;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < Q; ++q) w[u][q] = again ? ld16(p + u * (kWarps * 32 * Q) + q * 32) : ld16_stream(p + u * (kWarps * 32 * Q) + q * 32);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int q = 0; q < Q; ++q) {
          const int c = c0 + u * kWarps;
          // (a chunk past the end reads as elements past the row's end)
          w[u][q] = load_raw<T>(row, c < c_end ? c * kChunkElems + (q * 32 + lane) * VEC - shift : V, V, minus_inf<T>());
        }
    }
    float mx = m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float cm = raw_max<T, false>(w[u][0]);
      if (Q == 2) cm = fmaxf(cm, raw_max<T, false>(w[u][Q - 1]));
      if (TOP) {
        asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(cm));
        const int c = c0 + u * kWarps;
        if (lane == 0 && c < c_end) chunk_max[r * nchunks + c] = cm;
      }
      mx = fmaxf(mx, cm);
    }
    if (!TOP) asm volatile("redux.sync.max.f32 %0, %0, 0xffffffff;" : "+f"(mx));
    if (mx > m) {
      rebase2(m, mx, s, t);
      m = mx;
    }
    const float base = -base_of(m);
    const f32x2 minus_base = pack2f(base, base);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int q = 0; q < Q; ++q)
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) accumulate2(raw_pair<T>(w[u][q], i), minus_base, s, t);
  }
  RowState st;
  float lo, hi;
  st.m = m;
  unpack2f(s, lo, hi);
  st.s = warp_sum(lo + hi);
  unpack2f(t, lo, hi);
  st.t = warp_sum(lo + hi);
  __shared__ RowState sh[kWarps];
  __shared__ RowState whole;
  if (lane == 0) sh[warp] = st;
  __syncthreads();
  if (warp == 0) {
    RowState a{-INFINITY, 0.f, 0.f};
    if (lane < kWarps) a = sh[lane];
    a = shfl_join(a);
    if (lane == 0) {
      whole = a;
      if (WHOLE) write_row(o, target, r, a);
      else part[r * gridDim.y + blockIdx.y] = make_float4(a.m, a.s, a.t, 0.f);
    }
  }
  if constexpr (TOP && WHOLE) {
    __shared__ TopShared ts;
    __syncthreads();   // (the chunks' maxima too)
    find_top<T, NT>(ts, row, r, V, nchunks, chunk_max + r * nchunks, whole, top, top_logp, top_ids);
  }
}

// Joins a row's parts (and finds its alternatives); one CTA per row.
template <typename T>
__global__ void __launch_bounds__(kThreads)
logprob_finish_kernel(const T* __restrict__ x, int V, int64_t ld, int nchunks, int nsplit, RowOut o,
                      const float4* __restrict__ part, float* chunk_max, int top, float* __restrict__ top_logp,
                      int32_t* __restrict__ top_ids) {
  __shared__ TopShared sh;
  __shared__ RowState whole;
  launch_gate();
  const int lane = threadIdx.x & 31;
  const int64_t r = blockIdx.x;
  const T* row = x + r * ld;
  if (threadIdx.x < 32) {
    const Target target = fetch_target<T>(o, row, r, V);
    RowState st{-INFINITY, 0.f, 0.f};
    for (int i = lane; i < nsplit; i += 32) {
      const float4 p = part[r * nsplit + i];
      st = join(st, RowState{p.x, p.y, p.z});
    }
    st = shfl_join(st);
    if (lane == 0) {
      write_row(o, target, r, st);
      whole = st;
    }
  }
  if (top == 0) return;
  __syncthreads();
  find_top<T, kThreads>(sh, row, r, V, nchunks, chunk_max + r * nchunks, whole, top, top_logp, top_ids);
}

// ---------------------------------------------------------------------------- gradient
// dx_j = dlp (1[j = t] - p_j) - dH p_j (log p_j + H): reads the logits once, writes once.
// With y = x - m (clamped far below, where p is zero): p = 2^(y log2 e - log2 S) and
// dx = -p (dH y + K), K = dlp + dH (H - log S).  A row with a NaN or +inf has log S = NaN.
struct GradRow {
  float base, minus_log2_s, d_h, k, d_lp;
  int32_t target;
  __device__ __forceinline__ float operator()(float x) const {
    const float y = fmaxf(x - base, kFarBelow);
    return -ex2(fmaf(y, kLog2e, minus_log2_s)) * fmaf(d_h, y, k);
  }
  __device__ __forceinline__ void pair(f32x2 x, float& lo, float& hi) const {
    unpack2f(add2(x, pack2f(-base, -base)), lo, hi);
    const f32x2 y = pack2f(fmaxf(lo, kFarBelow), fmaxf(hi, kFarBelow));
    unpack2f(fma2(y, pack2f(kLog2e, kLog2e), pack2f(minus_log2_s, minus_log2_s)), lo, hi);
    const f32x2 p = pack2f(ex2(lo), ex2(hi));
    unpack2f(mul2(p, fma2(pack2f(-d_h, -d_h), y, pack2f(-k, -k))), lo, hi);
  }
};

__device__ __forceinline__ GradRow grad_row(const LogprobGradArgs& a, int64_t r) {
  GradRow g;
  const float m = a.stats[2 * r], log_s = a.stats[2 * r + 1];
  const int32_t t = a.targets[r];
  const bool has = t >= 0 && t < a.V;
  g.target = has ? t : -1;
  g.d_lp = has && a.d_logp ? a.d_logp[r] : 0.f;
  g.d_h = a.d_entropy ? a.d_entropy[r] : 0.f;
  g.base = base_of(m);
  g.minus_log2_s = -log_s * kLog2e;
  g.k = fmaf(g.d_h, a.entropy[r] - log_s, g.d_lp);
  // A row that nothing is asked of, or without a distribution: p = 0 for every x, NaN and
  // infinities included (padding may hold anything).
  if ((g.d_lp == 0.f && g.d_h == 0.f) || (m == -INFINITY && log_s == 0.f)) {
    g.base = INFINITY;
    g.minus_log2_s = g.d_h = g.k = g.d_lp = 0.f;
  }
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
  for (int j = lane; j < (int)a.V; j += 32)
    out[j] = Elem<T>::from_float(g(Elem<T>::to_float(row[j])) + (j == g.target ? g.d_lp : 0.f));
}

// CTA (r, segment): kThreads * kUnroll pieces of row r.
template <typename T>
__global__ void __launch_bounds__(kThreads) logprob_grad_kernel(LogprobGradArgs a) {
  constexpr int VEC = Elem<T>::kVec;
  constexpr int U = kUnroll;
  launch_gate();
  const int64_t r = a.rows - 1 - blockIdx.x;   // from the row that was read last
  const int V = (int)a.V;
  const T* row = static_cast<const T*>(a.logits) + r * a.ld;
  T* out = static_cast<T*>(a.d_logits) + r * a.ldd;
  const int shift = row_shift(row);
  const bool aligned = row_shift(out) == shift;
  const bool large = a.rows * a.V * (int64_t)sizeof(T) > kKeepBytes;   // a gradient that L2 would not hold anyway
  const int j0 = ((int)blockIdx.y * (kThreads * U) + (int)threadIdx.x) * VEC - shift;
  uint4 w[U];
#pragma unroll
  for (int u = 0; u < U; ++u) w[u] = load_raw<T>(row, j0 + u * kThreads * VEC, V, 0);
  const GradRow g = grad_row(a, r);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int j = j0 + u * kThreads * VEC;
    if (j >= V) break;
    float d[VEC];
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) g.pair(raw_pair<T>(w[u], i), d[2 * i], d[2 * i + 1]);
    if (g.target >= j && g.target < j + VEC) {
#pragma unroll
      for (int e = 0; e < VEC; ++e)
        if (j + e == g.target) d[e] += g.d_lp;
    }
    if (large) store_floats<T, VEC, true>(out, j, V, aligned, d);
    else store_floats<T, VEC>(out, j, V, aligned, d);
  }
}

// ------------------------------------------------------------------------------ host
// upper bound over every alignment of a row
int64_t chunk_count(int64_t V, int dtype) {
  return (V + (dtype == OLSGD_F32 ? 3 : 7) + kChunkElems - 1) / kChunkElems;
}
// Parts a row is split into.  One part per row once the rows alone give every multiprocessor
// four CTAs (1021 rows of 50021 fp32 logits took no longer whole than in three parts); before that as
// many parts as fill the GPU that often, none shorter than one unrolled turn of a CTA's
// warps (32 chunks).
int split_count(int64_t rows, int64_t nchunks) {
  const int64_t want = (4LL * 148 + rows - 1) / rows;
  const int64_t most = (nchunks + kWarps * kUnroll - 1) / (kWarps * kUnroll);
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
  float* cmax = reinterpret_cast<float*>(part + a.rows * nsplit);
  const dim3 grid((unsigned)a.rows, (unsigned)nsplit);
  const bool whole = nsplit == 1;
  const bool narrow = whole && (a.top > 0 || a.V <= kNarrowRow);
  auto k = narrow ? (a.top > 0 ? logprob_row_kernel<T, true, true, kThreads / 2> : logprob_row_kernel<T, false, true, kThreads / 2>)
           : whole ? logprob_row_kernel<T, false, true, kThreads>
                   : (a.top > 0 ? logprob_row_kernel<T, true, false, kThreads> : logprob_row_kernel<T, false, false, kThreads>);
  const cudaError_t e = launch_chained(k, grid, dim3(narrow ? kThreads / 2 : kThreads), 0, s, x, (int)a.V, a.ld, nchunks, cps,
                                       o, part, cmax, a.top, a.top_logp, a.top_ids);
  if (e != cudaSuccess || whole) return e;
  return launch_chained(logprob_finish_kernel<T>, dim3((unsigned)a.rows), dim3(kThreads), 0, s, x, (int)a.V, a.ld, nchunks,
                        nsplit, o, (const float4*)part, cmax, a.top, a.top_logp, a.top_ids);
}

template <typename T>
cudaError_t backward(const LogprobGradArgs& a, cudaStream_t s) {
  if (a.V <= kWarpRowMax)
    return launch_chained(logprob_grad_warp_kernel<T>, dim3((unsigned)((a.rows + kWarps - 1) / kWarps)), dim3(kThreads),
                          0, s, a);
  // rows that all start on a 16-byte boundary have no partial first piece
  const bool on = ((reinterpret_cast<uintptr_t>(a.logits) | (uintptr_t)(a.ld * sizeof(T))) & 15) == 0;
  const int64_t pieces = (a.V + (on ? 1 : 2) * (Elem<T>::kVec - 1)) / Elem<T>::kVec;
  const int64_t per = kThreads * kUnroll;
  return launch_chained(logprob_grad_kernel<T>, dim3((unsigned)a.rows, (unsigned)((pieces + per - 1) / per)),
                        dim3(kThreads), 0, s, a);
}

}  // namespace

size_t logprob_workspace(int dtype, int64_t rows, int64_t V, int top) {
  if (V <= kWarpRowMax) return 0;
  const Plan p = plan(rows, V, dtype);
  if (p.nsplit == 1 && top == 0) return 0;
  // the parts of every row, and the chunk maxima
  return (size_t)rows * p.nsplit * sizeof(float4) + (top > 0 ? (size_t)rows * p.nchunks * sizeof(float) : 0);
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
