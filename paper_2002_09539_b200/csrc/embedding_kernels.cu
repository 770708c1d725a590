// Embedding lookup with a scale, and the gradient of the table by sorted tokens.
//
//   out[t] = scale * W[id_t];   dW[v] = scale * sum over {t : id_t = v} of dout[t]
//
// Lookup: a warp per token, 16 bytes per lane; bound by the rows read and written.
//
// Gradient: the tokens are sorted by id with a stable radix sort (8 bits a pass, counts and
// prefix sums only: no order depends on timing), so that a row of the table gets its tokens in
// the order of their positions.  The sorted list is cut into chunks of kChunk tokens; a CTA
// adds up a chunk's rows in fp32 registers and writes every table row whose tokens all lie
// in the chunk.  Rows that reach over a chunk's end leave partial sums, which a third kernel adds
// in chunk order: a token that fills half of the batch costs as much as any other.  Table rows
// without a token are zeroed meanwhile.  Each sum is rounded once.
// Bound by dout read once and the table's gradient written once; writing the zeros is most of it
// where the vocabulary is larger than the batch, so it runs beside the sort (which fills eight
// multiprocessors a list and moves next to nothing).
//
// Ids outside [0, V) mark positions without a token: a zero row, no gradient.
#include "operator_common.cuh"
#include "operators_internal.h"

namespace olsgd {
namespace {

using namespace op;

// ------------------------------------------------------------------------------ lookup
constexpr int kLookupThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kLookupThreads)
embedding_kernel(const T* __restrict__ table, int64_t V, int64_t D, int64_t table_worker, int64_t table_row,
                 const int32_t* __restrict__ ids, int64_t tokens, T* __restrict__ out, float scale, bool vec) {
  constexpr int N = Elem<T>::kVec;
  launch_gate();
  const int lane = threadIdx.x & 31;
  const int64_t t = (int64_t)blockIdx.x * (kLookupThreads / 32) + (threadIdx.x >> 5);
  if (t >= tokens) return;
  const int64_t row = (int64_t)blockIdx.y * tokens + t;
  const int32_t id = ids[row];
  const bool has = id >= 0 && id < V;
  const T* src = table + (int64_t)blockIdx.y * table_worker + (has ? id : 0) * table_row;
  T* dst = out + row * D;
  if (vec) {
    constexpr int U = 4;
    for (int64_t j0 = lane * N; j0 < D; j0 += 32 * N * U) {
      uint4 w[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t j = j0 + u * 32 * N;
        w[u] = (has && j < D) ? ld16(src + j) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t j = j0 + u * 32 * N;
        float v[N];
        Elem<T>::unpack(w[u], v);
#pragma unroll
        for (int e = 0; e < N; ++e) v[e] = has ? v[e] * scale : 0.f;
        if (j < D) *reinterpret_cast<uint4*>(dst + j) = Elem<T>::pack(v);
      }
    }
  } else {
    for (int64_t j = lane; j < D; j += 32)
      dst[j] = Elem<T>::from_float(has ? Elem<T>::to_float(src[j]) * scale : 0.f);
  }
}

// -------------------------------------------------------------------------------- sort
// Entries are (id << 32 | position); ids outside [0, V) become V and end up last.
constexpr int kSortThreads = 512;
constexpr int kSortWarps = kSortThreads / 32;
constexpr int kSortItems = 8;                              // entries per thread
constexpr int kSortTile = kSortThreads * kSortItems;       // entries per CTA
constexpr int kBins = 256;
constexpr int kSortCluster = 8;                            // CTAs that sort a list in one launch

// Table rows without a token: as many a CTA as give the GPU a few CTAs per multiprocessor, of 16 to 256 KB.
constexpr int64_t kZeroBytesMin = 16 << 10, kZeroBytesMax = 256 << 10;
constexpr int kZeroRowsMax = 2048;
struct ZeroArgs {
  void* dtable;              // [m][V][row_bytes], workers worker_bytes apart
  int64_t V, row_bytes, worker_bytes;
  int rows, ctas;            // rows of a CTA, CTAs of a worker
};
// Rows [v0, v0 + n) of a worker that are not present.  Zeros are the same in every type.  Long rows: a
// warp each, 32 bytes a lane between the boundaries, 2 at the ends.  Short ones are walked as one run
// of bytes, 32 a thread, which are stored whole where no present row shares them and by twos where
// one does (or where the run ends): a 4096-byte row costs that way 10 % more, one of 48 bytes a
// third.
constexpr uint32_t kLongRow = 1024;
__device__ __forceinline__ void store_zeros(char* p) {
  asm volatile("st.global.v8.b32 [%0], {%1, %1, %1, %1, %1, %1, %1, %1};" ::"l"(p), "r"(0u) : "memory");
}
__device__ __forceinline__ void zero_rows(const ZeroArgs& z, int64_t worker, int64_t v0, int n, const uint8_t* present) {
  char* run = static_cast<char*>(z.dtable) + worker * z.worker_bytes + v0 * z.row_bytes;
  const uint32_t row = (uint32_t)z.row_bytes;
  if (row >= kLongRow) {
    const int lane = threadIdx.x & 31;
    for (int r = threadIdx.x >> 5; r < n; r += blockDim.x >> 5) {
      if (present[r]) continue;
      char *p = run + (int64_t)r * row, *end = p + row;
      char* body = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(p) + 31) & ~(uintptr_t)31);
      char* tail = body + ((end - body) & ~(int64_t)31);
      for (char* q = p + lane * 2; q < body; q += 64) *reinterpret_cast<uint16_t*>(q) = 0;
      for (char* q = body + lane * 32; q < tail; q += 1024) store_zeros(q);
      for (char* q = tail + lane * 2; q < end; q += 64) *reinterpret_cast<uint16_t*>(q) = 0;
    }
    return;
  }
  const uint32_t bytes = row * n, shift = (uint32_t)(reinterpret_cast<uintptr_t>(run) & 31);
  for (uint32_t at = threadIdx.x * 32; at < bytes + shift; at += blockDim.x * 32) {
    // bytes [lo, hi) of the run
    const uint32_t lo = at < shift ? 0 : at - shift, hi = min(bytes, at + 32 - shift);
    const uint32_t r0 = lo / row, r1 = hi - r0 * row <= row ? r0 : (hi - 1) / row;
    bool any = false, all = true;
    for (uint32_t r = r0; r <= r1; ++r) {
      if (present[r]) any = true;
      else all = false;
    }
    if (all) continue;
    if (!any && hi - lo == 32) {
      store_zeros(run + lo);
    } else {
      uint32_t r = r0, next = (r0 + 1) * row;
      for (uint32_t b = lo; b < hi; b += 2) {
        if (b >= next) {
          ++r;
          next += row;
        }
        if (!present[r]) *reinterpret_cast<uint16_t*>(run + b) = 0;
      }
    }
  }
}

struct SortArgs {
  const int32_t* ids;        // [m][T]
  const uint64_t* in;        // [m][T], or null: the ids themselves
  uint64_t* out;             // [m][T]
  uint32_t* counts;          // [m][kBins][tiles]
  uint32_t* joins;           // two counters that the summing kernel starts from: zeroed here
  int64_t T;
  uint32_t V;
  int tiles, shift;
};

// (through L2: the other CTAs of a cluster wrote it)
__device__ __forceinline__ uint64_t entry_at(const SortArgs& a, const uint64_t* in, int64_t worker, int64_t t) {
  if (in) return __ldcg(reinterpret_cast<const unsigned long long*>(in + worker * a.T + t));
  const int32_t id = a.ids[worker * a.T + t];
  const uint32_t key = id >= 0 && (uint32_t)id < a.V ? (uint32_t)id : a.V;
  return ((uint64_t)key << 32) | (uint32_t)t;
}
__device__ __forceinline__ uint32_t digit_of(uint64_t e, int shift) { return (uint32_t)(e >> (32 + shift)) & (kBins - 1); }

// How often each digit occurs in a tile.
__global__ void __launch_bounds__(kSortThreads) sort_count_kernel(const SortArgs a) {
  __shared__ uint32_t hist[kBins];
  launch_gate();
  const int64_t worker = blockIdx.y, t0 = (int64_t)blockIdx.x * kSortTile;
  if (threadIdx.x < kBins) hist[threadIdx.x] = 0;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kSortItems; ++i) {
    const int64_t t = t0 + i * kSortThreads + threadIdx.x;
    if (t < a.T) atomicAdd(&hist[digit_of(entry_at(a, a.in, worker, t), a.shift)], 1u);
  }
  __syncthreads();
  if (threadIdx.x < kBins) a.counts[(worker * kBins + threadIdx.x) * a.tiles + blockIdx.x] = hist[threadIdx.x];
}

// One tile of one pass.  An entry's place is where its digit starts among all tiles, plus what
// earlier tiles, earlier warps and earlier entries of the warp hold of the digit.
struct TileSort {
  uint32_t warp_count[kSortWarps][kBins];
  uint32_t start[kBins];
  uint32_t warp_total[kBins / 32];
};
template <int ITEMS>
struct Ranked {
  uint64_t e[ITEMS];
  uint32_t rank[ITEMS];   // among the warp's entries of the digit
};

template <int ITEMS>
__device__ __forceinline__ void rank_tile(const SortArgs& a, const uint64_t* in, int shift, int64_t worker, int64_t t0, TileSort& sh,
                                          Ranked<ITEMS>& r) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  for (int b = lane; b < kBins; b += 32) sh.warp_count[warp][b] = 0;
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const int64_t t = t0 + i * 32 + lane;
    r.e[i] = t < a.T ? entry_at(a, in, worker, t) : ~0ull;
  }
  __syncwarp();
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    const bool live = t0 + i * 32 + lane < a.T;
    const uint32_t d = digit_of(r.e[i], shift);
    // the live lanes with the same digit, bit by bit (a match instruction walks over the distinct
    // digits instead)
    uint32_t same = __ballot_sync(0xffffffffu, live);
#pragma unroll
    for (int bit = 0; bit < 8; ++bit) {
      const bool set = (d >> bit) & 1;
      const uint32_t with = __ballot_sync(0xffffffffu, set);
      same &= set ? with : ~with;
    }
    const uint32_t before = live ? sh.warp_count[warp][d] : 0;
    r.rank[i] = before + __popc(same & ((1u << lane) - 1));
    __syncwarp();
    if (live && (same & ((1u << lane) - 1)) == 0) sh.warp_count[warp][d] = before + __popc(same);
    __syncwarp();
  }
  __syncthreads();
}

// total, earlier: what thread b < kBins knows of digit b over all tiles, and over the earlier ones.
template <int ITEMS>
__device__ __forceinline__ void place_tile(const SortArgs& a, uint64_t* out, int shift, int64_t worker, int64_t t0, uint32_t total,
                                           uint32_t earlier, TileSort& sh, const Ranked<ITEMS>& r) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, b = threadIdx.x;
  uint32_t scan = total;   // inclusive over the digits
  if (b < kBins) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const uint32_t n = __shfl_up_sync(0xffffffffu, scan, o);
      if (lane >= o) scan += n;
    }
    if (lane == 31) sh.warp_total[warp] = scan;
  }
  __syncthreads();
  if (b < kBins) {
    uint32_t base = scan - total + earlier;
    for (int w = 0; w < warp; ++w) base += sh.warp_total[w];
    sh.start[b] = base;
    // counts of a warp become what the warps before it hold
    uint32_t run = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) {
      const uint32_t n = sh.warp_count[w][b];
      sh.warp_count[w][b] = run;
      run += n;
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < ITEMS; ++i) {
    if (t0 + i * 32 + lane < a.T) {
      const uint32_t d = digit_of(r.e[i], shift);
      out[worker * a.T + sh.start[d] + sh.warp_count[warp][d] + r.rank[i]] = r.e[i];
    }
  }
}

__global__ void __launch_bounds__(kSortThreads) sort_place_kernel(const SortArgs a) {
  __shared__ TileSort sh;
  launch_gate();
  const int64_t worker = blockIdx.y, t0 = (int64_t)blockIdx.x * kSortTile + (threadIdx.x >> 5) * (32 * kSortItems);
  if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) a.joins[0] = a.joins[1] = 0;
  Ranked<kSortItems> r;
  rank_tile(a, a.in, a.shift, worker, t0, sh, r);
  uint32_t total = 0, earlier = 0;
  if (threadIdx.x < kBins) {
    const uint32_t* c = a.counts + (worker * kBins + threadIdx.x) * a.tiles;
#pragma unroll 4
    for (int i = 0; i < a.tiles; ++i) {
      const uint32_t n = c[i];
      total += n;
      if (i < (int)blockIdx.x) earlier += n;
    }
  }
  place_tile(a, a.out, a.shift, worker, t0, total, earlier, sh, r);
}

// Lists of up to kSortCluster tiles: a cluster of CTAs, one tile each, makes all passes in one
// launch and exchanges its counts through distributed shared memory (2 x 16384 tokens, two passes,
// cold: 14 us against 29 us as a count and a placing launch per pass).  Tiles are half as
// long (ITEMS = 4) where eight of those hold the list.  The passes alternate between two lists.
// CTAs past the lists' zero table rows: each looks through the ids for its rows itself (they come
// from L2), and so waits for no sort.
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release;" ::: "memory");
  asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
}
__device__ __forceinline__ uint32_t ld_cluster(const uint32_t* p, uint32_t cta) {
  uint32_t addr = static_cast<uint32_t>(__cvta_generic_to_shared(p)), v;
  asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(addr) : "r"(cta));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
  return v;
}
template <int ITEMS>
__global__ void __launch_bounds__(kSortThreads)
sort_cluster_kernel(const SortArgs a, uint64_t* first, uint64_t* second, int passes, int m, const ZeroArgs z) {
  __shared__ TileSort sh;
  __shared__ uint32_t hist[kBins];
  __shared__ uint8_t present[kZeroRowsMax];
  launch_gate();
  if (blockIdx.x >= (unsigned)m * a.tiles) {
    const int64_t at = blockIdx.x - (int64_t)m * a.tiles;
    const int64_t worker = at / z.ctas, v0 = at % z.ctas * z.rows;
    if (worker >= m) return;   // (the grid is a multiple of the cluster)
    const int n = (int)(z.V - v0 < z.rows ? z.V - v0 : z.rows);
    for (int r = threadIdx.x; r < n; r += kSortThreads) present[r] = 0;
    __syncthreads();
#pragma unroll 8
    for (int64_t t = threadIdx.x; t < a.T; t += kSortThreads) {
      const int64_t r = a.ids[worker * a.T + t] - v0;
      if (r >= 0 && r < n) present[r] = 1;
    }
    __syncthreads();
    zero_rows(z, worker, v0, n, present);
    return;
  }
  const int tile = blockIdx.x % a.tiles;
  const int64_t worker = blockIdx.x / a.tiles, t0 = ((int64_t)tile * kSortThreads + (threadIdx.x & ~31u)) * ITEMS;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.joins[0] = a.joins[1] = 0;
  const uint64_t* in = nullptr;
  uint64_t* out = first;
  for (int p = 0; p < passes; ++p) {
    Ranked<ITEMS> r;
    rank_tile(a, in, 8 * p, worker, t0, sh, r);
    const int b = threadIdx.x;
    if (b < kBins) {
      uint32_t n = 0;
#pragma unroll
      for (int w = 0; w < kSortWarps; ++w) n += sh.warp_count[w][b];
      hist[b] = n;
    }
    cluster_sync();
    uint32_t total = 0, earlier = 0;
    if (b < kBins) {
      for (int c = 0; c < a.tiles; ++c) {
        const uint32_t n = ld_cluster(&hist[b], c);
        total += n;
        if (c < tile) earlier += n;
      }
    }
    place_tile(a, out, 8 * p, worker, t0, total, earlier, sh, r);
    cluster_sync();   // the list is complete, and nobody reads this CTA's counts any more
    in = out;
    out = out == first ? second : first;
  }
}

// ---------------------------------------------------------------------------- reduction
constexpr int kChunk = 32;             // sorted tokens per CTA
constexpr int kSumThreads = 128;
constexpr int kCols = 8;               // columns per thread
constexpr int kSlice = kSumThreads * kCols;   // columns per CTA
constexpr int kShortRow = 8;           // parts that one warp adds up
constexpr int kJoinThreads = 256;
constexpr int kJoinCols = 128;         // columns per joining CTA

struct SumArgs {
  const uint64_t* sorted;   // [m][T]
  const void* dout;         // [m][T][D] with strides
  int64_t dout_worker, dout_row;
  void* dtable;             // [m][V][D], workers out_worker apart
  int64_t out_worker;
  float* part;              // [m][chunks][2][pitch]: the row a chunk shares with the one before, with the one after
  uint32_t* joins;          // how many chunks a row starts in that reaches past their end: short rows, long rows ...
  uint32_t* join_list;      // ... and which: worker * chunks + chunk, in any order, short ones from the front, long from the back
  int64_t T, V, D, pitch;
  int chunks;
  ZeroArgs zero;            // zero.ctas of a worker in the summing launch (none where the sort's launch had them)
  float scale;
  bool vec_in, vec_out;
};

__device__ __forceinline__ uint32_t key_at(const uint64_t* s, int64_t i) { return (uint32_t)(s[i] >> 32); }

// First position of the sorted list whose key is >= v; by a warp, 32 probes at a time.
__device__ __forceinline__ int64_t warp_lower_bound(const uint64_t* s, int64_t n, uint32_t v) {
  const int lane = threadIdx.x & 31;
  int64_t lo = 0, hi = n;   // answer in [lo, hi]
  while (lo < hi) {
    const int64_t width = (hi - lo + 31) / 32;
    const int64_t probe = lo + lane * width + width - 1;    // last of this lane's stretch
    const bool below = probe < hi && key_at(s, probe) < v;
    const int full = __popc(__ballot_sync(0xffffffffu, below));   // stretches that lie below v (a prefix)
    lo += full * width;
    if (lo > hi) lo = hi;
    const int64_t end = lo + width - 1;   // the stretch that is not, if there is one
    if (end < hi) hi = end;
    if (width == 1) break;
  }
  return lo;
}

template <typename TO>
__device__ __forceinline__ void write_cols(TO* row, int64_t c0, int64_t D, bool vec, bool strided, const float* v) {
  if (!strided) {
    store_floats<TO, kCols>(row, c0, D, vec, v);
  } else {
#pragma unroll
    for (int e = 0; e < kCols; ++e)
      if (c0 + e * kSumThreads < D) row[c0 + e * kSumThreads] = Elem<TO>::from_float(v[e]);
  }
}

// CTAs 0 .. chunks - 1 of a worker: one chunk each; the rest, if any: table rows without a token.
// VEC: rows of dout and of the table start on 16-byte boundaries; a thread has 8 consecutive
// columns then, and columns kSumThreads apart otherwise (coalesced either way).
template <typename TI, typename TO, bool VEC>
__global__ void __launch_bounds__(kSumThreads) embedding_sum_kernel(const SumArgs a) {
  launch_gate();
  const int64_t worker = blockIdx.z;
  const uint64_t* sorted = a.sorted + worker * a.T;
  TO* table = static_cast<TO*>(a.dtable) + worker * a.out_worker;
  const int64_t slice = (int64_t)blockIdx.y * kSlice;
  const int64_t c0 = slice + (VEC ? threadIdx.x * kCols : threadIdx.x);

  if ((int)blockIdx.x >= a.chunks) {
    // ---- rows without a token (long lists: the sorted one tells)
    __shared__ uint8_t present[kZeroRowsMax];
    __shared__ int64_t range[2];
    const int64_t v0 = (int64_t)(blockIdx.x - a.chunks) * a.zero.rows;
    const int n = (int)(a.V - v0 < a.zero.rows ? a.V - v0 : a.zero.rows);
    for (int r = threadIdx.x; r < n; r += kSumThreads) present[r] = 0;
    if (threadIdx.x < 64) {   // one warp for each end
      const int64_t p = warp_lower_bound(sorted, a.T, (uint32_t)(threadIdx.x < 32 ? v0 : v0 + n));
      if ((threadIdx.x & 31) == 0) range[threadIdx.x >> 5] = p;
    }
    __syncthreads();
    for (int64_t i = range[0] + threadIdx.x; i < range[1]; i += kSumThreads) present[key_at(sorted, i) - v0] = 1;
    __syncthreads();
    if (blockIdx.y == 0) zero_rows(a.zero, worker, v0, n, present);
    return;
  }

  // ---- a chunk of the sorted tokens
  __shared__ uint64_t entry[kChunk + 2];
  const int64_t i0 = (int64_t)blockIdx.x * kChunk;
  const int n = (int)(a.T - i0 < kChunk ? a.T - i0 : kChunk);
  if (threadIdx.x < kChunk + 2) {
    const int64_t i = i0 + threadIdx.x - 1;   // with the neighbours on both sides; ~0: none
    entry[threadIdx.x] = i >= 0 && i < a.T && (int)threadIdx.x <= n + 1 ? sorted[i] : ~0ull;
  }
  __syncthreads();
  const TI* dout = static_cast<const TI*>(a.dout) + worker * a.dout_worker;
  float* part = a.part + (worker * a.chunks + blockIdx.x) * 2 * a.pitch;
  constexpr int U = 8;
  float acc[kCols];
#pragma unroll
  for (int e = 0; e < kCols; ++e) acc[e] = 0.f;
  bool from_before = (uint32_t)(entry[0] >> 32) == (uint32_t)(entry[1] >> 32);
  for (int k0 = 0; k0 < n; k0 += U) {
    float v[U][kCols];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      // Every load is made, of a row and columns that exist (no branches between them); what does not
      // count is not stored.
      const TI* row = dout + (int64_t)(uint32_t)entry[1 + min(k0 + u, n - 1)] * a.dout_row;
      if (VEC) {
#pragma unroll
        for (int q = 0; q < kCols / Elem<TI>::kVec; ++q)
          Elem<TI>::unpack(ld16_stream(row + (c0 < a.D ? c0 : 0) + q * Elem<TI>::kVec), v[u] + q * Elem<TI>::kVec);
      } else {
#pragma unroll
        for (int e = 0; e < kCols; ++e) {
          const int64_t c = c0 + e * kSumThreads;
          v[u][e] = Elem<TI>::to_float(row[c < a.D ? c : 0]);
        }
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u;
      if (k >= n) break;
#pragma unroll
      for (int e = 0; e < kCols; ++e) acc[e] += v[u][e];
      const uint32_t key = (uint32_t)(entry[1 + k] >> 32), next = (uint32_t)(entry[2 + k] >> 32);
      if (k + 1 < n && next == key) continue;
      const bool to_after = k + 1 == n && next == key;
      if (key < a.V) {
        if (from_before || to_after) {
          if (!from_before && blockIdx.y == 0 && threadIdx.x == 0) {
            const uint32_t at = (uint32_t)worker * a.chunks + blockIdx.x;
            const int64_t far = ((int64_t)blockIdx.x + kShortRow) * kChunk;
            if (far < a.T && key_at(sorted, far) == key) a.join_list[gridDim.z * a.chunks - 1 - atomicAdd(a.joins + 1, 1u)] = at;
            else a.join_list[atomicAdd(a.joins, 1u)] = at;
          }
          write_cols<float>(part + (from_before ? 0 : a.pitch), c0, a.D, VEC, !VEC, acc);
        } else {
          float r[kCols];
#pragma unroll
          for (int e = 0; e < kCols; ++e) r[e] = acc[e] * a.scale;
          write_cols<TO>(table + (int64_t)key * a.D, c0, a.D, VEC, !VEC, r);
        }
      }
      from_before = false;
#pragma unroll
      for (int e = 0; e < kCols; ++e) acc[e] = 0.f;
    }
  }
}

// The table rows that start in one chunk and reach past its end, as listed by the summing kernel (in
// any order: each is formed by itself): the row's part of its first chunk, then those of the chunks
// that follow.  A short row is one CTA's, a warp per slice of columns; of a long one each slice is,
// each eighth of the parts by a warp of its own, joined in a fixed order.
template <typename TO>
__global__ void __launch_bounds__(kJoinThreads) embedding_join_kernel(const SumArgs a, int64_t n_lists) {
  constexpr int kJoinWarps = kJoinThreads / 32;
  __shared__ float4 sh[kJoinWarps][32];
  launch_gate();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int64_t slices = (a.D + kJoinCols - 1) / kJoinCols;
  const uint32_t n_short = a.joins[0];
  const int64_t items = n_short + (int64_t)a.joins[1] * slices;
  for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const bool is_short = item < n_short;
    const int64_t of_long = item - n_short;
    const uint32_t at = is_short ? a.join_list[item] : a.join_list[n_lists - 1 - of_long / slices];
    const int64_t worker = at / a.chunks, c = at % a.chunks;
    const uint64_t* sorted = a.sorted + worker * a.T;
    const uint32_t key = key_at(sorted, (c + 1) * kChunk - 1);
    // the last chunk that holds the key: chunks ahead are probed a warp's width at a time
    int64_t end = c + 1;
    for (;;) {
      const int64_t probe = end + lane;   // does chunk `probe` + 1 begin with the key?
      const int64_t i = (probe + 1) * kChunk;
      const bool more = i < a.T && key_at(sorted, i) == key;
      const uint32_t yes = __ballot_sync(0xffffffffu, more);
      const int run = yes == 0xffffffffu ? 32 : __ffs(~yes) - 1;
      end += run;
      if (run < 32) break;
    }
    const float* part = a.part + worker * a.chunks * 2 * a.pitch;
    TO* row = static_cast<TO*>(a.dtable) + worker * a.out_worker + (int64_t)key * a.D;
    // the parts first, first + step, ... of the row (part 0: in chunk c), columns col to col + 3
    // (pitch is a multiple of four: whole pieces; what lies past D is not stored)
    auto sum = [&](int64_t col, int64_t first, int64_t step) {
      float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
      if (col < a.D) {
#pragma unroll 4
        for (int64_t k = c + first; k <= end; k += step) {
          const float4 v = *reinterpret_cast<const float4*>(part + (k * 2 + (k == c ? 1 : 0)) * a.pitch + col);
          acc.x += v.x;
          acc.y += v.y;
          acc.z += v.z;
          acc.w += v.w;
        }
      }
      return acc;
    };
    auto store = [&](int64_t col, const float4& v) {
      const float r[4] = {v.x * a.scale, v.y * a.scale, v.z * a.scale, v.w * a.scale};
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < a.D) row[col + e] = Elem<TO>::from_float(r[e]);
    };
    if (is_short) {
      for (int64_t slice = warp; slice < slices; slice += kJoinWarps) {
        const int64_t col = slice * kJoinCols + lane * 4;
        store(col, sum(col, 0, 1));
      }
    } else {
      const int64_t col = of_long % slices * kJoinCols + lane * 4;
      sh[warp][lane] = sum(col, warp, kJoinWarps);
      __syncthreads();
      if (warp == 0) {
        float4 t = sh[0][lane];
#pragma unroll
        for (int w = 1; w < kJoinWarps; ++w) {
          const float4 v = sh[w][lane];
          t.x += v.x;
          t.y += v.y;
          t.z += v.z;
          t.w += v.w;
        }
        store(col, t);
      }
      __syncthreads();
    }
  }
}

// --------------------------------------------------------------------------------- host
constexpr size_t round256(size_t v) { return (v + 255) / 256 * 256; }
int64_t tiles_of(int64_t T) { return (T + kSortTile - 1) / kSortTile; }
int64_t chunks_of(int64_t T) { return (T + kChunk - 1) / kChunk; }
int64_t pitch_of(int64_t D) { return (D + 3) / 4 * 4; }

struct Layout {
  size_t a, b, counts, joins, part, total;
};
Layout layout_of(int64_t m, int64_t T, int64_t D) {
  Layout l;
  const size_t list = round256((size_t)m * T * sizeof(uint64_t));
  l.a = 0;
  l.b = list;
  l.counts = 2 * list;
  l.joins = l.counts + (tiles_of(T) > kSortCluster ? round256((size_t)m * kBins * tiles_of(T) * sizeof(uint32_t)) : 0);
  l.part = l.joins + 256 + round256((size_t)m * chunks_of(T) * sizeof(uint32_t));
  l.total = l.part + round256((size_t)m * chunks_of(T) * 2 * pitch_of(D) * sizeof(float));
  return l;
}

bool rows_of_16(const void* p, int64_t worker, int64_t row, int64_t m, int64_t rows, int size) {
  return (reinterpret_cast<uintptr_t>(p) & 15) == 0 && (rows == 1 || row * size % 16 == 0) && (m == 1 || worker * size % 16 == 0);
}

template <typename TI, typename TO>
cudaError_t sum_rows(const SumArgs& a, int64_t m, cudaStream_t s) {
  const dim3 grid((unsigned)(a.chunks + a.zero.ctas), (unsigned)((a.D + kSlice - 1) / kSlice), (unsigned)m);
  auto k = a.vec_in && a.vec_out ? embedding_sum_kernel<TI, TO, true> : embedding_sum_kernel<TI, TO, false>;
  cudaError_t e = launch_chained(k, grid, dim3(kSumThreads), 0, s, a);
  if (e != cudaSuccess || a.chunks <= 1) return e;
  const int64_t most = m * a.chunks * ((a.D + kJoinCols - 1) / kJoinCols), room = 148 * 8;
  return launch_chained(embedding_join_kernel<TO>, dim3((unsigned)(most < room ? most : room)), dim3(kJoinThreads), 0, s, a, m * a.chunks);
}

template <typename TI>
cudaError_t sum_rows_to(int dtype, const SumArgs& a, int64_t m, cudaStream_t s) {
  if (dtype == OLSGD_F32) return sum_rows<TI, float>(a, m, s);
  if (dtype == OLSGD_BF16) return sum_rows<TI, __nv_bfloat16>(a, m, s);
  return sum_rows<TI, __half>(a, m, s);
}

template <typename T>
cudaError_t lookup(const EmbeddingArgs& a, cudaStream_t s) {
  const bool vec = a.D % Elem<T>::kVec == 0 && rows_of_16(a.table, a.table_worker, a.table_row, a.m, a.V, sizeof(T)) &&
                   (reinterpret_cast<uintptr_t>(a.out) & 15) == 0;
  const dim3 grid((unsigned)((a.T + kLookupThreads / 32 - 1) / (kLookupThreads / 32)), (unsigned)a.m);
  return launch_chained(embedding_kernel<T>, grid, dim3(kLookupThreads), 0, s, static_cast<const T*>(a.table), a.V, a.D,
                        a.table_worker, a.table_row, a.ids, a.T, static_cast<T*>(a.out), a.scale, vec);
}

}  // namespace

cudaError_t launch_embedding_forward(const EmbeddingArgs& a, cudaStream_t s) {
  switch (a.dtype) {
    case OLSGD_F32: return lookup<float>(a, s);
    case OLSGD_BF16: return lookup<__nv_bfloat16>(a, s);
    default: return lookup<__half>(a, s);
  }
}

size_t embedding_workspace(int64_t m, int64_t T, int64_t D) { return layout_of(m, T, D).total; }

cudaError_t launch_embedding_backward(const EmbeddingGradArgs& g, cudaStream_t s) {
  const Layout l = layout_of(g.m, g.T, g.D);
  uint8_t* ws = static_cast<uint8_t*>(g.ws);
  uint64_t* lists[2] = {reinterpret_cast<uint64_t*>(ws + l.a), reinterpret_cast<uint64_t*>(ws + l.b)};
  uint32_t* joins = reinterpret_cast<uint32_t*>(ws + l.joins);
  SortArgs sort{g.ids, nullptr, nullptr, reinterpret_cast<uint32_t*>(ws + l.counts), joins, g.T, (uint32_t)g.V, (int)tiles_of(g.T), 0};
  const dim3 sort_grid((unsigned)sort.tiles, (unsigned)g.m);
  const int out_size = g.out_dtype == OLSGD_F32 ? 4 : 2;
  ZeroArgs zero{g.dtable, g.V, g.D * out_size, g.dtable_worker * out_size, 0, 0};
  int64_t share = g.m * g.V * zero.row_bytes / (148 * 4);
  share = share < kZeroBytesMin ? kZeroBytesMin : share > kZeroBytesMax ? kZeroBytesMax : share;
  zero.rows = (int)(share / zero.row_bytes < kZeroRowsMax ? share / zero.row_bytes : kZeroRowsMax);
  if (zero.rows < 16) zero.rows = 16;
  zero.ctas = (int)((g.V + zero.rows - 1) / zero.rows);
  int passes = 0;
  while (g.T > 0 && (g.V >> (8 * passes)) > 0) ++passes;   // keys are 0 .. V
  if (sort.tiles > kSortCluster) {
    for (int p = 0; p < passes; ++p) {
      sort.shift = 8 * p;
      sort.out = lists[p & 1];
      cudaError_t e = launch_chained(sort_count_kernel, sort_grid, dim3(kSortThreads), 0, s, sort);
      if (e != cudaSuccess) return e;
      e = launch_chained(sort_place_kernel, sort_grid, dim3(kSortThreads), 0, s, sort);
      if (e != cudaSuccess) return e;
      sort.in = lists[p & 1];
    }
  } else if (passes > 0) {
    cudaLaunchConfig_t cfg{};
    const bool half = g.T <= kSortCluster * kSortTile / 2;
    if (half) sort.tiles = (int)((g.T + kSortTile / 2 - 1) / (kSortTile / 2));
    const int64_t zeros = (g.m * zero.ctas + sort.tiles - 1) / sort.tiles * sort.tiles;
    cfg.gridDim = dim3((unsigned)(g.m * sort.tiles + zeros));
    cfg.blockDim = dim3(kSortThreads);
    cfg.stream = s;
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)sort.tiles;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = g_launch_overlap ? 2 : 1;
    const cudaError_t e = cudaLaunchKernelEx(&cfg, half ? sort_cluster_kernel<kSortItems / 2> : sort_cluster_kernel<kSortItems>, sort, lists[0], lists[1], passes,
                                             (int)g.m, zero);
    if (e != cudaSuccess) return e;
    zero.ctas = 0;   // done
    sort.in = lists[(passes - 1) & 1];
  }
  SumArgs a;
  a.sorted = sort.in;
  a.dout = g.dout;
  a.dout_worker = g.dout_worker;
  a.dout_row = g.dout_row;
  a.dtable = g.dtable;
  a.out_worker = g.dtable_worker;
  a.part = reinterpret_cast<float*>(ws + l.part);
  a.joins = joins;
  a.join_list = joins + 64;
  a.T = g.T;
  a.V = g.V;
  a.D = g.D;
  a.pitch = pitch_of(g.D);
  a.chunks = (int)chunks_of(g.T);
  a.zero = zero;
  a.scale = g.scale;
  const int si = g.dtype == OLSGD_F32 ? 4 : 2;
  // whole pieces: the columns end on a piece's end too
  a.vec_in = g.D % kCols == 0 && rows_of_16(g.dout, g.dout_worker, g.dout_row, g.m, g.T, si);
  a.vec_out = g.D % kCols == 0 && rows_of_16(g.dtable, g.dtable_worker, g.D, g.m, g.V, out_size);
  switch (g.dtype) {
    case OLSGD_F32: return sum_rows_to<float>(g.out_dtype, a, g.m, s);
    case OLSGD_BF16: return sum_rows_to<__nv_bfloat16>(g.out_dtype, a, g.m, s);
    default: return sum_rows_to<__half>(g.out_dtype, a, g.m, s);
  }
}

}  // namespace olsgd
