// Per-worker gradient norm over many tensors, and clipping.
//
//   n_i = sqrt(sum over all tensors of worker i's g^2),  c_i = min(1, max_norm / (n_i + 1e-6)),
//   out = c_i g, rounded once to the output's type.
//
// Two launches bound by HBM: the first reads every gradient and leaves one partial sum per
// CTA, the second adds its worker's partial sums in a fixed order (every CTA for itself: a few
// hundred numbers), reads the gradients again and writes.  Sums are held in fp64 (eight
// squares of 16-bit values in fp32 first, where that is safe): no gradient of any type over- or
// underflows them, and the conversions hide behind the loads.
// The second kernel walks the tiles in the opposite order, so that what the first one read
// last is still in L2 when it is read again.  No atomics: the same bits every time.
//
// The tensors' descriptors travel as a kernel parameter, up to kMaxTensors per launch; a
// longer list takes more launches of each kernel.
#include "operator_common.cuh"
#include "operators_internal.h"

namespace olsgd {
namespace {

using namespace op;

constexpr int kThreads = 256;
constexpr int kUnroll = 8;                 // 16-byte loads a thread has in flight
constexpr int kCtasPerSm = 4;              // resident, and launched: a fifth in a second wave would run alone
constexpr int kTilePieces = kThreads * kUnroll;
constexpr int kMaxTensors = 256;
constexpr int64_t kKeepBytes = 80LL << 20;

struct Item {
  const void* in;
  void* out;
  int64_t n, in_stride, out_stride;   // elements per worker; elements between workers
  int64_t first_tile;                 // of this worker's tile list
  int32_t in_dtype, out_dtype;
};
// N: descriptors a launch has room for.  Short lists go with few, since the host copies the parameters
// several times with each launch (a call on one tensor takes 12.9 us of its time, 16.2 with room for
// all; on twenty, with room for kSomeTensors, 37 and 43; 48 and 49, either side of that, 78 and 82: from there on the
// descriptors themselves are what takes the time).
template <int N>
struct Items {
  int32_t count, pad;
  int64_t tiles;                      // per worker
  Item item[N];
};
constexpr int kFewTensors = 8, kSomeTensors = 48;
static_assert(sizeof(Items<kMaxTensors>) <= 32764 - 64, "kernel parameter space");

template <int N>
__device__ __forceinline__ int find_item(const Items<N>& it, int64_t tile) {
  int lo = 0, hi = it.count - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (it.item[mid].first_tile <= tile) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

// A tile's pieces of this thread; zeros past the row's ends.
template <typename T>
__device__ __forceinline__ void load_tile(const T* row, int64_t j0, int64_t n, bool again, uint4* w) {
  constexpr int V = Elem<T>::kVec;
  if (j0 >= 0 && j0 + ((kUnroll - 1) * kThreads + 1) * V <= n) {   // one address, constant distances
    const uint4* p = reinterpret_cast<const uint4*>(row + j0);
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) w[u] = again ? ld16(p + u * kThreads) : ld16_stream(p + u * kThreads);
  } else {
#pragma unroll
    for (int u = 0; u < kUnroll; ++u) w[u] = load_raw<T>(row, j0 + (int64_t)u * kThreads * V, n, 0);
  }
}

template <typename T>
__device__ __forceinline__ double tile_square_sum(const Item& it, int64_t worker, int64_t tile, bool again) {
  constexpr int V = Elem<T>::kVec;
  const T* row = static_cast<const T*>(it.in) + worker * it.in_stride;
  uint4 w[kUnroll];
  load_tile<T>(row, (tile * kTilePieces + threadIdx.x) * V - row_shift(row), it.n, again, w);
  double s = 0.0;
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    // Converting every element to fp64 would take longer than loading it.  Squares of 16-bit
    // values are exact in fp32 and eight of them are added there; where that sum leaves fp32's
    // comfortable range (or is zero) they are taken in fp64 after all.
    if constexpr (V == 8) {
      f32x2 p = raw_pair<T>(w[u], 0), q = mul2(p, p);
#pragma unroll
      for (int e = 1; e < 4; ++e) {
        p = raw_pair<T>(w[u], e);
        q = fma2(p, p, q);
      }
      float lo, hi;
      unpack2f(q, lo, hi);
      lo += hi;
      if (lo > 1e-20f && lo < 1e30f) {
        s += (double)lo;
        continue;
      }
    }
    float v[V];
    Elem<T>::unpack(w[u], v);
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const double d = (double)v[e];
      s = fma(d, d, s);
    }
  }
  return s;
}

__device__ __forceinline__ double block_sum(double s) {
  __shared__ double sh[kThreads / 32];
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = s;
  __syncthreads();
  double t = 0.0;
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) t += sh[w];
  return t;
}

// CTA (b, worker): tiles b, b + gridDim.x, ... of the worker's list.
template <int N>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
square_sum_kernel(const __grid_constant__ Items<N> it, double* __restrict__ part, int part_ld, int part_off) {
  launch_gate();
  const int64_t worker = blockIdx.y;
  // what the second kernel will find in L2: the last of what is read here, at normal priority
  const int64_t keep = kKeepBytes / (kTilePieces * 16) / gridDim.y;
  double s = 0.0;
  for (int64_t t = blockIdx.x; t < it.tiles; t += gridDim.x) {
    const Item& item = it.item[find_item(it, t)];
    const int64_t tile = t - item.first_tile;
    const bool again = t >= it.tiles - keep;
    if (item.in_dtype == OLSGD_F32) s += tile_square_sum<float>(item, worker, tile, again);
    else if (item.in_dtype == OLSGD_BF16) s += tile_square_sum<__nv_bfloat16>(item, worker, tile, again);
    else s += tile_square_sum<__half>(item, worker, tile, again);
  }
  s = block_sum(s);
  if (threadIdx.x == 0) part[worker * part_ld + part_off + blockIdx.x] = s;
}

template <typename TI, typename TO>
__device__ __forceinline__ void scale_tile(const Item& it, int64_t worker, int64_t tile, float c) {
  constexpr int V = Elem<TI>::kVec;
  const TI* row = static_cast<const TI*>(it.in) + worker * it.in_stride;
  TO* out = static_cast<TO*>(it.out) + worker * it.out_stride;
  const int shift = row_shift(row);
  // pieces start at elements j = -shift mod V; stores go out whole where such an element
  // lies on the boundary that a store of V elements needs
  constexpr int kStoreBytes = V * (int)sizeof(TO) < 16 ? V * (int)sizeof(TO) : 16;
  const bool aligned =
      ((reinterpret_cast<uintptr_t>(out) - (uintptr_t)shift * sizeof(TO)) & (kStoreBytes - 1)) == 0;
  const int64_t j0 = (tile * kTilePieces + threadIdx.x) * V - shift;
  uint4 w[kUnroll];
  load_tile<TI>(row, j0, it.n, false, w);
  const f32x2 cc = pack2f(c, c);
#pragma unroll
  for (int u = 0; u < kUnroll; ++u) {
    float v[V];
#pragma unroll
    for (int e = 0; e < V / 2; ++e) unpack2f(mul2(raw_pair<TI>(w[u], e), cc), v[2 * e], v[2 * e + 1]);
    store_floats<TO, V, true>(out, j0 + (int64_t)u * kThreads * V, it.n, aligned, v);
  }
}

template <typename TI>
__device__ __forceinline__ void scale_tile_to(const Item& it, int64_t worker, int64_t tile, float c) {
  if (it.out_dtype == OLSGD_F32) scale_tile<TI, float>(it, worker, tile, c);
  else if (it.out_dtype == OLSGD_BF16) scale_tile<TI, __nv_bfloat16>(it, worker, tile, c);
  else scale_tile<TI, __half>(it, worker, tile, c);
}

template <int N>
__global__ void __launch_bounds__(kThreads, kCtasPerSm)
clip_scale_kernel(const __grid_constant__ Items<N> it, const double* __restrict__ part, int part_ld, int n_part,
                  float max_norm, float* __restrict__ norms) {
  launch_gate();
  const int64_t worker = blockIdx.y;
  double s = 0.0;
  for (int i = threadIdx.x; i < n_part; i += kThreads) s += part[worker * part_ld + i];
  const double norm = sqrt(block_sum(s));
  if (norms && blockIdx.x == 0 && threadIdx.x == 0) norms[worker] = (float)norm;
  // NaN stays NaN (every comparison with it is false), an infinite norm gives 0
  const double ratio = (double)max_norm / (norm + 1e-6);
  const float c = ratio >= 1.0 ? 1.f : (float)ratio;
  for (int64_t b = blockIdx.x; b < it.tiles; b += gridDim.x) {
    const int64_t t = it.tiles - 1 - b;
    const Item& item = it.item[find_item(it, t)];
    // a gradient that is clipped in place and is short enough stays as it is
    if (c == 1.f && item.in == item.out && item.in_dtype == item.out_dtype && item.in_stride == item.out_stride) continue;
    const int64_t tile = t - item.first_tile;
    if (item.in_dtype == OLSGD_F32) scale_tile_to<float>(item, worker, tile, c);
    else if (item.in_dtype == OLSGD_BF16) scale_tile_to<__nv_bfloat16>(item, worker, tile, c);
    else scale_tile_to<__half>(item, worker, tile, c);
  }
}

int ctas_per_worker(int32_t m) {
  const int room = kCtasPerSm * 148;
  return m >= room ? 1 : room / m;
}

// Descriptors of tensors [first, first + count).
template <int N>
void fill(Items<N>& it, const olsgd_clip_tensor* t, int32_t first, int32_t count) {
  it.count = 0;
  it.pad = 0;
  it.tiles = 0;
  for (int32_t i = first; i < first + count; ++i) {
    if (t[i].n == 0) continue;
    const int vec = t[i].in_dtype == OLSGD_F32 ? 4 : 8;
    const int64_t pieces = (t[i].n + 2 * vec - 2) / vec;   // at any alignment of the rows
    it.item[it.count++] = Item{t[i].in, t[i].out, t[i].n, t[i].in_stride, t[i].out_stride, it.tiles,
                               t[i].in_dtype, t[i].out_dtype};
    it.tiles += (pieces + kTilePieces - 1) / kTilePieces;
  }
}

}  // namespace

// one partial sum per CTA and worker, for each launch over kMaxTensors tensors
size_t clip_workspace(int32_t m, int32_t n_tensors) {
  const int64_t launches = (n_tensors + kMaxTensors - 1) / kMaxTensors;
  return (size_t)m * ctas_per_worker(m) * (launches < 1 ? 1 : launches) * sizeof(double);
}

namespace {
template <int N>
cudaError_t clip(const olsgd_clip_tensor* t, int32_t n_tensors, int32_t m, float max_norm, float* norms, void* ws,
                 cudaStream_t s) {
  double* part = static_cast<double*>(ws);
  const int launches = n_tensors <= N ? 1 : (n_tensors + N - 1) / N;
  const int per = ctas_per_worker(m), part_ld = per * launches;
  Items<N> it;
  // every launch writes all of its `ctas` partial sums (zero where it has no tile); the grids
  // of a single launch are cut to the tiles there are
  int ctas = per;
  for (int l = 0; l < launches; ++l) {
    fill(it, t, l * N, n_tensors - l * N < N ? n_tensors - l * N : N);
    if (launches == 1) ctas = it.tiles < per ? (it.tiles < 1 ? 1 : (int)it.tiles) : per;
    const cudaError_t e = launch_chained(square_sum_kernel<N>, dim3((unsigned)ctas, (unsigned)m), dim3(kThreads), 0, s, it,
                                         part, part_ld, l * per);
    if (e != cudaSuccess) return e;
  }
  for (int l = 0; l < launches; ++l) {
    if (launches > 1)
      fill(it, t, l * N, n_tensors - l * N < N ? n_tensors - l * N : N);
    const cudaError_t e =
        launch_chained(clip_scale_kernel<N>, dim3((unsigned)ctas, (unsigned)m), dim3(kThreads), 0, s, it,
                       (const double*)part, part_ld, launches == 1 ? ctas : part_ld, max_norm, l == 0 ? norms : nullptr);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}
}  // namespace

cudaError_t launch_clip(const olsgd_clip_tensor* t, int32_t n_tensors, int32_t m, float max_norm, float* norms, void* ws,
                        cudaStream_t s) {
  if (n_tensors <= kFewTensors) return clip<kFewTensors>(t, n_tensors, m, max_norm, norms, ws, s);
  if (n_tensors <= kSomeTensors) return clip<kSomeTensors>(t, n_tensors, m, max_norm, norms, ws, s);
  return clip<kMaxTensors>(t, n_tensors, m, max_norm, norms, ws, s);
}

}  // namespace olsgd
