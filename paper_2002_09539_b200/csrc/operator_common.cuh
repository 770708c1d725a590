// What the operators on caller-owned tensors share: element types, 16-byte pieces of a row
// that need not start on a 16-byte boundary, packed arithmetic, warp reductions.
#pragma once

#include <cuda_fp16.h>

#include "olsgd_internal.h"

namespace olsgd {
namespace op {

constexpr float kLog2e = 1.4426950408889634f;

template <typename T>
struct Elem;
template <>
struct Elem<float> {
  static constexpr int kVec = 4;   // elements in 16 bytes
  static __device__ __forceinline__ float to_float(float v) { return v; }
  static __device__ __forceinline__ float from_float(float v) { return v; }
  static __device__ __forceinline__ void unpack(const uint4& w, float* v) {
    v[0] = __uint_as_float(w.x);
    v[1] = __uint_as_float(w.y);
    v[2] = __uint_as_float(w.z);
    v[3] = __uint_as_float(w.w);
  }
  static __device__ __forceinline__ uint4 pack(const float* v) {
    return make_uint4(__float_as_uint(v[0]), __float_as_uint(v[1]), __float_as_uint(v[2]),
                      __float_as_uint(v[3]));
  }
};
template <>
struct Elem<__nv_bfloat16> {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
  static __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
  static __device__ __forceinline__ void unpack(const uint4& w, float* v) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[2 * i] = __uint_as_float(u[i] << 16);
      v[2 * i + 1] = __uint_as_float(u[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ uint4 pack(const float* v) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 b = __floats2bfloat162_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&b);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
};
template <>
struct Elem<__half> {
  static constexpr int kVec = 8;
  static __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
  static __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }
  static __device__ __forceinline__ void unpack(const uint4& w, float* v) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
      v[2 * i] = f.x;
      v[2 * i + 1] = f.y;
    }
  }
  static __device__ __forceinline__ uint4 pack(const float* v) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
      u[i] = *reinterpret_cast<const uint32_t*>(&h);
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  }
};

// 16 bytes that are read once (no other thread wants the line): streaming load.
__device__ __forceinline__ uint4 ld16_stream(const void* p) { return __ldcs(static_cast<const uint4*>(p)); }
__device__ __forceinline__ uint4 ld16(const void* p) { return *static_cast<const uint4*>(p); }

// Elements by which p lies past a 16-byte boundary.  A row is walked in 16-byte pieces from
// the boundary at or before its first element: piece q holds the elements q * kVec - shift
// and up, and only the first and the last piece of a row can be partial.
template <typename T>
__host__ __device__ __forceinline__ int row_shift(const T* p) {
  return (int)((reinterpret_cast<uintptr_t>(p) & 15) / sizeof(T));
}

// The piece that starts at element j (j may be negative or reach past n): whole pieces with
// one 16-byte load, partial ones element by element; elements outside the row read as `fill`.
template <typename T>
__device__ __forceinline__ void load_piece(const T* row, int64_t j, int64_t n, float fill, float* v) {
  constexpr int V = Elem<T>::kVec;
  if (j >= 0 && j + V <= n) {
    Elem<T>::unpack(ld16_stream(row + j), v);
  } else {
#pragma unroll
    for (int e = 0; e < V; ++e) v[e] = (j + e >= 0 && j + e < n) ? Elem<T>::to_float(row[j + e]) : fill;
  }
}

// N floats to row[j ..], where the caller knows whether row + j starts on a boundary that
// whole pieces can be stored at; elements outside [0, n) are left alone.
template <typename T, int N>
__device__ __forceinline__ void store_floats(T* row, int64_t j, int64_t n, bool aligned, const float* v) {
  constexpr int V = Elem<T>::kVec;
  if (aligned && j >= 0 && j + N <= n) {
    if constexpr (N >= V) {
#pragma unroll
      for (int q = 0; q < N / V; ++q) reinterpret_cast<uint4*>(row + j)[q] = Elem<T>::pack(v + q * V);
    } else {
      float w[V];
#pragma unroll
      for (int e = 0; e < V; ++e) w[e] = e < N ? v[e] : 0.f;
      const uint4 p = Elem<T>::pack(w);
      *reinterpret_cast<uint2*>(row + j) = make_uint2(p.x, p.y);   // N == V / 2: 8 bytes
    }
  } else {
#pragma unroll
    for (int e = 0; e < N; ++e)
      if (j + e >= 0 && j + e < n) row[j + e] = Elem<T>::from_float(v[e]);
  }
}

// Maximum that keeps a NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}
__device__ __forceinline__ float ex2(float v) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

}  // namespace op
}  // namespace olsgd
