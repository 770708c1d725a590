// What the operators on caller-owned tensors share: element types, 16-byte pieces of a row
// that need not start on a 16-byte boundary, packed arithmetic, warp reductions.
#pragma once

#include <cuda_fp16.h>

#include <type_traits>

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
// ONCE: results that nothing reads soon; their lines are the first that L2 gives up.
template <typename T, int N, bool ONCE = false>
__device__ __forceinline__ void store_floats(T* row, int64_t j, int64_t n, bool aligned, const float* v) {
  constexpr int V = Elem<T>::kVec;
  if (aligned && j >= 0 && j + N <= n) {
    if constexpr (N * sizeof(T) == 32) {
      // one 32-byte store (a whole sector) where the address allows it
      if ((reinterpret_cast<uintptr_t>(row + j) & 31) == 0) {
        const uint4 a = Elem<T>::pack(v), b = Elem<T>::pack(v + V);
        if constexpr (ONCE)
          asm volatile("st.global.cs.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(row + j), "r"(a.x), "r"(a.y),
                       "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                       : "memory");
        else
          asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(row + j), "r"(a.x), "r"(a.y),
                       "r"(a.z), "r"(a.w), "r"(b.x), "r"(b.y), "r"(b.z), "r"(b.w)
                       : "memory");
        return;
      }
    }
    if constexpr (N >= V) {
#pragma unroll
      for (int q = 0; q < N / V; ++q) {
        if constexpr (ONCE) __stcs(reinterpret_cast<uint4*>(row + j) + q, Elem<T>::pack(v + q * V));
        else reinterpret_cast<uint4*>(row + j)[q] = Elem<T>::pack(v + q * V);
      }
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

// Two floats in one register pair: Blackwell's packed fp32 arithmetic.
typedef uint64_t f32x2;
__device__ __forceinline__ f32x2 pack2f(float lo, float hi) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpack2f(f32x2 v, float& lo, float& hi) {
  asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v));
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// The piece that starts at element j as it lies in memory; elements outside [0, n) are `fill`
// (the bits of one element).
template <typename T, typename Index>
__device__ __forceinline__ uint4 load_raw(const T* row, Index j, Index n, uint32_t fill) {
  constexpr int V = Elem<T>::kVec;
  if (j >= 0 && j + V <= n) return ld16_stream(row + j);
  uint32_t w[4];
  if constexpr (V == 4) {
#pragma unroll
    for (int e = 0; e < 4; ++e) w[e] = (j + e >= 0 && j + e < n) ? reinterpret_cast<const uint32_t*>(row)[j + e] : fill;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const Index k = j + 2 * e;
      const uint32_t lo = (k >= 0 && k < n) ? reinterpret_cast<const uint16_t*>(row)[k] : fill;
      const uint32_t hi = (k + 1 >= 0 && k + 1 < n) ? reinterpret_cast<const uint16_t*>(row)[k + 1] : fill;
      w[e] = lo | (hi << 16);
    }
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
// Elements 2 i and 2 i + 1 of a piece.
template <typename T>
__device__ __forceinline__ f32x2 raw_pair(const uint4& w, int i) {
  const uint32_t u[4] = {w.x, w.y, w.z, w.w};
  if constexpr (sizeof(T) == 4) {
    return pack2f(__uint_as_float(u[2 * i]), __uint_as_float(u[2 * i + 1]));
  } else if constexpr (std::is_same<T, __half>::value) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&u[i]));
    return pack2f(f.x, f.y);
  } else {
    return pack2f(__uint_as_float(u[i] << 16), __uint_as_float(u[i] & 0xFFFF0000u));
  }
}
// The largest element of a piece; KEEP_NAN: NaN if there is one (else it is passed over).
template <typename T, bool KEEP_NAN>
__device__ __forceinline__ float raw_max(const uint4& w) {
  if constexpr (sizeof(T) == 4) {
    const float a = __uint_as_float(w.x), b = __uint_as_float(w.y), c = __uint_as_float(w.z), d = __uint_as_float(w.w);
    if constexpr (KEEP_NAN) return max_nan(max_nan(a, b), max_nan(c, d));
    else return fmaxf(fmaxf(a, b), fmaxf(c, d));
  } else if constexpr (std::is_same<T, __half>::value) {
    const __half2* h = reinterpret_cast<const __half2*>(&w);
    const __half2 m = KEEP_NAN ? __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]))
                               : __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    const float2 f = __half22float2(m);
    return KEEP_NAN ? max_nan(f.x, f.y) : fmaxf(f.x, f.y);
  } else {
    const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&w);
    const __nv_bfloat162 m = KEEP_NAN ? __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]))
                                      : __hmax2(__hmax2(h[0], h[1]), __hmax2(h[2], h[3]));
    const float2 f = __bfloat1622float2(m);
    return KEEP_NAN ? max_nan(f.x, f.y) : fmaxf(f.x, f.y);
  }
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
