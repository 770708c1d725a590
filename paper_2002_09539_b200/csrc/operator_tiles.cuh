// What the tensor-core operators on caller-owned tensors share: accumulators on their way from tensor
// memory to rows of any alignment, copies of operands whose rows TMA cannot take, tensor maps of 16-bit
// operands.  (In an unnamed namespace: each file that includes this has its own kernel.)
#pragma once

#include "operator_common.cuh"
#include "operators_internal.h"
#include "tc_common.cuh"

namespace olsgd {
namespace {

using namespace tc;
using namespace op;

constexpr int kEpiWarps = 8;

__device__ __forceinline__ void tmem_ld16x2(uint32_t ta, uint32_t tb, float* a, float* b) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(ta)
      : "memory");
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(tb)
      : "memory");
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int j = 0; j < 16; ++j) {
    a[j] = __uint_as_float(r[j]);
    b[j] = __uint_as_float(r[16 + j]);
  }
}

__device__ __forceinline__ uint32_t pack2(float lo, float hi, int f16) {
  if (f16) {
    const __half2 h = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&h);
  }
  const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&b);
}

// Predicated stores: in the epilogue a branch around a store costs more than the store.
__device__ __forceinline__ void store_sector_if(float* p, const float* v, bool yes) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %9, 0;\n\t@q st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n\t}" ::"l"(p),
               "r"(__float_as_uint(v[0])), "r"(__float_as_uint(v[1])), "r"(__float_as_uint(v[2])), "r"(__float_as_uint(v[3])),
               "r"(__float_as_uint(v[4])), "r"(__float_as_uint(v[5])), "r"(__float_as_uint(v[6])), "r"(__float_as_uint(v[7])), "r"((int)yes)
               : "memory");
}
__device__ __forceinline__ void store_piece_if(void* p, const uint4& v, bool yes) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %5, 0;\n\t@q st.global.v4.b32 [%0], {%1, %2, %3, %4};\n\t}" ::"l"(p), "r"(v.x),
               "r"(v.y), "r"(v.z), "r"(v.w), "r"((int)yes)
               : "memory");
}

__device__ __forceinline__ void store_word_if(uint16_t* p, uint32_t v, bool yes) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q st.global.b32 [%0], %1;\n\t}" ::"l"(p), "r"(v), "r"((int)yes)
               : "memory");
}
__device__ __forceinline__ void store_half_if(uint16_t* p, uint32_t v, bool yes) {
  asm volatile("{\n\t.reg .pred q;\n\tsetp.ne.b32 q, %2, 0;\n\t@q st.global.b16 [%0], %1;\n\t}" ::"l"(p), "h"((uint16_t)v),
               "r"((int)yes)
               : "memory");
}

// A warp's block of 32 rows x W columns of results on its way out: TMEM hands every lane a row,
// memory wants whole lines.  16-byte pieces, swizzled so that neither side meets bank conflicts
// (W = 64).
template <int W>
struct Staged {
  static constexpr int kPieces = W / 8;   // 16-byte pieces of a row
  uint4* buf;
  __device__ __forceinline__ static int at(int row, int piece) { return row * kPieces + (piece ^ (row & (kPieces - 1))); }
  // 16 values of this lane's row, from column 16 q of the block on
  __device__ __forceinline__ void put(int lane, int q, const float* v, int f16, float scale = 1.f) {
    uint32_t p[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) p[j] = pack2(v[2 * j] * scale, v[2 * j + 1] * scale, f16);
    buf[at(lane, 2 * q)] = make_uint4(p[0], p[1], p[2], p[3]);
    buf[at(lane, 2 * q + 1)] = make_uint4(p[4], p[5], p[6], p[7]);
  }
  // The block to rows [0, rows) of dst (row pitch ld elements), of whose columns `cols` exist.  width:
  // bytes that dst, ld and cols are multiples of (16, 8, 4 or 2).
  __device__ __forceinline__ void flush(int lane, uint16_t* dst, int64_t ld, int64_t rows, int64_t cols, int width) {
    __syncwarp();
    const int n = rows < 32 ? (int)rows : 32, nc = cols < W ? (int)cols : W;
    if (width == 16) {
      // (all reads ahead of the stores, which the compiler does not move them across)
      uint4 v[kPieces];
#pragma unroll
      for (int i = 0; i < kPieces; ++i) v[i] = buf[at((i * 32 + lane) / kPieces, (i * 32 + lane) % kPieces)];
#pragma unroll
      for (int i = 0; i < kPieces; ++i) {
        const int k = i * 32 + lane, r = k / kPieces, c = k % kPieces;
        store_piece_if(dst + r * ld + c * 8, v[i], r < n && c * 8 < nc);
      }
    } else {
      flush_narrow(buf, lane, dst, ld, n, nc, width);
    }
    __syncwarp();
  }
  __device__ __forceinline__ static void flush_narrow(const uint4* buf, int lane, uint16_t* dst, int64_t ld, int n, int nc, int width) {
    if (width == 8) {
      const uint2* half = reinterpret_cast<const uint2*>(buf);
#pragma unroll
      for (int i = 0; i < 2 * kPieces; ++i) {
        const int k = i * 32 + lane, r = k / (2 * kPieces), c = k % (2 * kPieces);
        const uint2 v = half[at(r, c >> 1) * 2 + (c & 1)];
        if (r < n && c * 4 < nc) *reinterpret_cast<uint2*>(dst + r * ld + c * 4) = v;
      }
    } else {
      // Two columns a lane, one word of the block.  Rows of an odd pitch start between the words every
      // other time: there a lane stores its second column with the next lane's first, and the block's
      // first and last column go by themselves.
      const uint32_t* words = reinterpret_cast<const uint32_t*>(buf);
      constexpr int kPairs = W / 2, kRows = 32 / kPairs;   // rows a step
      const int pair = lane % kPairs;
      int r = lane / kPairs;
      uint16_t* row = dst + r * ld;
      constexpr int U = 8;
#pragma unroll 1
      for (int step = 0; step < 32 / kRows; step += U) {
        uint32_t w[U], next[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          w[u] = words[at(r + u * kRows, pair >> 2) * 4 + (pair & 3)];
          next[u] = __shfl_down_sync(0xffffffffu, w[u], 1);
        }
#pragma unroll
        for (int u = 0; u < U; ++u, r += kRows, row += kRows * ld) {
          const int odd = (int)(reinterpret_cast<uintptr_t>(row) >> 1) & 1, c = 2 * pair + odd;
          const uint32_t v = odd ? __funnelshift_r(w[u], next[u], 16) : w[u];
          store_word_if(row + c, v, r < n && c + 1 < nc);
          store_half_if(row + c, v, r < n && c + 1 == nc);
          store_half_if(row, w[u], r < n && odd && pair == 0);   // (a block has a column)
        }
      }
    }
  }
};

// The same for fp32 sums: 32 rows x COLS (16 or 32) columns, straight from tensor memory to rows of
// dst (pitch ld, a multiple of 8) of which `cols` columns (a multiple of 8) exist.  Lanes that stored
// their own rows would keep the store unit busy with one sector each.
template <int COLS>
__device__ __forceinline__ void spill_sums(uint4* buf, int lane, uint32_t acc, float* dst, int64_t ld, int64_t rows, int64_t cols) {
  constexpr int kPieces = COLS / 4;
  const auto at = [](int row, int piece) { return row * kPieces + (piece ^ (row & (kPieces - 1))); };
  float v[32];
  tmem_ld16x2(acc, COLS == 32 ? acc + 16 : acc, v, v + 16);
#pragma unroll
  for (int q = 0; q < kPieces; ++q) buf[at(lane, q)] = Elem<float>::pack(v + 4 * q);
  __syncwarp();
  uint4 w[kPieces];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) w[i] = buf[at((i * 32 + lane) / kPieces, (i * 32 + lane) % kPieces)];
#pragma unroll
  for (int i = 0; i < kPieces; ++i) {
    const int k = i * 32 + lane, r = k / kPieces, c = k % kPieces;
    store_piece_if(dst + r * ld + c * 4, w[i], r < rows && c * 4 < cols);
  }
  __syncwarp();
}

// Arrives on the barrier at this offset in the pair's leader.  What it orders are this warp's reads
// of tensor memory, which have completed (tcgen05.wait::ld): no cluster-wide release, which
// would wait for the results on their way to global memory too (3 us a tile).
__device__ __forceinline__ void arrive_leader(uint32_t bar) {
  uint32_t remote;
  asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(remote) : "r"(bar));
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(remote) : "memory");
}

// Rows of any pitch to rows of a pitch that TMA takes: up to three operands [m][rows][cols] of
// 16-bit values, one after another in the grid; a warp per row.  A lane makes one aligned 16-byte piece out
// of the two that its elements lie in (`begin` and `end` bound the tensor: nothing outside it is
// read).
struct PadOperand {
  const uint16_t *begin, *end;
  uint16_t* out;
  int64_t rows, workers, in_worker, in_row;   // rows of a worker
  int64_t cols, pitch, first;                 // pitch of the copies, zeros behind cols; first: block
};
struct PadOperands {
  PadOperand op[3];
  int count;
};
__global__ void __launch_bounds__(256) pad_rows_kernel(const __grid_constant__ PadOperands all) {
  launch_gate();
  int which = 0;
  while (which + 1 < all.count && blockIdx.x >= all.op[which + 1].first) ++which;
  const PadOperand& o = all.op[which];
  const int lane = threadIdx.x & 31;
  const int64_t at = (blockIdx.x - o.first) * 8 + (threadIdx.x >> 5), worker = at / o.rows, r = at - worker * o.rows;
  if (worker >= o.workers) return;
  const int cols = (int)o.cols, whole = cols / 8, pieces = (int)(o.pitch / 8);
  const uint16_t* src = o.begin + worker * o.in_worker + r * o.in_row;
  uint4* dst = reinterpret_cast<uint4*>(o.out) + at * pieces;
  const int off = (int)((reinterpret_cast<uintptr_t>(src) & 15) / 2);
  int first_slow = 0;   // pieces from here on are made element by element
  if (src - off >= o.begin && src - off + whole * 8 + 8 <= o.end) {
    // every whole piece of the row, and its neighbour, lie inside the tensor
    first_slow = whole;
    const uint4* base = reinterpret_cast<const uint4*>(src - off);
    constexpr int U = 4;
    for (int p0 = lane; p0 < whole; p0 += 32 * U) {
      uint4 a[U], b[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int p = min(p0 + u * 32, whole - 1);
        a[u] = base[p];
        b[u] = base[p + 1];
      }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (p0 + u * 32 < whole) dst[p0 + u * 32] = eight_from(a[u], b[u], off);
    }
  }
  for (int p = first_slow + lane; p < pieces; p += 32) {
    uint32_t w[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const int j = p * 8 + 2 * e;
      const uint32_t lo = j < cols ? src[j] : 0, hi = j + 1 < cols ? src[j + 1] : 0;
      w[e] = lo | (hi << 16);
    }
    dst[p] = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

// --------------------------------------------------------------------------------- host
constexpr int64_t round8(int64_t v) { return (v + 7) / 8 * 8; }
constexpr size_t round256(size_t v) { return (v + 255) / 256 * 256; }

// [m][rows][cols] 16-bit, cols contiguous; boxes of 64 columns by box_rows rows.
bool make_map16(CUtensorMap* map, const GatedOperand& o, int64_t cols, int64_t rows, int64_t m, int box_rows, bool f16) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const int64_t worker = m > 1 ? o.worker_stride : round8(cols) * rows;
  const int64_t row = rows > 1 ? o.row_stride : round8(cols);
  cuuint64_t dims[3] = {(cuuint64_t)cols, (cuuint64_t)rows, (cuuint64_t)m};
  cuuint64_t strides[2] = {(cuuint64_t)row * 2, (cuuint64_t)worker * 2};
  cuuint32_t box[3] = {(cuuint32_t)kBK, (cuuint32_t)box_rows, 1};
  cuuint32_t estr[3] = {1, 1, 1};
  return fn(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(o.p), dims,
            strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

bool tma_ready(const GatedOperand& o, int64_t rows, int64_t m) {
  return (reinterpret_cast<uintptr_t>(o.p) & 15) == 0 && (rows == 1 || o.row_stride % 8 == 0) &&
         (m == 1 || o.worker_stride % 8 == 0);
}

// Replaces those of the operands [m][rows][cols] that TMA cannot take by copies in rows of
// round8(cols) from ws on; says whether there were any.
struct Wanted {
  GatedOperand* o;
  int64_t rows;
};
// Copies of a call, made by one launch.
struct Pads {
  PadOperands all{};
  int64_t blocks = 0;
  void add(const void* begin, int64_t workers, int64_t worker_stride, int64_t rows, int64_t row_stride, int64_t cols, int64_t pitch,
           uint8_t* dst) {
    const uint16_t* p = static_cast<const uint16_t*>(begin);
    const uint16_t* end = p + (workers > 1 ? (workers - 1) * worker_stride : 0) + (rows > 1 ? (rows - 1) * row_stride : 0) + cols;
    all.op[all.count++] = PadOperand{p, end, reinterpret_cast<uint16_t*>(dst), rows, workers, worker_stride, row_stride, cols, pitch, blocks};
    blocks += (rows * workers + 7) / 8;
  }
  cudaError_t launch(cudaStream_t s) const {
    return all.count == 0 ? cudaSuccess : launch_chained(pad_rows_kernel, dim3((unsigned)blocks), dim3(256), 0, s, all);
  }
};
void make_ready(Pads& pads, const Wanted* wanted, int count, int64_t cols, int64_t pitch, int64_t m, uint8_t* ws) {
  for (int i = 0; i < count; ++i) {
    GatedOperand& o = *wanted[i].o;
    const int64_t rows = wanted[i].rows;
    if (tma_ready(o, rows, m)) continue;
    pads.add(o.p, m, o.worker_stride, rows, o.row_stride, cols, pitch, ws);
    o = GatedOperand{ws, rows * pitch, pitch};
    ws += round256((size_t)m * rows * pitch * 2);
  }
}
cudaError_t make_ready(const Wanted* wanted, int count, int64_t cols, int64_t m, uint8_t* ws, cudaStream_t s, bool* any = nullptr) {
  Pads pads;
  make_ready(pads, wanted, count, cols, round8(cols), m, ws);
  if (any) *any = pads.all.count > 0;
  return pads.launch(s);
}

int store_width(const void* p, int64_t cols) {
  const uintptr_t bits = reinterpret_cast<uintptr_t>(p) | (uintptr_t)(cols * 2);
  return bits % 16 == 0 ? 16 : bits % 8 == 0 ? 8 : bits % 4 == 0 ? 4 : 2;
}

}  // namespace
}  // namespace olsgd
