// Products grouped by expert on the fifth-generation tensor cores, worker-batched.  Rows
// offsets[e] .. offsets[e + 1] - 1 of a worker belong to its expert e:
//   y_r = W_e x_r           (forward)        x [m][R][D], W [m][E][F][D], y [m][R][F]
//   dx_r = W_e^T dy_r,  dW_e = sum over the expert's rows of dy_r x_r^T      (backward)
// 16-bit operands, fp32 accumulation in tensor memory, one rounding of each result.
//
// The sizes of the groups are known to the GPU alone.  The kernel is persistent; each CTA turns the offsets into a table
// of row tiles in its shared memory first.
//
// One kernel, three modes.  Warp 0 feeds a ring of shared-memory stages with TMA, warp 1 issues the MMAs into
// accumulators in tensor memory, eight warps empty them.  A tile has 128 features, or 256 as two MMAs that share their B
// (HALVES = 2); two accumulators take turns.  A tile of 256 x 256, for which a CTA takes in 64 KB a
// 256 x 256 x 64 multiply-adds, which L2 keeps up with, fills tensor memory: its halves are emptied one by one while the
// next tile's first MMAs run.
//   FORWARD   A = W (K-major), B = the tile's rows of x (K-major)
//   DX        A = W read along D (MN-major), B = the tile's rows of dy
//   DW        A = dy, B = x, both read along their features (MN-major), K = the group's rows
// The weights are the MMA's M, so that the ragged dimension is its N: a tile of n rows costs n rounded
// up to 16, not to 128, in MMAs and in loads.  Rows of other groups that come
// with a box end up in columns of the accumulator that are not stored.  Along K they would be
// summed: there the warp that issues the MMAs zeroes them in shared memory first (up to 15 rows of a group's last block).
//
// Bound by the weights' way from memory where there are few rows (16 rows, 64 experts, 1024 -> 2048 bf16: 67 MB at
// most in 12.8 us, 17 with cold caches), by the GPU's power where there are many (32768 rows, 8 experts, 2048 -> 4096 bf16: 382,
// 372 and 400 us, 1.37 to 1.48 PFLOP/s).  In between by the operands' way in and, for weights' gradients, the results' way
// out (16 workers x 512 rows, 4 experts, 1024 -> 1024 bf16: 39, 38 and 44 us for 168 MB each, 4.3 TB/s).
//
// TMA wants 16-byte row pitches: operands that do not have them are copied to padded rows in
// the workspace first (3 x 1001 rows, 11 experts, 1021 -> 515: 12 to 13 us beside products of 17, 19 and 28).  Every wait is bounded, as in the library's other tensor-core kernels.
#include <cmath>

#include "operator_tiles.cuh"

namespace olsgd {
namespace {

enum Mode { FORWARD = 0, DX = 1, DW = 2 };
constexpr int kGroup = 8;            // DW: row tiles walked together (operand reuse in L2)
constexpr int kSmallBox = 16;        // rows of a box of B where a tile is not full; K of an MMA
constexpr int kMaxGroups = 1024;     // of a launch of FORWARD or DX: its table's room
constexpr int kMaxStarts = 2 * kMaxGroups;

// Rows come in boxes of 16, 32, 64, 128 and 256, one of each at most (a TMA instruction takes some 200 cycles however
// small its box is).  DW: boxes of 16, 32 and 64 rows by 64 columns; or, of operands whose rows are made of whole panels of 64
// columns, one of 64 rows by all the panels of the tile (rows behind the group's reach no MMA, or are zeroed).
constexpr int kBoxes = 5, kPanels = 3;
struct alignas(64) ProductMaps {
  CUtensorMap a[kBoxes], b[kBoxes];   // FORWARD, DX: a[0] are the weights; DW: [kPanels] the operand by panels
};
struct ProductArgs {
  int num_kb, k_extent;       // FORWARD, DX: K in blocks of 64, and in elements
  int m_tiles, n_tiles;       // tiles of the features; DW: and of the columns
  int features, cols;         // rows of A in all; DW: columns of the output
  int R, E, m, first_worker;  // rows and experts of a worker; workers of this launch
  int f16;
  int a_panels, b_panels;     // DW: the operand goes by panels
  int beside;                 // runs beside the kernel ahead of it: see launch_product_backward
  int out_width;              // bytes (16, 8, 4, 2) that the output's base and rows are multiples of
  const int32_t* offsets;     // [workers][E + 1]
  void* out;
  int* status;                // status_word()
  // K by parts, where the tiles are few: `splits` units for a tile, whose sums go to parts[split][...] in fp32 (rows of
  // features; DW: [group][column][feature]), part_size values each, for join_kernel
  int splits;
  float* parts;
  int64_t part_size;
};

template <int STAGES>
struct Control {
  uint64_t full[STAGES], empty[STAGES];
  uint64_t acc_full[2], acc_empty[2];
  uint64_t last;             // MMAs in flight when a wait gave up
  uint32_t tmem_base;
  int abort_flag;
};
// FORWARD, DX: where the rows of each expert begin, [m][E + 1], and the first row tile of each group.
struct Table {
  int32_t start[kMaxStarts];
  int32_t first[kMaxGroups + 1];
  int32_t sums[kThreads / 32];
};

// ------------------------------------------------------------------------------- products
// By a whole CTA.  Offsets that fall, or leave [0, R], are taken as the largest so far, so that groups never overlap.
__device__ __forceinline__ void make_table(const ProductArgs& g, Table& tb, int bn) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, width = g.E + 1, groups = g.m * g.E;
  for (int w = warp; w < g.m; w += kThreads / 32) {
    int most = 0;
    for (int e0 = 0; e0 < width; e0 += 32) {
      int v = e0 + lane < width ? min(max(g.offsets[(int64_t)(g.first_worker + w) * width + e0 + lane], 0), g.R) : 0;
      v = max(v, most);
#pragma unroll
      for (int off = 1; off < 32; off <<= 1) {
        const int up = __shfl_up_sync(0xffffffffu, v, off);
        if (lane >= off) v = max(v, up);
      }
      if (e0 + lane < width) tb.start[w * width + e0 + lane] = v;
      most = __shfl_sync(0xffffffffu, v, 31);
    }
  }
  __syncthreads();
  const auto tiles_of = [&](int i) {
    const int32_t* s = tb.start + i + i / g.E;
    return (s[1] - s[0] + bn - 1) / bn;
  };
  const int per = (groups + kThreads - 1) / kThreads, begin = min(groups, (int)threadIdx.x * per), end = min(groups, begin + per);
  int mine = 0;
  for (int i = begin; i < end; ++i) mine += tiles_of(i);
  int scan = mine;
#pragma unroll
  for (int off = 1; off < 32; off <<= 1) {
    const int up = __shfl_up_sync(0xffffffffu, scan, off);
    if (lane >= off) scan += up;
  }
  if (lane == 31) tb.sums[warp] = scan;
  __syncthreads();
  int before = scan - mine;
  for (int w = 0; w < warp; ++w) before += tb.sums[w];
  for (int i = begin; i < end; ++i) {
    tb.first[i] = before;
    before += tiles_of(i);
  }
  if (threadIdx.x == kThreads - 1) tb.first[groups] = before;
  __syncthreads();
}

// One lane of a whole warp.  (Of lanes chosen this way the compiler knows that they are one: operands of TMA and MMA
// instructions stay in uniform registers.  193 cycles a block of 64 along K, 160 a copy and 100 an MMA where lane 0 was asked for.)
__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}

// Of the weights: [m][E][F][D].
__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, uint32_t bar, int c0, int c1, int c2, int c3) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes"
      " [%0], [%1, {%3, %4, %5, %6}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(c0), "r"(c1), "r"(c2), "r"(c3)
      : "memory");
}

// A unit of work, and a role's walk over them.
struct Unit {
  int worker, group;     // DW: group of the worker's and all before it; FORWARD, DX: expert of the worker
  int m, col;            // feature tile; DW: column tile
  int row0, n;           // rows (FORWARD, DX: the tile's, DW: the group's)
  int split, kb, end;    // blocks of K
};
template <int MODE, int BN>
struct Walk {
  const ProductArgs& g;
  const Table& tb;
  uint32_t total, step;
  int at_group = 0;
  // DW: the offsets of the next unit's group, on their way while this unit is worked at (each unit would wait for L2 first)
  int2 ahead;
  uint32_t ahead_group = 0, ahead_worker = 0, ahead_tile = 0;
  bool has_ahead = false;
  __device__ __forceinline__ Walk(const ProductArgs& args, const Table& table, uint32_t by) : g(args), tb(table), step(by) {
    total = (MODE == DW ? (uint32_t)(g.m * g.E) * g.m_tiles * g.n_tiles : (uint32_t)tb.first[g.m * g.E] * g.m_tiles) * g.splits;
  }
  // DW: unit t's group, worker, place in the group, and offsets
  __device__ __forceinline__ void look(uint32_t t) {
    const uint32_t per = (uint32_t)g.m_tiles * g.n_tiles * g.splits;
    ahead_group = t / per;
    ahead_tile = t - ahead_group * per;
    ahead_worker = ahead_group / g.E;
    const int32_t* o = g.offsets + ahead_group + ahead_worker;   // (a worker has E + 1 of them)
    ahead = make_int2(__ldcg(o), __ldcg(o + 1));                 // (past L1: DW may run beside its predecessor)
  }
  // t: `step` more than at the call before
  __device__ __forceinline__ Unit at(uint32_t t) {
    Unit u;
    u.split = 0;
    if (MODE == DW) {
      if (!has_ahead) look(t);
      u.group = ahead_group;
      u.worker = ahead_worker;
      uint32_t i = ahead_tile;
      if (g.splits > 1) {
        const uint32_t tile = i / g.splits;
        u.split = i - tile * g.splits;
        i = tile;
      }
      const int2 r = ahead;
      has_ahead = t + step < total;
      if (has_ahead) look(t + step);
      const uint32_t group_tiles = kGroup * g.n_tiles, block = i / group_tiles, first = block * kGroup;
      const uint32_t height = min((uint32_t)kGroup, g.m_tiles - first), j = i - block * group_tiles;
      u.col = height == kGroup ? j / kGroup : j / height;
      u.m = first + j - u.col * height;
      // (whatever the offsets hold)
      u.row0 = min(max(r.x, 0), g.R);
      u.n = min(max(r.y, u.row0), g.R) - u.row0;
    } else {
      if (g.splits > 1) {
        u.split = t % g.splits;
        t /= g.splits;
      }
      const int i = t / g.m_tiles;
      while (tb.first[at_group + 1] <= i) ++at_group;
      const int worker = at_group / g.E;
      const int32_t* s = tb.start + at_group + worker;
      u.row0 = s[0] + (i - tb.first[at_group]) * BN;
      u.n = min(BN, s[1] - u.row0);
      u.worker = g.first_worker + worker;
      u.group = at_group - worker * g.E;
      u.m = t - i * g.m_tiles;
      u.col = 0;
    }
    const int blocks = MODE == DW ? (u.n + kBK - 1) / kBK : g.num_kb;
    u.kb = 0;
    u.end = blocks;
    if (g.splits > 1) {
      u.kb = (int)((int64_t)blocks * u.split / g.splits);
      u.end = (int)((int64_t)blocks * (u.split + 1) / g.splits);
    }
    return u;
  }
};

// 32 accumulator columns of this lane's feature, rows row .. row + 31 of the output, of which n exist: a row's 32 features
// leave by one store of 64 bytes.  For outputs whose rows are not multiples of 16 bytes.
__device__ __forceinline__ void store_rows(const float* v, uint16_t* dst, int64_t pitch, int n, bool live, int f16) {
#pragma unroll
  for (int j = 0; j < 32; j += 2) {
    const uint32_t two = pack2(v[j], v[j + 1], f16);
    store_half_if(dst + j * pitch, two, live && j < n);
    store_half_if(dst + (j + 1) * pitch, two >> 16, live && j + 1 < n);
  }
}

// 32 or 64 columns of this lane's row of tensor memory.
template <int W>
__device__ __forceinline__ void tmem_ld_wide(uint32_t taddr, float* v) {
  static_assert(W == 32 || W == 64, "");
  uint32_t r[W];
#pragma unroll
  for (int c = 0; c < W; c += 32) {
    uint32_t* p = r + c;
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
        : "=r"(p[0]), "=r"(p[1]), "=r"(p[2]), "=r"(p[3]), "=r"(p[4]), "=r"(p[5]), "=r"(p[6]), "=r"(p[7]), "=r"(p[8]), "=r"(p[9]), "=r"(p[10]),
          "=r"(p[11]), "=r"(p[12]), "=r"(p[13]), "=r"(p[14]), "=r"(p[15]), "=r"(p[16]), "=r"(p[17]), "=r"(p[18]), "=r"(p[19]), "=r"(p[20]),
          "=r"(p[21]), "=r"(p[22]), "=r"(p[23]), "=r"(p[24]), "=r"(p[25]), "=r"(p[26]), "=r"(p[27]), "=r"(p[28]), "=r"(p[29]), "=r"(p[30]),
          "=r"(p[31])
        : "r"(taddr + c)
        : "memory");
  }
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
  for (int k = 0; k < W; ++k) v[k] = __uint_as_float(r[k]);
}

// 16 lanes x (8 BLOCKS) columns of tensor memory, as the fragments of 8 x 8 matrices: of block i, v[4 i] and v[4 i + 1] are
// row lane / 4, columns 2 (lane % 4) and the next, v[4 i + 2] and v[4 i + 3] eight rows below.
template <int BLOCKS>
__device__ __forceinline__ void tmem_ld_fragments(uint32_t taddr, uint32_t* r) {
  static_assert(BLOCKS == 2 || BLOCKS == 4, "");
  if constexpr (BLOCKS == 4) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]),
          "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
        : "r"(taddr)
        : "memory");
  } else {
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
  }
}
// 8 BLOCKS accumulator columns (rows of the output) of a warp's 32 features, to rows of dst, of which n rows and `features`
// features (a multiple of 8) exist.  The accumulator has the features in its lanes, memory wants them side by side:
// fragments are stored transposed (stmatrix), 8 x 8 values an instruction and matrix, and leave by 16 bytes a lane.
template <int BLOCKS>
__device__ __forceinline__ void store_transposed(uint8_t* buf, int lane, uint32_t acc, uint16_t* dst, int64_t pitch, int n, int features, int f16) {
  uint32_t lo[4 * BLOCKS], hi[4 * BLOCKS];   // features 0 .. 15 and 16 .. 31
  tmem_ld_fragments<BLOCKS>(acc, lo);
  tmem_ld_fragments<BLOCKS>(acc + (16u << 16), hi);
  asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
  const auto at = [&](int row, int piece) { return row * 64 + ((piece ^ ((row >> 1) & 3)) * 16); };
  const uint32_t base = smem_u32(buf);
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i) {
    const auto pair = [&](const uint32_t* v) { return pack2(__uint_as_float(v[0]), __uint_as_float(v[1]), f16); };
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(base + at(8 * i + (lane & 7), lane >> 3)),
                 "r"(pair(lo + 4 * i)), "r"(pair(lo + 4 * i + 2)), "r"(pair(hi + 4 * i)), "r"(pair(hi + 4 * i + 2))
                 : "memory");
  }
  __syncwarp();
  uint4 w[BLOCKS];
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i) w[i] = *reinterpret_cast<const uint4*>(buf + at(8 * i + (lane >> 2), lane & 3));
#pragma unroll
  for (int i = 0; i < BLOCKS; ++i) {
    const int row = 8 * i + (lane >> 2), f = (lane & 3) * 8;
    store_piece_if(dst + row * pitch + f, w[i], row < n && f < features);
  }
  __syncwarp();
}

// FORWARD, DX: rows outside every group become zeros; by warps `at`, `at + warps`, ... of the grid.
__device__ __forceinline__ void zero_rows(const ProductArgs& g, const Table& tb, int at, int warps, int lane) {
  const int64_t bytes = (int64_t)g.features * 2;
  for (int w = 0; w < g.m; ++w) {
    const int head = tb.start[w * (g.E + 1)], tail = g.R - tb.start[w * (g.E + 1) + g.E];
    for (int i = at; i < head + tail; i += warps) {
      const int row = i < head ? i : g.R - tail + (i - head);
      if (g.parts) {
        float* dst = g.parts + ((int64_t)(g.first_worker + w) * g.R + row) * g.features;
        for (int split = 0; split < g.splits; ++split)
          for (int c = lane; c < g.features; c += 32) dst[split * g.part_size + c] = 0.f;
        continue;
      }
      uint8_t* dst = static_cast<uint8_t*>(g.out) + ((int64_t)(g.first_worker + w) * g.R + row) * bytes;
      if (g.out_width == 16)
        for (int64_t c = lane * 16; c < bytes; c += 512) *reinterpret_cast<uint4*>(dst + c) = make_uint4(0, 0, 0, 0);
      else
        for (int64_t c = lane * 2; c < bytes; c += 64) *reinterpret_cast<uint16_t*>(dst + c) = 0;
    }
  }
}

template <int MODE, int HALVES, int BN, int STAGES>
__global__ void __launch_bounds__(kThreads, 1)
product_kernel(const __grid_constant__ ProductMaps maps, const ProductArgs g) {
  constexpr bool A_MN = MODE != FORWARD, B_MN = MODE == DW;
  constexpr int kTileM = HALVES * kBM;
  constexpr uint32_t kHalfBytes = kBM * kBK * 2;          // of A
  constexpr uint32_t kABytes = HALVES * kHalfBytes;
  constexpr uint32_t kBBytes = BN * kBK * 2;
  constexpr uint32_t kStageBytes = kABytes + kBBytes;
  constexpr int kBlockCols = BN / 2 < 64 ? BN / 2 : 64;   // DW: columns an epilogue warp stages at a time
  constexpr uint32_t kStagingBytes = kEpiWarps * (MODE == DW ? 4096 : 2048);
  constexpr int kBufs = HALVES * BN <= 256 ? 2 : 1;       // accumulators
  constexpr uint32_t kTmemCols = kBufs * HALVES * BN;
  static_assert(kTmemCols <= 512 && (kTmemCols & (kTmemCols - 1)) == 0 && kTmemCols >= 32, "columns of tensor memory");
  static_assert(MODE != DW || BN % 64 == 0, "boxes of 64 columns");

  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  Control<STAGES>* ctl = reinterpret_cast<Control<STAGES>*>(tiles + STAGES * kStageBytes + kStagingBytes);
  Table& table = *reinterpret_cast<Table*>(ctl + 1);   // (FORWARD, DX)
  volatile int* abort_flag = &ctl->abort_flag;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t first = blockIdx.x, step = gridDim.x;

  if (threadIdx.x == 0) {
    prefetch_tensormap(&maps.a[MODE == DW ? 2 : 0]);
    prefetch_tensormap(&maps.b[MODE == DW ? 2 : 0]);
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&ctl->acc_full[b]), 1);
      mbar_init(smem_u32(&ctl->acc_empty[b]), kEpiWarps);
    }
    mbar_init(smem_u32(&ctl->last), 1);
    ctl->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (!g.beside) launch_gate();
  if (warp == 1) tmem_alloc(smem_u32(&ctl->tmem_base), kTmemCols);
  tc_fence_before();
  if (MODE != DW) make_table(g, table, BN);
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base;
  Walk<MODE, BN> walk(g, table, step);
  const uint32_t total = walk.total;
  const auto mma_cols = [&](const Unit& u) { return MODE == DW ? BN : (u.n + kSmallBox - 1) / kSmallBox * kSmallBox; };
  // Boxes of A and (DW) of B: none lies wholly outside its tensor.  What stays in their place reaches only parts of the
  // accumulator that are not stored.
  const auto a_boxes = [&](const Unit& u) {
    constexpr int kBox = A_MN ? 64 : kBM;
    return min(kTileM / kBox, (g.features - u.m * kTileM + kBox - 1) / kBox);
  };
  const auto b_boxes = [&](const Unit& u) { return min(BN / 64, (g.cols - u.col * BN + 63) / 64); };

  const bool one = MODE == DW ? lane == 0 : elect_one();   // (DW: its MMA warp has work for all lanes)
  uint32_t copied = 0;   // blocks that this thread has asked for
  if (warp == 0 && one) {
    // ---------------- TMA producer
    uint32_t& it = copied;
    for (uint32_t t = first; t < total && !*abort_flag; t += step) {
      const Unit u = walk.at(t);
      const int m0 = u.m * kTileM, held = mma_cols(u), na = a_boxes(u), nb = MODE == DW ? b_boxes(u) : 0;
      for (int kb = u.kb; kb < u.end; ++kb, ++it) {
        const int s = it % STAGES, k0 = kb * kBK;
        if (!mbar_wait(smem_u32(&ctl->empty[s]), ((it / STAGES) & 1) ^ 1, abort_flag)) break;
        const uint32_t bar = smem_u32(&ctl->full[s]);
        const uint32_t a_dst = smem_u32(tiles + s * kStageBytes), b_dst = a_dst + kABytes;
        if (MODE == DW) {
          const int n0 = u.col * BN, left = u.n - k0;
          const int rows = left >= kBK ? kBK : (left + kSmallBox - 1) / kSmallBox * kSmallBox;   // (some of them not the group's)
          // (what lies outside the tensor, as zeros, counts in a box)
          mbar_expect_tx(bar, (g.a_panels ? kABytes : (uint32_t)(na * rows * 128)) + (g.b_panels ? kBBytes : (uint32_t)(nb * rows * 128)));
          if (g.a_panels) tma_load_4d(a_dst, &maps.a[kPanels], bar, 0, u.row0 + k0, m0 / 64, u.worker);
          if (g.b_panels) tma_load_4d(b_dst, &maps.b[kPanels], bar, 0, u.row0 + k0, n0 / 64, u.worker);
          if (!g.a_panels || !g.b_panels) {
            int at = 0;
#pragma unroll
            for (int i = 2; i >= 0; --i)
              if (rows & (kSmallBox << i)) {
                const int row = u.row0 + k0 + at;
                for (int j = 0; j < na && !g.a_panels; ++j) tma_load_3d(a_dst + j * 8192 + at * 128, &maps.a[i], bar, m0 + 64 * j, row, u.worker);
                for (int j = 0; j < nb && !g.b_panels; ++j) tma_load_3d(b_dst + j * 8192 + at * 128, &maps.b[i], bar, n0 + 64 * j, row, u.worker);
                at += kSmallBox << i;
              }
          }
        } else {
          mbar_expect_tx(bar, (uint32_t)(na * (A_MN ? 8192 : (int)kHalfBytes) + held * 128));
          for (int j = 0; j < na; ++j) {
            if (A_MN) tma_load_4d(a_dst + j * 8192, &maps.a[0], bar, m0 + 64 * j, k0, u.group, u.worker);
            else tma_load_4d(a_dst + j * kHalfBytes, &maps.a[0], bar, k0, m0 + j * kBM, u.group, u.worker);
          }
          int at = 0;
#pragma unroll
          for (int i = kBoxes - 1; i >= 0; --i)
            if (held & (kSmallBox << i)) {
              tma_load_3d(b_dst + at * 128, &maps.b[i], bar, k0, u.row0 + at, u.worker);
              at += kSmallBox << i;
            }
        }
      }
    }
  } else if (warp == 1 && (MODE == DW || one)) {
    // ---------------- MMA issuer: one lane; DW: its warp comes along, for the zeros
    const uint32_t fmt = g.f16 ? 0u : ((1u << 7) | (1u << 10));
    const uint32_t idesc0 = (1u << 4) | fmt | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) | ((uint32_t)(kBM >> 4) << 24);
    uint32_t it = 0, n = 0;
    bool ok = true;
    for (uint32_t t = first; t < total && ok; t += step) {
      const Unit u = walk.at(t);
      if (u.kb == u.end) continue;
      const uint32_t idesc = idesc0 | ((uint32_t)(mma_cols(u) >> 3) << 17);
      const int k_extent = MODE == DW ? u.n : g.k_extent;
      const auto multiply = [&](int kb, uint32_t s, int half, uint32_t acc) {
        if (MODE == DW && lane != 0) return;
        const uint32_t a_addr = smem_u32(tiles + s * kStageBytes) + half * kHalfBytes, b_addr = smem_u32(tiles + s * kStageBytes) + kABytes;
        const uint64_t a_desc = A_MN ? smem_desc_mn_sw128(a_addr) : smem_desc_k_sw128(a_addr);
        const uint64_t b_desc = B_MN ? smem_desc_mn_sw128(b_addr) : smem_desc_k_sw128(b_addr);
        // 16 K elements: 32 bytes along a K-major row, 16 rows of 128 bytes of an MN-major tile
        constexpr uint64_t a_step = A_MN ? 128 : 2, b_step = B_MN ? 128 : 2;
        const int left = k_extent - kb * kBK;   // (what lies behind is zeros, or was not loaded)
#pragma unroll
        for (int k = 0; k < kBK / kUmmaK; ++k)
          if (k * kUmmaK < left) umma_bf16(acc, a_desc + a_step * k, b_desc + b_step * k, idesc, (kb > u.kb || k > 0) ? 1u : 0u);
      };
      const auto wait = [&](uint64_t* bar, uint32_t parity) {
        // (DW: one lane waits, for MMAs and commits of its own.  The others store zeros over what the barrier says has come: a
        // shuffle tells them so, but orders no memory)
        int done = 1;
        if (MODE != DW || lane == 0) done = mbar_wait(smem_u32(bar), parity, abort_flag);
        if (MODE == DW) {
          __syncwarp();
          done = __shfl_sync(0xffffffffu, done, 0);
        }
        tc_fence_after();
        return done != 0;
      };
      const auto commit = [&](uint64_t* bar) {
        if (MODE != DW || lane == 0) umma_commit(smem_u32(bar));
      };
      const auto arrived = [&](int kb, uint32_t i) {
        ok = wait(&ctl->full[i % STAGES], (i / STAGES) & 1);
        const int left = k_extent - kb * kBK;
        if (MODE == DW && ok && left < kBK && left % kSmallBox) {
          // (rows of 128 bytes, whatever the swizzle does inside them; up to 120 pieces a box)
          const int zeros = (kSmallBox - left % kSmallBox) * 8;
          uint4* row = reinterpret_cast<uint4*>(tiles + (i % STAGES) * kStageBytes + left * 128);
#pragma unroll
          for (int box = 0; box < kTileM / 64 + BN / 64; ++box)
#pragma unroll
            for (int q = 0; q < 4; ++q)
              if (q * 32 + lane < zeros) row[box * 512 + q * 32 + lane] = make_uint4(0, 0, 0, 0);
          fence_async_smem();
          __syncwarp();
        }
        return ok;
      };
      if constexpr (kBufs == 2) {
        const uint32_t buf = n & 1, acc = tmem_base + buf * (HALVES * BN);
        ok = wait(&ctl->acc_empty[buf], ((n >> 1) & 1) ^ 1);
        if (!ok) break;
        for (int kb = u.kb; kb < u.end; ++kb, ++it) {
          if (!arrived(kb, it)) break;
#pragma unroll
          for (int half = 0; half < HALVES; ++half) multiply(kb, it % STAGES, half, acc + half * BN);
          commit(&ctl->empty[it % STAGES]);
        }
        commit(&ctl->acc_full[buf]);
      } else {
        // The first blocks' MMAs of the first half run while the second is emptied.
        const int lead = u.kb + min(u.end - u.kb, STAGES);
        ok = wait(&ctl->acc_empty[0], (n & 1) ^ 1);
        if (!ok) break;
        for (int kb = u.kb; kb < lead; ++kb) {
          const uint32_t i = it + (kb - u.kb);
          if (!arrived(kb, i)) break;
          multiply(kb, i % STAGES, 0, tmem_base);
        }
        if (!ok) break;
        ok = wait(&ctl->acc_empty[1], (n & 1) ^ 1);
        if (!ok) break;
        for (int kb = u.kb; kb < lead; ++kb, ++it) {
          multiply(kb, it % STAGES, 1, tmem_base + BN);
          commit(&ctl->empty[it % STAGES]);
        }
        for (int kb = lead; kb < u.end; ++kb, ++it) {
          if (!arrived(kb, it)) break;
          multiply(kb, it % STAGES, 0, tmem_base);
          multiply(kb, it % STAGES, 1, tmem_base + BN);
          commit(&ctl->empty[it % STAGES]);
        }
        commit(&ctl->acc_full[0]);
      }
      ++n;
    }
  } else if (warp >= 2) {
    // ---------------- epilogue: warp w reads TMEM lanes 32 (w % 4) .. + 31; warps 2-5 and 6-9 share the columns
    const int lane_group = warp & 3, side = (warp - 2) >> 2;
    if (MODE != DW) zero_rows(g, table, blockIdx.x * kEpiWarps + warp - 2, gridDim.x * kEpiWarps, lane);
    uint32_t n = 0;
    for (uint32_t t = first; t < total; t += step) {
      const Unit u = walk.at(t);
      const bool none = MODE == DW && u.kb == u.end;   // zeros, and no accumulator
      const uint32_t buf = kBufs == 2 ? n & 1 : 0, parity = kBufs == 2 ? (n >> 1) & 1 : n & 1;
      // one lane waits for its warp (ordered by __syncwarp: the shuffle orders no memory): what follows wants all lanes together
      int ok = 1;
      if (lane == 0 && !none) ok = mbar_wait(smem_u32(&ctl->acc_full[buf]), parity, abort_flag);
      __syncwarp();
      ok = __shfl_sync(0xffffffffu, ok, 0);
      if (!ok) break;
      tc_fence_after();
#pragma unroll 1
      for (int half = 0; half < HALVES; ++half) {
        const int feature0 = u.m * kTileM + half * kBM + lane_group * 32;
        const uint32_t acc = tmem_base + (buf * HALVES + half) * BN + ((uint32_t)(lane_group * 32) << 16);
        if (feature0 < g.features) {
          if (g.parts) {
            // a row of 32 features a store; join_kernel rounds
            const int columns = MODE == DW ? min(BN, g.cols - u.col * BN) : u.n;
            const int64_t row = MODE == DW ? (int64_t)u.group * g.cols + u.col * BN : (int64_t)u.worker * g.R + u.row0;
            float* dst = g.parts + u.split * g.part_size + row * g.features + feature0 + lane;
#pragma unroll 1
            for (int c = side * 32; c < columns; c += 64) {
              float v[32];
              if (none) {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = 0.f;
              } else {
                tmem_ld32(acc + c, v);
              }
              if (feature0 + lane < g.features) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                  if (c + j < columns) dst[(int64_t)(c + j) * g.features] = v[j];
              }
              __syncwarp();
            }
          } else if constexpr (MODE == DW) {
            constexpr int W = kBlockCols;
            Staged<W> out{reinterpret_cast<uint4*>(tiles + STAGES * kStageBytes) + (warp - 2) * 256};
            uint16_t* dst = static_cast<uint16_t*>(g.out) + ((int64_t)u.group * g.features + feature0) * g.cols;
            for (int c0 = side * (BN / 2); c0 < (side + 1) * (BN / 2); c0 += W) {
              const int64_t col = (int64_t)u.col * BN + c0, cols = g.cols - col;
              if (cols <= 0) break;
              float v[W];
              if (none) {
#pragma unroll
                for (int k = 0; k < W; ++k) v[k] = 0.f;
              } else {
                tmem_ld_wide<W>(acc + c0, v);
              }
#pragma unroll
              for (int q = 0; q < W / 16; ++q) out.put(lane, q, v + 16 * q, g.f16);
              out.flush(lane, dst + col, g.cols, g.features - feature0, cols, g.out_width);
            }
          } else {
            uint16_t* dst = static_cast<uint16_t*>(g.out) + ((int64_t)u.worker * g.R + u.row0) * g.features + feature0;
            const bool live = feature0 + lane < g.features;
            uint8_t* buf_out = tiles + STAGES * kStageBytes + (warp - 2) * 2048;
            if (BN == 32) {
              // (sixteen columns for either side)
              uint16_t* first_row = dst + (int64_t)side * 16 * g.features;
              if (side * 16 < u.n) {
                if (g.out_width == 16) {
                  store_transposed<2>(buf_out, lane, acc + side * 16, first_row, g.features, u.n - side * 16, g.features - feature0, g.f16);
                } else {
                  float v[32];
                  tmem_ld16x2(acc + side * 16, acc + side * 16, v, v + 16);
                  store_rows(v, first_row + lane, g.features, min(16, u.n - side * 16), live, g.f16);
                }
              }
            } else if (g.out_width == 16) {
#pragma unroll 1
              for (int c = side * 32; c < u.n; c += 64)
                store_transposed<4>(buf_out, lane, acc + c, dst + (int64_t)c * g.features, g.features, u.n - c, g.features - feature0, g.f16);
            } else {
#pragma unroll 1
              for (int c = side * 32; c < u.n; c += 64) {
                float v[32];
                tmem_ld32(acc + c, v);
                store_rows(v, dst + (int64_t)c * g.features + lane, g.features, u.n - c, live, g.f16);
              }
            }
          }
        }
        if (none || (kBufs == 2 && half + 1 < HALVES)) continue;
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(smem_u32(&ctl->acc_empty[kBufs == 2 ? buf : half]));
        __syncwarp();
      }
      if (!none) ++n;
    }
  }

  // ---------------- teardown: every role arrives here, all waits above are bounded
  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    // Somebody gave up: what is still on its way into shared or tensor memory arrives (or is waited for long enough) before the CTA
    // gives them back.  The thread that asked for the copies waits for each stage's last one, whether it had left its loop before or
    // not; the thread that issued the MMAs, committed or not, for all of them.
    const uint64_t t0 = global_ns();
    const auto arrives = [&](uint64_t* bar, uint32_t parity) {
      while (!mbar_try_wait(smem_u32(bar), parity) && global_ns() - t0 < 10000000ull) {
      }
    };
    for (uint32_t i = copied > STAGES ? copied - STAGES : 0; i < copied; ++i) arrives(&ctl->full[i % STAGES], (i / STAGES) & 1);
    if (warp == 1 && one) {
      umma_commit(smem_u32(&ctl->last));
      arrives(&ctl->last, 0);
    }
    if (threadIdx.x == 0) atomicExch(g.status, (int)OLSGD_ETIMEOUT);
  }
  __syncthreads();
  __syncwarp();
  if (warp == 1) {
    tc_fence_after();
    tmem_dealloc(tmem_base, kTmemCols);
  }
  // what follows in the stream waits for this kernel: so this one waits for the kernel it ran beside
  if (g.beside) launch_gate();
}

// The sums of the parts of K, in their order, and the one rounding.  At most two products at a time (a backward call's),
// the first by the first blocks.  FORWARD, DX: the parts lie as the output does, V values a thread.  DW: they lie with features
// side by side, the output with columns: 32 x 32 at a time through shared memory.
struct JoinJob {
  const float* parts;
  void* out;
  int64_t part_size;
  int64_t blocks;
  int64_t features, cols;   // DW
  int splits, transposed, wide;   // wide: 4 values of the output are aligned together (and of the parts)
};
struct JoinArgs {
  JoinJob job[2];
  int f16;
};
template <int V>
__device__ __forceinline__ void sum_parts(const float* p, int64_t part_size, int splits, float* v) {
#pragma unroll
  for (int j = 0; j < V; ++j) v[j] = 0.f;
#pragma unroll 4
  for (int s = 0; s < splits; ++s) {
    if (V == 4) {
      const float4 x = __ldcg(reinterpret_cast<const float4*>(p + s * part_size));
      v[0] += x.x, v[1] += x.y, v[2] += x.z, v[3] += x.w;
    } else {
      v[0] += __ldcg(p + s * part_size);
    }
  }
}
__global__ void __launch_bounds__(256) join_kernel(const JoinArgs a) {
  launch_gate();
  __shared__ float tile[32][33];
  int64_t block = blockIdx.x;
  const bool second = block >= a.job[0].blocks;
  const JoinJob& j = a.job[second];
  if (second) block -= a.job[0].blocks;
  uint16_t* out = static_cast<uint16_t*>(j.out);
  if (!j.transposed) {
    const int64_t i = (block * 256 + threadIdx.x) * (j.wide ? 4 : 1);
    if (i >= j.part_size) return;
    float v[4];
    if (j.wide) {
      sum_parts<4>(j.parts + i, j.part_size, j.splits, v);
      *reinterpret_cast<uint2*>(out + i) = make_uint2(pack2(v[0], v[1], a.f16), pack2(v[2], v[3], a.f16));
    } else {
      sum_parts<1>(j.parts + i, j.part_size, j.splits, v);
      out[i] = (uint16_t)pack2(v[0], 0.f, a.f16);
    }
    return;
  }
  const int64_t f_tiles = (j.features + 31) / 32, c_tiles = (j.cols + 31) / 32;
  const int64_t group = block / (f_tiles * c_tiles), at = block - group * f_tiles * c_tiles;
  const int64_t c0 = at / f_tiles * 32, f0 = (at % f_tiles) * 32;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    const int64_t c = c0 + warp * 4 + q, f = f0 + lane;
    float v = 0.f;
    if (c < j.cols && f < j.features) sum_parts<1>(j.parts + (group * j.cols + c) * j.features + f, j.part_size, j.splits, &v);
    tile[lane][warp * 4 + q] = v;
  }
  __syncthreads();
  const int64_t f = f0 + threadIdx.x / 8, c = c0 + threadIdx.x % 8 * 4;
  if (f >= j.features || c >= j.cols) return;
  const float* v = tile[threadIdx.x / 8] + threadIdx.x % 8 * 4;
  uint16_t* dst = out + (group * j.features + f) * j.cols + c;
  const uint32_t lo = pack2(v[0], v[1], a.f16), hi = pack2(v[2], v[3], a.f16);
  if (j.wide) {
    *reinterpret_cast<uint2*>(dst) = make_uint2(lo, hi);
  } else {
    store_half_if(dst, lo, true);
    store_half_if(dst + 1, lo >> 16, c + 1 < j.cols);
    store_half_if(dst + 2, hi, c + 2 < j.cols);
    store_half_if(dst + 3, hi >> 16, c + 3 < j.cols);
  }
}

// --------------------------------------------------------------------------------- host
constexpr int kSms = 148;

template <int MODE, int HALVES, int BN, int STAGES>
cudaError_t launch_variant(const ProductMaps& maps, ProductArgs g, cudaStream_t s) {
  constexpr size_t smem = (size_t)STAGES * (HALVES * kBM + BN) * kBK * 2 + kEpiWarps * (MODE == DW ? 4096 : 2048) + (MODE == DW ? 0 : sizeof(Table)) +
                          sizeof(Control<STAGES>) + 1024;
  static_assert(smem <= 227 * 1024, "shared memory of one CTA");
  static PerDeviceSmem configured;
  auto kern = product_kernel<MODE, HALVES, BN, STAGES>;
  cudaError_t e = ensure_dynamic_smem(configured, kern, smem);
  if (e == cudaSuccess) e = status_word(&g.status);
  if (e != cudaSuccess) return e;
  g.m_tiles = (g.features + HALVES * kBM - 1) / (HALVES * kBM);
  g.n_tiles = (g.cols + BN - 1) / BN;
  // (of row tiles, disjoint groups have no more)
  const int64_t total = (int64_t)g.splits * g.m_tiles * g.m * (MODE == DW ? (int64_t)g.E * g.n_tiles : g.R / BN + (g.E < g.R ? g.E : g.R));
  const int64_t room = sm_count();
  g_tc_launches += 1;
  return launch_chained(kern, dim3((unsigned)(total < room ? total : room)), dim3(kThreads), smem, s, maps, g);
}

// Which tiles, and how many parts of K: by the sizes alone; how the rows fall to the experts is not known here and taken as even.
// A tile takes, in cycles, 1000 and per K block the longest of its operands' way from L2 (36 bytes a cycle and multiprocessor
// when all take in something, 44 when few do), its MMAs (M N / 64) and, where each weight is used by one tile only, the weights'
// way from memory (26 bytes a cycle of 148); its results' way out (24 bytes a cycle) passes beside the next tile where
// there are two accumulators, and for the most part does not where there is one.  The launch takes as many waves as its tiles need.
//   Tiles: of 23 sizes (16 to 65536 rows, 1 to 128 experts, widths of 128 to 8192) each tile was timed: what this
// picks is 1.1, 0.7 and 0.3 percent slower than the best of each on average (FORWARD, DX, DW), and up to 9 percent at the worst; one
// tile for all would be 6 (256 x 128 or 128 x 128, FORWARD) to 92 percent (128 x 32).
//   Parts: where the tiles leave multiprocessors without work, up to as many as fill one wave, of two blocks or more.  Adding
// them takes a launch and their way through L2.  us without and with them: DW of 65536 rows, 4 experts, 128 -> 256: 168 and 30; of
// 20000 rows, 512 -> 512: 129 and 34; FORWARD of one row, 4096 -> 4096: 17.9 and 10.2; of 64 rows, 4 experts, 2048 -> 1024: 11.3 and
// 8.9.  Forced where this does not take them: FORWARD of 3000 rows, 1024 -> 1024: 11.7 and 24.6; of 512 rows, 8 experts, 512 -> 512:
// 6.6 and 9.2; of 300 rows, 4096 -> 4096: 20.5 and 25.1.
struct Shape {
  int halves, bn, splits;
};
constexpr double kOutRate = 24;
double tile_cycles(const Shape& sh, double rows, double kbs, bool once, int bytes, double tiles) {
  const double m = sh.halves * kBM, share = kSms / (tiles < kSms ? tiles : kSms);
  const auto rate = [&](double all) { return all * share < 44 ? all * share : 44; };
  double block = (m + rows) * 128 / rate(36);
  if (m * rows / 64 > block) block = m * rows / 64;
  if (once && m * 128 / rate(26) > block) block = m * 128 / rate(26);
  const double in = kbs * block, out = m * rows * bytes / kOutRate;
  return 1000 + (sh.halves * sh.bn > 256 ? in + 0.8 * out : in > out ? in : out);
}
// The least of a launch's cost over tiles and parts of K: cost(shape), which knows its splits.
template <typename Tiles, typename Cost>
Shape least(double kbs, double values, const Tiles& tiles, const Cost& cost) {
  constexpr Shape shapes[] = {{1, 32, 1}, {1, 64, 1}, {1, 128, 1}, {1, 256, 1}, {2, 128, 1}, {2, 256, 1}};
  Shape best = shapes[0];
  double lowest = 1e300;
  for (Shape sh : shapes) {
    const double room = kSms / tiles(sh), deep = kbs / 2;
    const int fit = (int)(room < deep ? room : deep), most = fit < 32 ? fit : 32;
    for (sh.splits = 1;; sh.splits = 2 * sh.splits < most ? 2 * sh.splits : most) {
      double c = cost(sh);
      if (sh.splits > 1) c = 1.15 * (c + 4500 + 300 * sh.splits + values * (4 * sh.splits + 2) / (kSms * kOutRate));
      if (c < lowest) {
        lowest = c;
        best = sh;
      }
      if (sh.splits >= most) break;
    }
  }
  return best;
}
Shape shape_rows(const ProductShape& d, int64_t features, int64_t k) {
  const int64_t used = d.E < d.R ? d.E : d.R;
  const double rows = (double)d.R / used, kbs = (double)((k + kBK - 1) / kBK);
  const auto per_group = [&](const Shape& sh) { return rows <= 0.7 * sh.bn ? 1.0 : rows / sh.bn + 0.5; };
  const auto tiles = [&](const Shape& sh) { return d.m * used * per_group(sh) * ((features + sh.halves * kBM - 1) / (sh.halves * kBM)); };
  return least(kbs, (double)d.m * d.R * features, tiles, [&](const Shape& sh) {
    const double held = rows / per_group(sh), all = tiles(sh) * sh.splits, waves = all <= kSms ? 1.0 : all / kSms + 0.5;
    const int bytes = sh.splits > 1 ? 4 : 2;
    return waves * tile_cycles(sh, held, kbs / sh.splits, per_group(sh) < 1.5, bytes, all) + sh.halves * kBM * held * bytes / kOutRate;
  });
}
Shape shape_weights(const ProductShape& d) {
  const double kbs = (double)d.R / d.E / kBK + 0.5;
  const auto tiles = [&](const Shape& sh) {
    return (double)(d.m * d.E * ((d.F + sh.halves * kBM - 1) / (sh.halves * kBM)) * ((d.D + sh.bn - 1) / sh.bn));
  };
  return least(kbs, (double)d.m * d.E * d.F * d.D, tiles, [&](const Shape& sh) {
    if (sh.bn < 64) return 1e300;   // (a box of its operands has 64 columns)
    const int bytes = sh.splits > 1 ? 4 : 2;
    return ceil(tiles(sh) * sh.splits / kSms) * tile_cycles(sh, sh.bn, kbs / sh.splits, false, bytes, tiles(sh) * sh.splits) + sh.halves * kBM * sh.bn * bytes / kOutRate;
  });
}

// The workspace: copies of operands that TMA cannot take, and parts of K.
size_t parts_bytes(const Shape& sh, int64_t values) { return sh.splits > 1 ? round256((size_t)sh.splits * values * 4) : 0; }
size_t copied_bytes(int64_t groups, int64_t rows, int64_t pitch) { return round256((size_t)groups * rows * pitch * 2); }
// Of rows for a backward call: whole panels.
constexpr int64_t panels64(int64_t cols) { return (cols + 63) / 64 * 64; }

#define OLSGD_STEP(call)                    \
  do {                                      \
    const cudaError_t e_ = (call);          \
    if (e_ != cudaSuccess) return e_;       \
  } while (0)

// [m][E][F][D] 16-bit; boxes of 64 columns by box_rows rows.
bool make_map_weights(CUtensorMap* map, const ExpertOperand& w, const ProductShape& d, int box_rows) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const int64_t row = d.F > 1 ? w.row_stride : round8(d.D), expert = d.E > 1 ? w.expert_stride : row * d.F,
                worker = d.m > 1 ? w.worker_stride : expert * d.E;
  cuuint64_t dims[4] = {(cuuint64_t)d.D, (cuuint64_t)d.F, (cuuint64_t)d.E, (cuuint64_t)d.m};
  cuuint64_t strides[3] = {(cuuint64_t)row * 2, (cuuint64_t)expert * 2, (cuuint64_t)worker * 2};
  cuuint32_t box[4] = {(cuuint32_t)kBK, (cuuint32_t)box_rows, 1, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, d.f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(w.p), dims, strides,
            box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
bool weights_ready(const ExpertOperand& w, const ProductShape& d) {
  return (reinterpret_cast<uintptr_t>(w.p) & 15) == 0 && (d.F == 1 || w.row_stride % 8 == 0) && (d.E == 1 || w.expert_stride % 8 == 0) &&
         (d.m == 1 || w.worker_stride % 8 == 0);
}
// Weights that TMA cannot take, copied to padded rows at dst: all experts at once where they lie at one distance, else worker by
// worker in launches of their own.
cudaError_t weights_copied(Pads& pads, ExpertOperand& w, const ProductShape& d, uint8_t* dst, cudaStream_t s) {
  if (weights_ready(w, d)) return cudaSuccess;
  const int64_t pitch = round8(d.D);
  if (d.m == 1 || d.E == 1 || w.worker_stride == d.E * w.expert_stride) {
    pads.add(w.p, d.m * d.E, d.E > 1 ? w.expert_stride : w.worker_stride, d.F, w.row_stride, d.D, pitch, dst);
  } else {
    for (int64_t i = 0; i < d.m; ++i) {
      Pads one;
      one.add(static_cast<const uint16_t*>(w.p) + i * w.worker_stride, d.E, w.expert_stride, d.F, w.row_stride, d.D, pitch, dst + i * d.E * d.F * pitch * 2);
      OLSGD_STEP(one.launch(s));
    }
  }
  w = ExpertOperand{dst, d.E * d.F * pitch, d.F * pitch, pitch};
  return cudaSuccess;
}

// FORWARD and DX: out rows = weights x rows of `in`.  Workers go by as many a launch as its table holds.
template <int MODE>
cudaError_t launch_rows(const ProductShape& d, const Shape& sh, const ExpertOperand& w, const GatedOperand& in, const int32_t* offsets, void* out,
                        float* parts, cudaStream_t s) {
  const int64_t k = MODE == FORWARD ? d.D : d.F, features = MODE == FORWARD ? d.F : d.D;
  ProductMaps maps;
  bool ok = make_map_weights(&maps.a[0], w, d, MODE == FORWARD ? kBM : kBK);
  for (int i = 0; i < kBoxes; ++i) {
    // (boxes that the tile has no room for are not used)
    ok = ok && make_map16(&maps.b[i], in, k, d.R, d.m, kSmallBox << i, d.f16);
    if (i > 0) maps.a[i] = maps.a[0];
  }
  if (!ok) return cudaErrorInvalidValue;
  ProductArgs g{};
  g.R = (int)d.R;
  g.E = (int)d.E;
  g.f16 = d.f16;
  g.offsets = offsets;
  g.k_extent = (int)k;
  g.num_kb = (int)((k + kBK - 1) / kBK);
  g.features = (int)features;
  g.out = out;
  g.out_width = store_width(out, features);
  g.splits = sh.splits;
  g.parts = sh.splits > 1 ? parts : nullptr;
  g.part_size = d.m * d.R * features;
  const int64_t most = kMaxStarts / (d.E + 1) < kMaxGroups / d.E ? kMaxStarts / (d.E + 1) : kMaxGroups / d.E;
  for (int64_t at = 0; at < d.m; at += most) {
    g.first_worker = (int)at;
    g.m = (int)(d.m - at < most ? d.m - at : most);
    const cudaError_t e = sh.halves == 2 ? (sh.bn == 256 ? launch_variant<MODE, 2, 256, 3>(maps, g, s) : launch_variant<MODE, 2, 128, 4>(maps, g, s))
                          : sh.bn == 256 ? launch_variant<MODE, 1, 256, 4>(maps, g, s)
                          : sh.bn == 128 ? launch_variant<MODE, 1, 128, 6>(maps, g, s)
                          : sh.bn == 64  ? launch_variant<MODE, 1, 64, 8>(maps, g, s)
                                         : launch_variant<MODE, 1, 32, 9>(maps, g, s);
    if (e != cudaSuccess) return e;
  }
  return cudaSuccess;
}

// [m][rows][cols] 16-bit by panels of 64 columns: boxes of 64 rows by `panels` panels.
bool make_map_panels(CUtensorMap* map, const GatedOperand& o, int64_t cols, int64_t rows, int64_t m, int panels, bool f16) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const int64_t row = rows > 1 ? o.row_stride : cols, worker = m > 1 ? o.worker_stride : rows * row;
  cuuint64_t dims[4] = {64, (cuuint64_t)rows, (cuuint64_t)(cols / 64), (cuuint64_t)m};
  cuuint64_t strides[3] = {(cuuint64_t)row * 2, 128, (cuuint64_t)worker * 2};
  cuuint32_t box[4] = {64, (cuuint32_t)kBK, (cuuint32_t)panels, 1};
  cuuint32_t estr[4] = {1, 1, 1, 1};
  return fn(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(o.p), dims, strides, box, estr,
            CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) ==
         CUDA_SUCCESS;
}

// x_width, dy_width: columns of their rows in memory (of copies, with the zeros behind).
cudaError_t launch_weights(const ProductBackward& a, int64_t x_width, int64_t dy_width, const Shape& sh, bool beside, float* parts, cudaStream_t s) {
  ProductMaps maps;
  bool ok = true;
  for (int i = 0; i < kBoxes; ++i) {
    const int rows = i < 2 ? kSmallBox << i : kBK;
    ok = ok && make_map16(&maps.a[i], a.dy, a.F, a.R, a.m, rows, a.f16) && make_map16(&maps.b[i], a.x, a.D, a.R, a.m, rows, a.f16);
  }
  ProductArgs g{};
  g.a_panels = dy_width % 64 == 0;
  g.b_panels = x_width % 64 == 0;
  if (g.a_panels) ok = ok && make_map_panels(&maps.a[kPanels], a.dy, dy_width, a.R, a.m, sh.halves * kBM / 64, a.f16);
  if (g.b_panels) ok = ok && make_map_panels(&maps.b[kPanels], a.x, x_width, a.R, a.m, sh.bn / 64, a.f16);
  if (!ok) return cudaErrorInvalidValue;
  g.R = (int)a.R;
  g.E = (int)a.E;
  g.m = (int)a.m;
  g.f16 = a.f16;
  g.offsets = a.offsets;
  g.features = (int)a.F;
  g.cols = (int)a.D;
  g.beside = beside;
  g.out = a.dw;
  g.out_width = store_width(a.dw, a.D);
  g.splits = sh.splits;
  g.parts = sh.splits > 1 ? parts : nullptr;
  g.part_size = a.m * a.E * a.F * a.D;
  return sh.halves == 2 ? (sh.bn == 256 ? launch_variant<DW, 2, 256, 3>(maps, g, s) : launch_variant<DW, 2, 128, 4>(maps, g, s))
         : sh.bn == 256 ? launch_variant<DW, 1, 256, 4>(maps, g, s)
         : sh.bn == 128 ? launch_variant<DW, 1, 128, 6>(maps, g, s)
                        : launch_variant<DW, 1, 64, 7>(maps, g, s);
}

JoinJob join_rows(const Shape& sh, const float* parts, void* out, int64_t rows, int64_t features) {
  JoinJob j{};
  if (sh.splits == 1) return j;
  j.parts = parts;
  j.out = out;
  j.part_size = rows * features;
  j.splits = sh.splits;
  j.wide = store_width(out, features) >= 8;
  j.blocks = (j.part_size + 256 * (j.wide ? 4 : 1) - 1) / (256 * (j.wide ? 4 : 1));
  return j;
}
JoinJob join_weights(const Shape& sh, const float* parts, const ProductBackward& a) {
  JoinJob j{};
  if (sh.splits == 1) return j;
  j.parts = parts;
  j.out = a.dw;
  j.part_size = a.m * a.E * a.F * a.D;
  j.features = a.F;
  j.cols = a.D;
  j.splits = sh.splits;
  j.transposed = 1;
  j.wide = store_width(a.dw, a.D) >= 8;
  j.blocks = a.m * a.E * ((a.F + 31) / 32) * ((a.D + 31) / 32);
  return j;
}
cudaError_t launch_join(const JoinJob& x, const JoinJob& y, bool f16, cudaStream_t s) {
  if (x.blocks + y.blocks == 0) return cudaSuccess;
  return launch_chained(join_kernel, dim3((unsigned)(x.blocks + y.blocks)), dim3(256), 0, s, JoinArgs{{x, y}, f16});
}

}  // namespace

bool product_needs_copies(const ProductShape& d, const GatedOperand& x, const ExpertOperand& w, const GatedOperand* dy) {
  return !tma_ready(x, d.R, d.m) || !weights_ready(w, d) || (dy && !tma_ready(*dy, d.R, d.m));
}
size_t product_workspace(const ProductShape& d, bool backward, bool copies) {
  size_t bytes = 0;
  if (copies) bytes += copied_bytes(d.m, d.R, backward ? panels64(d.D) : round8(d.D)) + copied_bytes(d.m * d.E, d.F, round8(d.D));
  if (copies && backward) bytes += copied_bytes(d.m, d.R, panels64(d.F));
  if (!backward) return bytes + parts_bytes(shape_rows(d, d.F, d.D), d.m * d.R * d.F);
  return bytes + parts_bytes(shape_rows(d, d.D, d.F), d.m * d.R * d.D) + parts_bytes(shape_weights(d), d.m * d.E * d.F * d.D);
}

cudaError_t launch_product(ProductForward a, cudaStream_t s) {
  uint8_t* ws = static_cast<uint8_t*>(a.ws);
  const Shape sh = shape_rows(a, a.F, a.D);
  float* parts = reinterpret_cast<float*>(ws);
  ws += parts_bytes(sh, a.m * a.R * a.F);
  const Wanted x[] = {{&a.x, a.R}};
  Pads pads;
  make_ready(pads, x, 1, a.D, round8(a.D), a.m, ws);
  OLSGD_STEP(weights_copied(pads, a.w, a, ws + copied_bytes(a.m, a.R, round8(a.D)), s));
  OLSGD_STEP(pads.launch(s));
  OLSGD_STEP(launch_rows<FORWARD>(a, sh, a.w, a.x, a.offsets, a.y, parts, s));
  return launch_join(join_rows(sh, parts, a.y, a.m * a.R, a.F), JoinJob{}, a.f16, s);
}

cudaError_t launch_product_backward(ProductBackward a, cudaStream_t s) {
  uint8_t* ws = static_cast<uint8_t*>(a.ws);
  const Shape rows = shape_rows(a, a.D, a.F), weights = shape_weights(a);
  float* row_parts = reinterpret_cast<float*>(ws);
  ws += parts_bytes(rows, a.m * a.R * a.D);
  float* weight_parts = reinterpret_cast<float*>(ws);
  ws += parts_bytes(weights, a.m * a.E * a.F * a.D);
  // dy for both, the weights for dx, x for the weights' gradient
  const Wanted x[] = {{&a.x, a.R}}, dy[] = {{&a.dy, a.R}};
  Pads pads;
  const int64_t x_width = tma_ready(a.x, a.R, a.m) ? a.D : panels64(a.D), dy_width = tma_ready(a.dy, a.R, a.m) ? a.F : panels64(a.F);
  if (a.dw) make_ready(pads, x, 1, a.D, x_width, a.m, ws);
  ws += copied_bytes(a.m, a.R, panels64(a.D));
  if (a.dx) OLSGD_STEP(weights_copied(pads, a.w, a, ws, s));
  ws += copied_bytes(a.m * a.E, a.F, round8(a.D));
  make_ready(pads, dy, 1, a.F, dy_width, a.m, ws);
  OLSGD_STEP(pads.launch(s));
  // Neither product reads what the other writes.  The second is launched beside the first: its CTAs may start once all of
  // the first one's have passed their gate (whatever came before has completed then), it takes the multiprocessors as they
  // become free, and at its end it waits for the first.
  if (a.dx) OLSGD_STEP(launch_rows<DX>(a, rows, a.w, a.dy, a.offsets, a.dx, row_parts, s));
  if (a.dw) OLSGD_STEP(launch_weights(a, x_width, dy_width, weights, a.dx != nullptr, weight_parts, s));
  return launch_join(a.dx ? join_rows(rows, row_parts, a.dx, a.m * a.R, a.D) : JoinJob{}, a.dw ? join_weights(weights, weight_parts, a) : JoinJob{},
                     a.f16, s);
}

}  // namespace olsgd
