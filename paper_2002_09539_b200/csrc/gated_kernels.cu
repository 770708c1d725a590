// Gated feed-forward block on the fifth-generation tensor cores, worker-batched:
//   a = x Wg^T,  b = x Wu^T,  h = act(a) * b                                   (forward)
//   da = dh * b * act'(a),  db = dh * act(a)                                   (element-wise)
//   dx = da Wg + db Wu,  dWg = da^T x,  dWu = db^T x                           (backward)
// x [m][T][D], Wg and Wu [m][F][D], h [m][T][F]; 16-bit operands, fp32 accumulation in tensor
// memory, one rounding of each result.  Training keeps a and b, in fp32: 2 T F values written once
// and read once, against 4 T D F more multiply-adds to form them again.  da and db have to be
// rounded to 16 bits as operands; were a and b too, the gradients would be 1.7 times as far
// from the exact ones as the rounding of the result alone leaves them, instead of 1.4 times.  In fp16 they
// are scaled by a power of two where they would leave the type's range (scale_for).
//
// One kernel, three modes, persistent: a CTA (or a pair of CTAs on one 256-row tile,
// tcgen05 cta_group::2) walks over tiles of its output.  Warp 0 feeds a ring of shared-memory
// stages with TMA, warp 1 issues the MMAs into one of two accumulators in tensor memory, eight
// warps empty the other one.
//   FORWARD   A = x (K-major), B = the tile's rows of Wg and, below them, of Wu: both
//             projections are one MMA, so a thread of the epilogue finds a and b of the same
//             element in its own lane and forms h without any exchange.
//   DX        A = da then db (K-major), B = Wg then Wu read along D (MN-major): one
//             accumulation over 2 F, nothing transposed or concatenated in memory.
//   DW        A = da or db, B = x, both read along their rows (MN-major), K = T.
//
// Tiles: 128 rows (256 by a pair) x 64, 128 or 256 columns, by shape_for below.
//
// TMA wants 16-byte row pitches: operands that do not have them are copied to padded rows in
// the workspace first.  Every wait is bounded, as in the library's other tensor-core kernels.
#include "operator_tiles.cuh"

namespace olsgd {
namespace {

enum Mode { FORWARD = 0, DX = 1, DW = 2 };
constexpr int kGroup = 8;            // row tiles walked together (operand reuse in L2)

__device__ int g_operator_status;    // a bounded wait gave up (olsgd_operators_join)

struct alignas(64) GatedMaps {
  CUtensorMap a0, a1, b0, b1;
};
struct GatedArgs {
  int num_kb, kb_half;        // K blocks in all; of the first half (DX)
  int row_tiles, col_tiles;   // per problem
  int problems;               // workers (DW: workers x 2)
  int splits, kb_split;       // parts that K is cut into, K blocks of a part
  int rows, cols;             // extents of one problem's output (FORWARD: cols = F)
  int act, f16;
  int beside;                 // runs beside the kernel ahead of it: see launch_gated_backward
  int a_rows;                 // rows of A that are loaded (K-major): all 128 unless the problem has fewer
  int out_width;              // bytes (16, 8, 4, 2) that the output's base and rows are multiples of
  void* out0;                 // h, dx or dWg
  void* out1;                 // dWu
  float* pre;                 // FORWARD: a, b [m][T][2][Fp], or null
  int64_t pre_pitch;          // Fp
  const float* unscale;       // DX, DW: factors of the workers' results, or null
  float* parts;               // splits > 1: sums of the parts, [splits][problems][rows][parts_row]
  int64_t parts_row;          // (FORWARD: a, b as in pre)
};

template <int STAGES>
struct Control {
  uint64_t full[STAGES], empty[STAGES];
  uint64_t acc_full[2], acc_empty[2];
  uint32_t tmem_base;
  int abort_flag;
};

// ------------------------------------------------------------------------- activations
// By one exponential and one division: sigmoid(a) = 1 / (1 + e^-a), and 0.5 (1 + tanh z) =
// sigmoid(2 z) for gelu.  Limits are exact at both ends.
struct ActPair {
  float f, df;   // act(a), act'(a)
};
constexpr float kGeluK = 0.7978845608028654f;   // sqrt(2 / pi)
constexpr float kGeluC = 0.044715f;

__device__ __forceinline__ float sigmoid_of(float a) { return __fdividef(1.f, 1.f + ex2(-kLog2e * a)); }

template <int ACT>
__device__ __forceinline__ float act_value(float a) {
  if (ACT == OLSGD_ACT_RELU) return a > 0.f ? a : (a != a ? a : 0.f);
  if (ACT == OLSGD_ACT_SIGMOID) return sigmoid_of(a);
  const float s = ACT == OLSGD_ACT_SILU ? sigmoid_of(a) : sigmoid_of(2.f * kGeluK * a * fmaf(kGeluC * a, a, 1.f));
  // a = -inf (an overflowed product) meets s = 0: the limit is 0
  return s == 0.f ? 0.f : a * s;
}

template <int ACT>
__device__ __forceinline__ ActPair act_pair(float a) {
  ActPair r;
  if (ACT == OLSGD_ACT_RELU) {
    r.f = a > 0.f ? a : (a != a ? a : 0.f);
    r.df = a > 0.f ? 1.f : (a != a ? a : 0.f);
  } else if (ACT == OLSGD_ACT_SIGMOID) {
    // e^-|a| and 1 / (1 + e^-|a|) give f and 1 - f, whichever is small, without a difference
    const float e = ex2(-kLog2e * fabsf(a)), q = __fdividef(1.f, 1.f + e);
    r.f = a < 0.f ? e * q : q;
    r.df = e * q * q;
  } else if (ACT == OLSGD_ACT_SILU) {
    const float s = sigmoid_of(a);
    r.f = s == 0.f ? 0.f : a * s;
    r.df = s == 0.f ? 0.f : s * fmaf(a, 1.f - s, 1.f);
    if (s == 1.f) r.df = 1.f;
  } else {
    const float s = sigmoid_of(2.f * kGeluK * a * fmaf(kGeluC * a, a, 1.f));
    r.f = s == 0.f ? 0.f : a * s;
    // z' = k (1 + 3 c a^2); act' = s + a s (1 - s) 2 z'
    const float w = s * (1.f - s);
    r.df = w == 0.f ? s : fmaf(a * w, 2.f * kGeluK * fmaf(3.f * kGeluC * a, a, 1.f), s);
  }
  return r;
}

struct Tile {
  int problem, split, row, col;   // row and column tile
};
// Tiles of one problem in groups of kGroup row tiles, column by column inside a group.  (A launch of
// 2^31 tiles would write terabytes: 32 bits do, and divide quickly.)
__device__ __forceinline__ Tile tile_at(const GatedArgs& g, uint32_t t) {
  const uint32_t per = g.row_tiles * g.col_tiles, outer = t / per, i = t - outer * per;
  Tile r;
  r.problem = outer;
  r.split = 0;
  if (g.splits > 1) {
    r.problem = outer / g.splits;
    r.split = outer - r.problem * g.splits;
  }
  const uint32_t group_tiles = kGroup * g.col_tiles, group = i / group_tiles, first = group * kGroup;
  const uint32_t height = min((uint32_t)kGroup, g.row_tiles - first), j = i - group * group_tiles;
  r.col = j / height;
  r.row = first + j - r.col * height;
  return r;
}

template <int ACT>
__device__ __forceinline__ void activate16(const float* a, const float* b, float* h) {
#pragma unroll
  for (int j = 0; j < 16; ++j) h[j] = act_value<ACT>(a[j]) * b[j];
}

// SCALED: the results are fp16, times their worker's factor (as a variant: the factor's register costs bf16's weight gradients of
// 16 workers 2 us of 21).
template <int MODE, int CTAS, int BN, int STAGES, bool SCALED>
__global__ void __launch_bounds__(kThreads, 1)
gated_gemm_kernel(const __grid_constant__ GatedMaps maps, const GatedArgs g) {
  constexpr bool A_MN = MODE == DW, B_MN = MODE != FORWARD;
  constexpr int kBRows = BN / CTAS;                       // rows (columns of D) of B held by this CTA
  constexpr uint32_t kABytes = kBM * kBK * 2;
  constexpr uint32_t kBBytes = kBRows * kBK * 2;
  constexpr uint32_t kStageBytes = kABytes + kBBytes;
  constexpr int kColsOut = MODE == FORWARD ? BN / 2 : BN;  // output columns of a tile
  constexpr int kBlockCols = kColsOut / 2 < 64 ? kColsOut / 2 : 64;   // columns an epilogue warp stages at a time
  constexpr uint32_t kStagingBytes = kEpiWarps * 4096;
  constexpr uint32_t kTmemCols = 2 * BN;
  static_assert(kTmemCols <= 512 && (kTmemCols & (kTmemCols - 1)) == 0, "two accumulators");
  static_assert(CTAS == 1 || BN == 256, "pairs take whole tiles");

  extern __shared__ uint8_t smem_raw[];
  uint8_t* tiles = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) &
                                              ~static_cast<uintptr_t>(1023));
  Control<STAGES>* ctl = reinterpret_cast<Control<STAGES>*>(tiles + STAGES * kStageBytes + kStagingBytes);
  volatile int* abort_flag = &ctl->abort_flag;

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int rank = CTAS == 2 ? (int)cluster_ctarank() : 0;
  const bool leader = rank == 0;
  const uint32_t first = blockIdx.x / CTAS, step = gridDim.x / CTAS;
  const uint32_t total = (uint32_t)g.problems * g.splits * g.row_tiles * g.col_tiles;

  if (threadIdx.x == 0) {
    prefetch_tensormap(&maps.a0);
    prefetch_tensormap(&maps.b0);
    if (MODE != FORWARD) prefetch_tensormap(&maps.a1);
    if (MODE != DW) prefetch_tensormap(&maps.b1);
    for (int s = 0; s < STAGES; ++s) {
      mbar_init(smem_u32(&ctl->full[s]), 1);
      mbar_init(smem_u32(&ctl->empty[s]), 1);
    }
    for (int b = 0; b < 2; ++b) {
      mbar_init(smem_u32(&ctl->acc_full[b]), 1);
      mbar_init(smem_u32(&ctl->acc_empty[b]), CTAS * kEpiWarps);
    }
    ctl->abort_flag = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == 1) {
    if (CTAS == 2) tmem_alloc_pair(smem_u32(&ctl->tmem_base), kTmemCols);
    else tmem_alloc(smem_u32(&ctl->tmem_base), kTmemCols);
  }
  tc_fence_before();
  __syncthreads();
  if (CTAS == 2) cluster_barrier();   // the peer's barriers are initialised
  tc_fence_after();
  const uint32_t tmem_base = ctl->tmem_base;
  if (!g.beside) launch_gate();

  if (warp == 0 && lane == 0) {
    // ---------------- TMA producer (both CTAs of a pair; the leader announces both's bytes)
    uint32_t it = 0;
    for (uint32_t t = first; t < total && !*abort_flag; t += step) {
      const Tile tl = tile_at(g, t);
      const int worker = MODE == DW ? tl.problem >> 1 : tl.problem;
      const int m0 = (tl.row * CTAS + rank) * kBM;
      for (int kb = tl.split * g.kb_split, end = min(g.num_kb, kb + g.kb_split); kb < end; ++kb, ++it) {
        const int s = it % STAGES;
        if (!mbar_wait(smem_u32(&ctl->empty[s]), ((it / STAGES) & 1) ^ 1, abort_flag)) break;
        const uint32_t bar_own = smem_u32(&ctl->full[s]);
        if (leader) mbar_expect_tx(bar_own, A_MN ? CTAS * kStageBytes : CTAS * (g.a_rows * (kBK * 2) + kBBytes));
        const uint32_t a_dst = smem_u32(tiles + s * kStageBytes), b_dst = a_dst + kABytes;
        const bool second = MODE == DX && kb >= g.kb_half;
        const int k0 = (second ? kb - g.kb_half : kb) * kBK;
        auto load = [&](uint32_t dst, const CUtensorMap* map, int c0, int c1) {
          if (CTAS == 2) tma_load_3d_pair(dst, map, pair_leader_addr(bar_own), c0, c1, worker);
          else tma_load_3d(dst, map, bar_own, c0, c1, worker);
        };
        if (A_MN) {
          const CUtensorMap* map = (tl.problem & 1) ? &maps.a1 : &maps.a0;
          load(a_dst, map, m0, k0);
          load(a_dst + kABytes / 2, map, m0 + 64, k0);
        } else {
          load(a_dst, second ? &maps.a1 : &maps.a0, k0, m0);
        }
        if (MODE == FORWARD) {
          const int f0 = tl.col * kColsOut;
          if (CTAS == 2) {
            load(b_dst, rank ? &maps.b1 : &maps.b0, k0, f0);
          } else {
            load(b_dst, &maps.b0, k0, f0);
            load(b_dst + kBBytes / 2, &maps.b1, k0, f0);
          }
        } else {
          const int n0 = tl.col * BN + rank * kBRows;
#pragma unroll
          for (int j = 0; j < kBRows / 64; ++j)
            load(b_dst + j * 8192, MODE == DX && second ? &maps.b1 : &maps.b0, n0 + 64 * j, k0);
        }
      }
    }
    // drain: whoever gave up waits (bounded) for the copies of this CTA still in flight
    if (CTAS == 1 && *abort_flag) {
      const uint32_t from = it > STAGES ? it - STAGES : 0;
      for (uint32_t i = from; i < it; ++i)
        for (uint32_t n = 0; n < kSpinLimit && !mbar_try_wait(smem_u32(&ctl->full[i % STAGES]), (i / STAGES) & 1); ++n)
          if ((n & 1023u) == 1023u && global_ns() == 0) break;
    }
  } else if (warp == 1 && lane == 0 && leader) {
    // ---------------- MMA issuer
    const uint32_t fmt = g.f16 ? 0u : ((1u << 7) | (1u << 10));
    const uint32_t idesc = (1u << 4) | fmt | (A_MN ? 1u << 15 : 0u) | (B_MN ? 1u << 16 : 0u) |
                           ((uint32_t)(BN >> 3) << 17) | ((uint32_t)((CTAS * kBM) >> 4) << 24);
    uint32_t it = 0, n = 0;
    bool ok = true;
    for (uint32_t t = first; t < total && ok; t += step, ++n) {
      const uint32_t buf = n & 1;
      ok = mbar_wait(smem_u32(&ctl->acc_empty[buf]), ((n >> 1) & 1) ^ 1, abort_flag);
      if (!ok) break;
      tc_fence_after();
      const uint32_t acc = tmem_base + buf * BN;
      const int kb0 = g.splits > 1 ? tile_at(g, t).split * g.kb_split : 0, kb_end = min(g.num_kb, kb0 + g.kb_split);
      for (int kb = kb0; kb < kb_end; ++kb, ++it) {
        const int s = it % STAGES;
        ok = mbar_wait(smem_u32(&ctl->full[s]), (it / STAGES) & 1, abort_flag);
        if (!ok) break;
        tc_fence_after();
        const uint32_t a_addr = smem_u32(tiles + s * kStageBytes), b_addr = a_addr + kABytes;
        const uint64_t a_desc = A_MN ? smem_desc_mn_sw128(a_addr) : smem_desc_k_sw128(a_addr);
        const uint64_t b_desc = B_MN ? smem_desc_mn_sw128(b_addr) : smem_desc_k_sw128(b_addr);
        // 16 K elements: 32 bytes along a K-major row, 16 rows of 128 bytes of an MN-major tile
        constexpr uint64_t a_step = A_MN ? 128 : 2, b_step = B_MN ? 128 : 2;
#pragma unroll
        for (int k = 0; k < kBK / kUmmaK; ++k) {
          const uint32_t accumulate = (kb > kb0 || k > 0) ? 1u : 0u;
          if (CTAS == 2) umma_bf16_pair(acc, a_desc + a_step * k, b_desc + b_step * k, idesc, accumulate);
          else umma_bf16(acc, a_desc + a_step * k, b_desc + b_step * k, idesc, accumulate);
        }
        if (CTAS == 2) umma_commit_pair(smem_u32(&ctl->empty[s]));
        else umma_commit(smem_u32(&ctl->empty[s]));
      }
      if (CTAS == 2) umma_commit_pair(smem_u32(&ctl->acc_full[buf]));
      else umma_commit(smem_u32(&ctl->acc_full[buf]));
    }
  } else if (warp >= 2) {
    // ---------------- epilogue: warp w reads TMEM lanes 32 (w % 4) .. + 31; warps 2-5 take the
    // left half of the tile's 16-column blocks, warps 6-9 the right half
    const int lane_group = warp & 3, half = (warp - 2) >> 2;
    constexpr int W = kBlockCols;
    Staged<W> out{reinterpret_cast<uint4*>(tiles + STAGES * kStageBytes) + (warp - 2) * 256};
    uint32_t n = 0;
    for (uint32_t t = first; t < total; t += step, ++n) {
      const uint32_t buf = n & 1;
      const Tile tl = tile_at(g, t);
      const int64_t worker = MODE == DW ? tl.problem >> 1 : tl.problem;
      const int64_t row0 = (int64_t)(tl.row * CTAS + rank) * kBM + lane_group * 32;
      const int64_t rows = g.rows - row0;   // of this warp's block that exist
      if (!mbar_wait(smem_u32(&ctl->acc_full[buf]), (n >> 1) & 1, abort_flag) || *abort_flag) break;
      tc_fence_after();
      const uint32_t acc = tmem_base + buf * BN + ((uint32_t)(lane_group * 32) << 16);
      uint16_t* dst = static_cast<uint16_t*>(MODE == DW && (tl.problem & 1) ? g.out1 : g.out0) + (worker * g.rows + row0) * g.cols;
      // a part of K: sums in fp32 to this part's own place
      float* part = g.splits > 1 ? g.parts + (((int64_t)tl.split * g.problems + tl.problem) * g.rows + row0) * g.parts_row : nullptr;
      float* pre = !g.pre ? nullptr : g.pre + (worker * g.rows + row0) * g.parts_row;   // (rows of a and b, as in parts)
      if (MODE == FORWARD && part) pre = part;
      // (past L1: this kernel may run beside its predecessor)
      const float unscale = SCALED ? __ldcg(g.unscale + worker) : 1.f;
      if (rows > 0) {
        for (int c0 = half * (kColsOut / 2); c0 < (half + 1) * (kColsOut / 2); c0 += W) {
          const int64_t col = (int64_t)tl.col * kColsOut + c0;
          const int64_t cols = g.cols - col;
          if (cols <= 0) break;
          if (MODE == FORWARD) {
            if (pre) {
              // (columns up to pre_pitch exist)
              constexpr int kCols = W < 32 ? W : 32;
#pragma unroll 1
              for (int q = 0; q < 2 * (W / kCols); ++q) {
                const int c = q / 2 * kCols, z = q & 1;   // a, then b
                spill_sums<kCols>(out.buf, lane, acc + z * (BN / 2) + c0 + c, pre + z * g.pre_pitch + col + c, g.parts_row, rows,
                                  g.pre_pitch - col - c);
              }
            }
#pragma unroll 1
            for (int q = 0; q < (part ? 0 : W / 16); ++q) {
              float a[16], b[16], h[16];
              tmem_ld16x2(acc + c0 + q * 16, acc + BN / 2 + c0 + q * 16, a, b);
              switch (g.act) {
                case OLSGD_ACT_SILU: activate16<OLSGD_ACT_SILU>(a, b, h); break;
                case OLSGD_ACT_GELU: activate16<OLSGD_ACT_GELU>(a, b, h); break;
                case OLSGD_ACT_RELU: activate16<OLSGD_ACT_RELU>(a, b, h); break;
                default: activate16<OLSGD_ACT_SIGMOID>(a, b, h);
              }
              out.put(lane, q, h, g.f16);
            }
            if (!part) out.flush(lane, dst + col, g.cols, rows, cols, g.out_width);
          } else {
            if (part) {
#pragma unroll 1
              for (int c = 0; c < W; c += 32)
                spill_sums<32>(out.buf, lane, acc + c0 + c, part + col + c, g.parts_row, rows, g.parts_row - col - c);
            }
#pragma unroll 1
            for (int q = 0; q < (part ? 0 : W / 16); q += 2) {
              float v[16], w[16];
              tmem_ld16x2(acc + c0 + q * 16, acc + c0 + q * 16 + 16, v, w);
              out.put(lane, q, v, SCALED || g.f16, unscale);
              out.put(lane, q + 1, w, SCALED || g.f16, unscale);
            }
            if (!part) out.flush(lane, dst + col, g.cols, rows, cols, g.out_width);
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (CTAS == 2) arrive_leader(smem_u32(&ctl->acc_empty[buf]));
        else mbar_arrive(smem_u32(&ctl->acc_empty[buf]));
      }
    }
  }

  // ---------------- teardown: every role arrives here, all waits above are bounded
  tc_fence_before();
  __syncthreads();
  if (*abort_flag && threadIdx.x == 0) {
    // bounded grace period for copies and MMAs that may still be in flight
    const uint64_t t0 = global_ns();
    while (global_ns() - t0 < 1000000ull) {
    }
    atomicExch(&g_operator_status, (int)OLSGD_ETIMEOUT);
  }
  if (CTAS == 2) cluster_barrier();
  else __syncthreads();
  if (warp == 1) {
    tc_fence_after();
    if (CTAS == 2) tmem_dealloc_pair(tmem_base, kTmemCols);
    else tmem_dealloc(tmem_base, kTmemCols);
  }
  // what follows in the stream waits for this kernel: so this one waits for the kernel it ran beside
  if (g.beside) launch_gate();
}

// ------------------------------------------------------------------------- few tokens
// Up to kFewTokens tokens a worker: every weight is used that often, so reading the weights is
// all there is to it and the tensor cores have nothing to gain.  A warp per feature holds its
// rows of Wg and Wu 16 bytes a lane at a time against all tokens (x comes from L1), and adds
// the lanes up at the end.  1024 -> 4096 bf16: 4.7 us for one token and 5.3 us for two, against
// 8.5 us by 64-column tiles on the tensor cores, which take over at three (9.0 us here).
constexpr int kFewTokens = 2;

template <typename T, int NT, bool VEC>
__global__ void __launch_bounds__(256)
gated_few_kernel(GatedOperand x, GatedOperand wg, GatedOperand wu, int tokens, int64_t D, int64_t F, int act, T* __restrict__ h,
                 float* __restrict__ pre, int64_t pre_pitch) {
  launch_gate();
  const int lane = threadIdx.x & 31;
  const int64_t f = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), worker = blockIdx.y;
  if (f >= F) return;
  const T* xw = static_cast<const T*>(x.p) + worker * x.worker_stride;
  const T* g = static_cast<const T*>(wg.p) + worker * wg.worker_stride + f * wg.row_stride;
  const T* u = static_cast<const T*>(wu.p) + worker * wu.worker_stride + f * wu.row_stride;
  float a[NT], b[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) a[t] = b[t] = 0.f;
  const T* xt[NT];   // (with fewer tokens than NT the last one is formed again, and not stored)
#pragma unroll
  for (int t = 0; t < NT; ++t) xt[t] = xw + min(t, tokens - 1) * x.row_stride;
  if (VEC) {   // D a multiple of 8, every row on a 16-byte boundary
    constexpr int U = 4;
    f32x2 a2[NT], b2[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) a2[t] = b2[t] = 0;
    for (int64_t j0 = lane * 8; j0 < D; j0 += 256 * U) {
      uint4 rg[U], ru[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const bool live = j0 + i * 256 < D;
        rg[i] = live ? ld16_stream(g + j0 + i * 256) : make_uint4(0, 0, 0, 0);
        ru[i] = live ? ld16_stream(u + j0 + i * 256) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < U; ++i) {
        uint4 rx[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t) rx[t] = j0 + i * 256 < D ? ld16(xt[t] + j0 + i * 256) : make_uint4(0, 0, 0, 0);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const f32x2 vg = raw_pair<T>(rg[i], e), vu = raw_pair<T>(ru[i], e);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            const f32x2 vx = raw_pair<T>(rx[t], e);
            a2[t] = fma2(vx, vg, a2[t]);
            b2[t] = fma2(vx, vu, b2[t]);
          }
        }
      }
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      float lo, hi;
      unpack2f(a2[t], lo, hi);
      a[t] = lo + hi;
      unpack2f(b2[t], lo, hi);
      b[t] = lo + hi;
    }
  } else {
#pragma unroll 4
    for (int64_t j = lane; j < D; j += 32) {
      const float vg = Elem<T>::to_float(g[j]), vu = Elem<T>::to_float(u[j]);
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const float vx = Elem<T>::to_float(xt[t][j]);
        a[t] = fmaf(vx, vg, a[t]);
        b[t] = fmaf(vx, vu, b[t]);
      }
    }
  }
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    if (t >= tokens) break;
    const float at = warp_sum(a[t]), bt = warp_sum(b[t]);
    if (lane == 0) {
      const float v = act == OLSGD_ACT_SILU   ? act_value<OLSGD_ACT_SILU>(at)
                      : act == OLSGD_ACT_GELU ? act_value<OLSGD_ACT_GELU>(at)
                      : act == OLSGD_ACT_RELU ? act_value<OLSGD_ACT_RELU>(at)
                                              : act_value<OLSGD_ACT_SIGMOID>(at);
      const int64_t row = worker * tokens + t;
      h[row * F + f] = Elem<T>::from_float(v * bt);
      if (pre) {
        float* p = pre + row * 2 * pre_pitch;
        p[f] = at;
        p[pre_pitch + f] = bt;
        if (f == F - 1)   // the padding of the rows
          for (int64_t k = F; k < pre_pitch; ++k) p[k] = p[pre_pitch + k] = 0.f;
      }
    }
  }
}

// ------------------------------------------------------------------- element-wise kernels

// Adds up the parts that K was cut into (in order) and finishes as the epilogue would have.
template <typename T, int MODE>
__global__ void __launch_bounds__(256) gated_join_kernel(const GatedArgs g) {
  launch_gate();
  const int64_t width = MODE == FORWARD ? g.pre_pitch : g.parts_row;   // columns, rounded up to 8
  const int64_t problem = blockIdx.y, stretches = (width + 255) / 256;
  const int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), r = at / stretches;
  const int64_t c = (at - r * stretches) * 256 + (threadIdx.x & 31) * 8;
  if (r >= g.rows || c >= width) return;
  const float* p = g.parts + (problem * g.rows + r) * g.parts_row + c;
  float a[8], b[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) a[e] = b[e] = 0.f;
  for (int s = 0; s < g.splits; ++s, p += (int64_t)g.problems * g.rows * g.parts_row) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; k += 4) Elem<float>::unpack(ld16_stream(p + k), v + k);
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] += v[e];
    if (MODE == FORWARD) {
#pragma unroll
      for (int k = 0; k < 8; k += 4) Elem<float>::unpack(ld16_stream(p + g.pre_pitch + k), v + k);
#pragma unroll
      for (int e = 0; e < 8; ++e) b[e] += v[e];
    }
  }
  T* out = static_cast<T*>(MODE == DW && (problem & 1) ? g.out1 : g.out0) + ((MODE == DW ? problem >> 1 : problem) * g.rows + r) * g.cols;
  if (MODE == FORWARD) {
    if (g.pre) {
      float* pre = g.pre + (problem * g.rows + r) * 2 * g.pre_pitch + c;
      store_sector_if(pre, a, true);
      store_sector_if(pre + g.pre_pitch, b, true);
    }
#pragma unroll
    for (int e = 0; e < 8; ++e)
      a[e] = b[e] * (g.act == OLSGD_ACT_SILU   ? act_value<OLSGD_ACT_SILU>(a[e])
                     : g.act == OLSGD_ACT_GELU ? act_value<OLSGD_ACT_GELU>(a[e])
                     : g.act == OLSGD_ACT_RELU ? act_value<OLSGD_ACT_RELU>(a[e])
                                               : act_value<OLSGD_ACT_SIGMOID>(a[e]));
  } else if (g.unscale) {
    const float unscale = g.unscale[MODE == DW ? problem >> 1 : problem];
#pragma unroll
    for (int e = 0; e < 8; ++e) a[e] *= unscale;
  }
  store_floats<T, 8>(out, c, g.cols, g.out_width == 16, a);
}

constexpr int kStretch = 512;

// x . w over D in 64 bits, by a warp (every lane gets it).  Products of 16-bit values are exact in fp32.
template <typename T>
__device__ __forceinline__ double warp_dot(const T* x, const T* w, int64_t D, bool vec) {
  const int lane = threadIdx.x & 31;
  double part[4] = {0.0, 0.0, 0.0, 0.0};   // (a chain of additions takes longer than the loads)
  if (vec) {
#pragma unroll 2
    for (int64_t k = lane * 8; k < D; k += 256) {
      float vx[8], vw[8];
      Elem<T>::unpack(ld16(x + k), vx);
      Elem<T>::unpack(ld16(w + k), vw);
#pragma unroll
      for (int e = 0; e < 8; ++e) part[e & 3] += (double)(vx[e] * vw[e]);
    }
  } else {
    constexpr int U = 8;
    for (int64_t k0 = lane; k0 < D; k0 += 32 * U) {
      float v[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int64_t k = k0 + u * 32;
        v[u] = k < D ? Elem<T>::to_float(x[k]) * Elem<T>::to_float(w[k]) : 0.f;
      }
#pragma unroll
      for (int u = 0; u < U; ++u) part[u & 3] += (double)v[u];
    }
  }
  double s = (part[0] + part[1]) + (part[2] + part[3]);
#pragma unroll
  for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
  return s;
}

// Whether any element of x and the same one of w are both other than 0; by a warp.
template <typename T>
__device__ __forceinline__ bool warp_overlap(const T* x, const T* w, int64_t D, bool vec) {
  const int lane = threadIdx.x & 31;
  uint32_t any = 0;
  if (vec) {
#pragma unroll 4
    for (int64_t k = lane * 8; k < D; k += 256) {
      const uint4 a = ld16(x + k), b = ld16(w + k);
      any |= __vminu2(a.x & 0x7FFF7FFFu, b.x & 0x7FFF7FFFu) | __vminu2(a.y & 0x7FFF7FFFu, b.y & 0x7FFF7FFFu) |
             __vminu2(a.z & 0x7FFF7FFFu, b.z & 0x7FFF7FFFu) | __vminu2(a.w & 0x7FFF7FFFu, b.w & 0x7FFF7FFFu);
    }
  } else {
#pragma unroll 4
    for (int64_t k = lane; k < D; k += 32) any |= Elem<T>::to_float(x[k]) != 0.f && Elem<T>::to_float(w[k]) != 0.f;
  }
  return __any_sync(0xffffffffu, any != 0);
}

// The first element of a piece.
template <typename T>
__device__ __forceinline__ float raw_first(const uint4& w) {
  float lo, hi;
  unpack2f(raw_pair<T>(w, 0), lo, hi);
  return lo;
}

// relu's derivative jumps at 0, and an accumulation in fp32 is off by a share of its partial sums, none of which
// exceeds |x_t| |w_f| (Euclidean norms).  Where a lies within
//   (8 + D / 128) 2^-23 |x_t| |w_f|
// of 0 its side is not to be trusted, and a is formed again in 64 bits.  Measured (D from 16 to 65536): values of random
// signs are off by up to 2.4 of these units at any D, products that are positive in the first half of D and
// negative in the second by D / 200.  One element of 20000 is formed again at D = 1024, one of 4000 at D = 4096.
//
// Sums that are exact need no second look, and zeros are mostly that: rows of zeros (tokens that are padding, features
// that were pruned) and rows with one element other than 0 count as rows of norm 0; where both rows are coarse (multiples
// of a power of two that is 2^-10 of the norm or more: small integers), 22 bits hold every partial sum.
//
// row_norms_kernel: the norm of each row of x and w_gate, with the sign set on that of a coarse row; a warp per row.
// Most rows are done after their first reading; only those whose first 256 elements are coarse are read twice.  16
// workers, 128 tokens, 1024 -> 1024: 37 MB in 10.4 us from cold caches (3.6 TB/s; two rows a warp were no faster).
// relu's backward pass takes 54.6 us there, silu's, which needs no norms, 44.8; 8192 tokens, 4096 -> 8192: 1895 and 1872.
template <typename T>
__global__ void __launch_bounds__(256)
row_norms_kernel(GatedOperand x, GatedOperand w, int64_t tokens, int64_t F, int64_t D, float* __restrict__ xn, float* __restrict__ wn,
                 int64_t wn_pitch) {
  constexpr int V = Elem<T>::kVec;
  launch_gate();
  const int lane = threadIdx.x & 31;
  const bool of_w = blockIdx.z != 0;
  const int64_t r = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), worker = blockIdx.y;
  if (r >= (of_w ? F : tokens)) return;
  const GatedOperand& o = of_w ? w : x;
  const T* row = static_cast<const T*>(o.p) + worker * o.worker_stride + r * o.row_stride;
  const int64_t n = D + row_shift(row), j0 = lane * V - row_shift(row);
  constexpr int kStep = 32 * V, U = 4;
  f32x2 sum = 0;
  uint4 first;
  for (int64_t p = 0; p < n; p += U * kStep) {
    const int64_t j = j0 + p;
    uint4 v[U];
    if (j >= 0 && j + (U - 1) * kStep + V <= D) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = ld16(row + j + u * kStep);
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = load_raw<T>(row, j + u * kStep, D, 0);
    }
    if (p == 0) first = v[0];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int e = 0; e < V / 2; ++e) {
        const f32x2 t = raw_pair<T>(v[u], e);
        sum = fma2(t, t, sum);
      }
  }
  float lo, hi;
  unpack2f(sum, lo, hi);
  lo = warp_sum(lo + hi);
  float norm = sqrtf(lo);
  if (!(lo > 1e-20f && lo < 1e30f)) {   // zeros, or squares outside fp32's comfortable range
    double s = 0.0;
    for (int64_t j = lane; j < D; j += 32) {
      const double v = (double)Elem<T>::to_float(row[j]);
      s = fma(v, v, s);
    }
#pragma unroll
    for (int off = 16; off; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
    norm = (float)sqrt(s);
  }
  // (2^10 over the norm's power of two; rows whose norm is next to the ends of fp32's range are not coarse)
  const int exponent = (int)(__float_as_uint(norm) >> 23);
  bool coarse = exponent > 30 && exponent < 220;
  const float to_grid = __uint_as_float((uint32_t)(coarse ? 127 + 127 + 10 - exponent : 127) << 23);
  // (one element a lane tells nearly every row that is not)
  if (coarse) {
    const float t = raw_first<T>(first) * to_grid;
    coarse = __all_sync(0xffffffffu, t == rintf(t));
  }
  int others = 0;   // elements other than 0
  for (int64_t p = 0; p < n && coarse; p += kStep) {
    float v[V];
    Elem<T>::unpack(p == 0 ? first : load_raw<T>(row, j0 + p, D, 0), v);
    bool on_grid = true;
#pragma unroll
    for (int e = 0; e < V; ++e) {
      const float t = v[e] * to_grid;
      on_grid = on_grid && t == rintf(t);
      others += v[e] != 0.f;
    }
    coarse = __all_sync(0xffffffffu, on_grid);
  }
  if (coarse) {
    others = __reduce_add_sync(0xffffffffu, others);
    norm = others <= 1 ? 0.f : -norm;
  }
  if (lane == 0) {
    if (of_w) wn[worker * wn_pitch + r] = norm;
    else xn[worker * tokens + r] = norm;
  }
}

struct Border {
  GatedOperand x, wg;
  int64_t D;
  bool vec;                 // rows of x and w_gate start on 16-byte boundaries, D is a multiple of 8
  float bound;              // (8 + D / 128) 2^-23
  const float *xn, *wn;     // norms [m][T], [m][pitch]
};

// da = dh b act'(a), db = dh act(a); a, b, da, db have rows of `pitch`.
struct GatedGrad {
  const void* dh;
  int64_t dh_worker, dh_row;
  const float* pre;
  void *da, *db;
  int64_t rows, F, pitch;
  bool vec;                 // rows of dh start on 16-byte boundaries, F is a multiple of 8
  Border border;            // relu
  float* maxima;            // fp16: the largest value of each CTA [m][CTAs] ...
  float* unscale;           // ... and one over the factor of each worker's da and db
};

// One column next to relu's border once more, by a warp; lane `from` stores.
template <typename T>
__device__ __forceinline__ void settle(const GatedGrad& g, int64_t worker, int64_t r, int64_t col, bool zero, int from, float scale) {
  const Border& o = g.border;
  const T* x = static_cast<const T*>(o.x.p) + worker * o.x.worker_stride + r * o.x.row_stride;
  const T* w = static_cast<const T*>(o.wg.p) + worker * o.wg.worker_stride + col * o.wg.row_stride;
  const int64_t wr = worker * g.rows + r;
  const float d = Elem<T>::to_float(__ldcg(static_cast<const T*>(g.dh) + worker * g.dh_worker + r * g.dh_row + col));
  const float b = __ldcg(g.pre + wr * 2 * g.pitch + g.pitch + col);
  // (sparse rows may have no element in common: nothing to add up)
  if (zero && !warp_overlap(x, w, o.D, o.vec)) return;
  const float exact = (float)warp_dot(x, w, o.D, o.vec);
  if ((threadIdx.x & 31) == from) {
    const ActPair p = act_pair<OLSGD_ACT_RELU>(exact);
    static_cast<T*>(g.da)[wr * g.pitch + col] = Elem<T>::from_float(d * b * p.df * scale);
    static_cast<T*>(g.db)[wr * g.pitch + col] = Elem<T>::from_float(d * p.f * scale);
  }
}

// A stretch of kStretch columns of row r, by a warp; da and db times `scale`.  most: the largest of their values (fp16).
// (The loads go past L1: the kernel may run beside its predecessor, see launch_gated_backward.)
template <typename T, int ACT>
__device__ __forceinline__ void form_stretch(const GatedGrad& g, int64_t worker, int64_t r, int64_t j_begin, float scale, float& most) {
  const int lane = threadIdx.x & 31;
  const int64_t wr = worker * g.rows + r;
  float xn = 0.f;
  if constexpr (ACT == OLSGD_ACT_RELU) xn = __ldcg(g.border.xn + wr);
#pragma unroll
  for (int q = 0; q < kStretch / 256; ++q) {
    const int64_t j0 = j_begin + q * 256, j = j0 + lane * 8;
    if (j0 >= g.pitch) break;
    const bool live = j < g.pitch;
    float a[8], b[8], d[8], va[8], vb[8], wn[8];
#pragma unroll
    for (int k = 0; k < 8; k += 4) {
      const float* from = g.pre + wr * 2 * g.pitch + (live ? j : 0) + k;
      Elem<float>::unpack(__ldcg(reinterpret_cast<const uint4*>(from)), a + k);
      Elem<float>::unpack(__ldcg(reinterpret_cast<const uint4*>(from + g.pitch)), b + k);
      if constexpr (ACT == OLSGD_ACT_RELU)
        Elem<float>::unpack(__ldcg(reinterpret_cast<const uint4*>(g.border.wn + worker * g.pitch + (live ? j : 0) + k)), wn + k);
    }
    const T* src = static_cast<const T*>(g.dh) + worker * g.dh_worker + r * g.dh_row + j;
    if (g.vec) {
      Elem<T>::unpack(live ? __ldcg(reinterpret_cast<const uint4*>(src)) : make_uint4(0, 0, 0, 0), d);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = j + e < g.F ? Elem<T>::to_float(__ldcg(src + e)) : 0.f;
    }
    uint32_t mask = 0, zeros = 0;   // next to relu's border; those of them that are 0
    if constexpr (ACT == OLSGD_ACT_RELU) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float near = xn < 0.f && wn[e] < 0.f ? 0.f : fabsf(g.border.bound * xn * wn[e]);
        mask |= (j + e < g.F && near < INFINITY && fabsf(a[e]) < near ? 1u : 0u) << e;
        zeros |= (a[e] == 0.f ? 1u : 0u) << e;
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const ActPair p = act_pair<ACT>(a[e]);
      va[e] = d[e] * b[e] * p.df;
      vb[e] = d[e] * p.f;
      if constexpr (std::is_same<T, __half>::value) {
        // (relu: as if its derivative were 1, as it may turn out to be next to the border)
        const float u = fabsf(ACT == OLSGD_ACT_RELU ? d[e] * b[e] : va[e]), v = fabsf(vb[e]);
        most = fmaxf(most, fmaxf(u < INFINITY ? u : 0.f, v < INFINITY ? v : 0.f));
        va[e] *= scale;
        vb[e] *= scale;
      }
    }
    if (live) {
      *reinterpret_cast<uint4*>(static_cast<T*>(g.da) + wr * g.pitch + j) = Elem<T>::pack(va);
      *reinterpret_cast<uint4*>(static_cast<T*>(g.db) + wr * g.pitch + j) = Elem<T>::pack(vb);
    }
    if constexpr (ACT == OLSGD_ACT_RELU) {
      // those next to the border again, after what their lane has stored
      for (uint32_t lanes = __ballot_sync(0xffffffffu, mask != 0); lanes; lanes &= lanes - 1) {
        const int from = __ffs(lanes) - 1;
        const uint32_t zero = __shfl_sync(0xffffffffu, zeros, from);
        for (uint32_t bits = __shfl_sync(0xffffffffu, mask, from); bits; bits &= bits - 1) {
          const int e = __ffs(bits) - 1;
          settle<T>(g, worker, r, j0 + from * 8 + e, (zero >> e) & 1, from, scale);
        }
      }
    }
  }
}

__device__ __forceinline__ float block_max(float v) {
  __shared__ float sh[8];
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  if ((threadIdx.x & 31) == 0) sh[threadIdx.x >> 5] = v;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < 8; ++w) v = fmaxf(v, sh[w]);
  return v;
}

// A warp per stretch.  (relu's border takes registers: with 48 of them some are spilled, 1 us of 16 workers' pass.)
template <typename T, int ACT>
__global__ void __launch_bounds__(256, ACT == OLSGD_ACT_RELU ? 4 : 5) gated_backward_kernel(const __grid_constant__ GatedGrad g, bool beside) {
  if (!beside) launch_gate();
  const int64_t stretches = (g.pitch + kStretch - 1) / kStretch;
  const int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5), r = at / stretches;
  float most = 0.f;
  if (r < g.rows) form_stretch<T, ACT>(g, blockIdx.y, r, (at - r * stretches) * kStretch, 1.f, most);
  if (beside) launch_gate();
  if constexpr (std::is_same<T, __half>::value) {
    most = block_max(most);
    if (threadIdx.x == 0) g.maxima[(int64_t)blockIdx.y * gridDim.x + blockIdx.x] = most;
  }
}

// fp16 ends at 65504 and 2^-24, where the sums over F and T that follow would still be values.  The largest value of a worker's
// da and db decides: from 2^-4 to 2^15 they stay as they are (what is below 2^-14, rounded to steps of 2^-24, is off by
// 2^-21 of the largest then).  Otherwise they are formed again times the power of two that brings the largest to
// [2^14, 2^15): 29 binary orders below it keep all their bits, and the products are scaled back in fp32 before they are
// rounded.  A backward pass takes 4 to 8 us longer for it with nothing to scale (16 workers, 128 tokens, 1024 -> 1024: 44.0 ->
// 48.5 us; 3 workers, 333 tokens, 1021 -> 2035: 55.5 -> 63), and 53 and 70 us where everything is scaled.
__device__ __forceinline__ float scale_for(float most) {
  if (most == 0.f || (most >= 0.0625f && most < 32768.f)) return 1.f;
  const int k = 14 - ((int)(__float_as_uint(most) >> 23) - 127);
  return __uint_as_float((uint32_t)(127 + (k < 120 ? k : 120)) << 23);
}
template <int ACT>
__global__ void __launch_bounds__(256, ACT == OLSGD_ACT_RELU ? 4 : 5) gated_rescale_kernel(const __grid_constant__ GatedGrad g, int64_t maxima) {
  launch_gate();
  const int64_t worker = blockIdx.y, stretches = (g.pitch + kStretch - 1) / kStretch;
  float most = 0.f;
#pragma unroll 8
  for (int64_t i = threadIdx.x; i < maxima; i += 256) most = fmaxf(most, g.maxima[worker * maxima + i]);
  const float scale = scale_for(block_max(most));
  if (blockIdx.x == 0 && threadIdx.x == 0) g.unscale[worker] = 1.f / scale;
  if (scale == 1.f) return;
  for (int64_t at = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5); at < g.rows * stretches; at += (int64_t)gridDim.x * 8) {
    const int64_t r = at / stretches;
    form_stretch<__half, ACT>(g, worker, r, (at - r * stretches) * kStretch, scale, most);
  }
}

// --------------------------------------------------------------------------------- host
template <int MODE, int CTAS, int BN, int STAGES, bool SCALED>
cudaError_t launch_variant(const GatedMaps& maps, GatedArgs g, cudaStream_t s) {
  constexpr int kColsOut = MODE == FORWARD ? BN / 2 : BN;
  constexpr size_t smem = (size_t)STAGES * (kBM * kBK * 2 + BN / CTAS * kBK * 2) +
                          kEpiWarps * 4096 + sizeof(Control<STAGES>) + 1024;
  static_assert(smem <= 227 * 1024, "shared memory of one CTA");
  static PerDeviceSmem configured;
  auto kern = gated_gemm_kernel<MODE, CTAS, BN, STAGES, SCALED>;
  cudaError_t e = ensure_dynamic_smem(configured, kern, smem);
  if (e != cudaSuccess) return e;
  g.row_tiles = (g.rows + CTAS * kBM - 1) / (CTAS * kBM);
  g.col_tiles = (g.cols + kColsOut - 1) / kColsOut;
  const int64_t total = (int64_t)g.problems * g.splits * g.row_tiles * g.col_tiles;
  const int64_t room = sm_count() / CTAS;
  const unsigned ctas = (unsigned)((total < room ? total : room) * CTAS);
  g_tc_launches += 1;
  if (CTAS == 1) return launch_chained(kern, dim3(ctas), dim3(kThreads), smem, s, maps, g);
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = 2;
  attr[0].val.clusterDim.y = 1;
  attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = g_launch_overlap ? 2 : 1;
  return cudaLaunchKernelEx(&cfg, kern, maps, g);
}

// Which tiles, and into how many parts K is cut.  A tile's time goes by the operand bytes that one
// CTA takes in per K block (128 rows of A and BN / CTAS rows of B), plus an epilogue that is not
// hidden in the last wave; the launch takes as many waves as its tiles need.  Where tiles are few
// and K is long, the parts' sums go through the workspace and a joining launch, which costs
// about as much as 12 K blocks of 256 rows and the traffic.  The least sum is taken: pairs for
// large problems, narrower tiles and parts of K where multiprocessors would be idle.  One worker,
// 512 tokens, 1024 <- 2 x 4096 (element-wise pass and DX): 24 us in eight parts, 47 us uncut.
// (Sizes alone decide, so that the workspace can be asked for anywhere.)
constexpr int kSms = 148;
constexpr int kMaxSplits = 16;
struct Shape {
  int ctas, bn, splits;
};
struct Product {
  int64_t problems, rows, cols, num_kb;
};
template <int MODE>
Shape shape_for(const Product& d) {
  constexpr Shape shapes[] = {{1, 64, 1}, {1, 128, 1}, {1, 256, 1}, {2, 256, 1}};
  Shape best = shapes[0];
  double least = 1e300;
  for (const Shape& sh : shapes) {
    const int64_t cols = MODE == FORWARD ? sh.bn / 2 : sh.bn;
    const int64_t tiles = d.problems * ((d.rows + sh.ctas * kBM - 1) / (sh.ctas * kBM)) * ((d.cols + cols - 1) / cols);
    const int64_t room = kSms / sh.ctas;
    for (int splits = 1; splits <= kMaxSplits && (splits == 1 || d.num_kb >= 4 * splits); splits *= 2) {
      const int64_t waves = (tiles * splits + room - 1) / room, kbs = (d.num_kb + splits - 1) / splits;
      double cost = (double)waves * (kbs + 4) * (kBM + sh.bn / sh.ctas);
      // the parts are written and read: 8 bytes an element at 6 bytes a picosecond, 900 rows a us
      if (splits > 1)
        cost += 3000.0 + splits * (double)d.problems * d.rows * d.cols * (MODE == FORWARD ? 2 : 1) * 8 / 6.0e6 * 900;
      if (cost < least) {
        least = cost;
        best = Shape{sh.ctas, sh.bn, splits};
      }
    }
  }
  return best;
}

Product product_of(int mode, const GatedShape& d) {
  const auto kbs = [](int64_t k) { return (k + kBK - 1) / kBK; };
  if (mode == FORWARD) return Product{d.m, d.T, d.F, kbs(d.D)};
  if (mode == DX) return Product{d.m, d.T, d.D, 2 * kbs(d.F)};
  return Product{2 * d.m, d.F, d.D, kbs(d.T)};
}
template <int MODE>
size_t parts_bytes(const GatedShape& d) {
  const Product p = product_of(MODE, d);
  const int splits = shape_for<MODE>(p).splits;
  return splits == 1 ? 0 : (size_t)splits * p.problems * p.rows * round8(p.cols) * (MODE == FORWARD ? 2 : 1) * sizeof(float);
}
// What shape_for decided, in the launch's arguments.
template <int MODE>
GatedArgs args_for(const GatedShape& d, const Shape& sh, uint8_t* parts) {
  const Product p = product_of(MODE, d);
  GatedArgs g{};
  g.num_kb = (int)p.num_kb;
  g.kb_half = (int)(p.num_kb / 2);
  g.problems = (int)p.problems;
  g.rows = (int)p.rows;
  g.cols = (int)p.cols;
  g.act = d.act;
  g.f16 = d.f16;
  g.pre_pitch = round8(p.cols);
  g.splits = sh.splits;
  g.kb_split = (int)((p.num_kb + sh.splits - 1) / sh.splits);
  g.splits = (int)((p.num_kb + g.kb_split - 1) / g.kb_split);   // none is empty
  g.parts = reinterpret_cast<float*>(parts);
  g.parts_row = (MODE == FORWARD ? 2 : 1) * round8(p.cols);
  return g;
}

template <int MODE, bool SCALED>
cudaError_t launch_shape(const Shape& sh, const GatedMaps& maps, const GatedArgs& g, cudaStream_t s) {
  return sh.bn == 64    ? launch_variant<MODE, 1, 64, 8, SCALED>(maps, g, s)
         : sh.bn == 128 ? launch_variant<MODE, 1, 128, 6, SCALED>(maps, g, s)
         : sh.ctas == 2 ? launch_variant<MODE, 2, 256, 6, SCALED>(maps, g, s)
                        : launch_variant<MODE, 1, 256, 4, SCALED>(maps, g, s);
}
template <int MODE>
cudaError_t launch_product(const Shape& sh, const GatedMaps& maps, const GatedArgs& g, cudaStream_t s) {
  if constexpr (MODE != FORWARD)
    if (g.unscale) return launch_shape<MODE, true>(sh, maps, g, s);
  return launch_shape<MODE, false>(sh, maps, g, s);
}
// Where K was cut: the joining launch.
template <int MODE>
cudaError_t launch_join(const GatedArgs& g, cudaStream_t s) {
  if (g.splits == 1) return cudaSuccess;
  const int64_t width = MODE == FORWARD ? g.pre_pitch : g.parts_row, warps = g.rows * ((width + 255) / 256);
  return launch_chained(g.f16 ? gated_join_kernel<__half, MODE> : gated_join_kernel<__nv_bfloat16, MODE>,
                        dim3((unsigned)((warps + 7) / 8), (unsigned)g.problems), dim3(256), 0, s, g);
}

// Rows of A worth loading: with fewer than 128 tokens the rest of the tile stays what it was (it
// reaches only accumulator rows that are not stored).
int loaded_rows(int64_t T) { return T >= kBM ? kBM : (int)round8(T); }

// relu: norms of the rows of x and w_gate.
template <typename T>
cudaError_t row_norms(const GatedBackward& a, int64_t pitch, float* xn, float* wn, cudaStream_t s) {
  const int64_t most = a.T > a.F ? a.T : a.F;
  return launch_chained(row_norms_kernel<T>, dim3((unsigned)((most + 7) / 8), (unsigned)a.m, 2), dim3(256), 0, s, a.x, a.wg, a.T, a.F, a.D,
                        xn, wn, pitch);
}

int64_t elementwise_ctas(int64_t T, int64_t pitch) { return (T * ((pitch + kStretch - 1) / kStretch) + 7) / 8; }

template <typename T>
cudaError_t elementwise(const GatedBackward& a, GatedGrad g, bool beside, cudaStream_t s) {
  const int64_t ctas = elementwise_ctas(a.T, g.pitch);
  g.dh = a.dh.p;
  g.dh_worker = a.dh.worker_stride;
  g.dh_row = a.dh.row_stride;
  g.pre = a.pre;
  g.rows = a.T;
  g.F = a.F;
  g.vec = a.F % 8 == 0 && tma_ready(a.dh, a.T, a.m);
  g.border.x = a.x;
  g.border.wg = a.wg;
  g.border.D = a.D;
  g.border.vec = a.D % 8 == 0 && tma_ready(a.x, a.T, a.m) && tma_ready(a.wg, a.F, a.m);
  g.border.bound = (8.f + (float)a.D / 128) / (1 << 23);
  auto k = a.act == OLSGD_ACT_SILU   ? gated_backward_kernel<T, OLSGD_ACT_SILU>
           : a.act == OLSGD_ACT_GELU ? gated_backward_kernel<T, OLSGD_ACT_GELU>
           : a.act == OLSGD_ACT_RELU ? gated_backward_kernel<T, OLSGD_ACT_RELU>
                                     : gated_backward_kernel<T, OLSGD_ACT_SIGMOID>;
  const cudaError_t e = launch_chained(k, dim3((unsigned)ctas, (unsigned)a.m), dim3(256), 0, s, g, beside);
  if (e != cudaSuccess || !std::is_same<T, __half>::value) return e;
  auto again = a.act == OLSGD_ACT_SILU   ? gated_rescale_kernel<OLSGD_ACT_SILU>
               : a.act == OLSGD_ACT_GELU ? gated_rescale_kernel<OLSGD_ACT_GELU>
               : a.act == OLSGD_ACT_RELU ? gated_rescale_kernel<OLSGD_ACT_RELU>
                                         : gated_rescale_kernel<OLSGD_ACT_SIGMOID>;
  const int64_t room = 4 * kSms / a.m < 1 ? 1 : 4 * kSms / a.m;   // every CTA reads its worker's maxima
  return launch_chained(again, dim3((unsigned)(ctas < room ? ctas : room), (unsigned)a.m), dim3(256), 0, s, g, ctas);
}

template <typename T>
cudaError_t few(const GatedForward& a, cudaStream_t s) {
  const bool vec = a.D % 8 == 0 && tma_ready(a.x, a.T, a.m) && tma_ready(a.wg, a.F, a.m) && tma_ready(a.wu, a.F, a.m);
  auto k = a.T == 1 ? (vec ? gated_few_kernel<T, 1, true> : gated_few_kernel<T, 1, false>)
                    : (vec ? gated_few_kernel<T, kFewTokens, true> : gated_few_kernel<T, kFewTokens, false>);
  return launch_chained(k, dim3((unsigned)((a.F + 7) / 8), (unsigned)a.m), dim3(256), 0, s, a.x, a.wg, a.wu, (int)a.T, a.D, a.F,
                        a.act, static_cast<T*>(a.h), a.pre, round8(a.F));
}

#define OLSGD_STEP(call)                    \
  do {                                      \
    const cudaError_t e_ = (call);          \
    if (e_ != cudaSuccess) return e_;       \
  } while (0)

}  // namespace

// The workspace: copies of operands that TMA cannot take, then (backward) da and db, the norms of the rows of x and w_gate,
// the largest values and the factors, then the parts of the products (backward: dx, then the weights' gradients, which run
// side by side).
struct Workspace {
  size_t da, db, xn, wn, maxima, unscale, parts, parts_dw, total;
};
Workspace layout(const GatedShape& d, bool backward, bool copies) {
  Workspace w{};
  w.da = copies ? round256((size_t)d.m * d.T * round8(d.D) * 2) + 2 * round256((size_t)d.m * d.F * round8(d.D) * 2) : 0;
  const size_t part = backward ? round256((size_t)d.m * d.T * round8(d.F) * 2) : 0;
  w.db = w.da + part;
  w.xn = w.db + part;
  w.wn = w.xn + (backward ? round256((size_t)d.m * d.T * sizeof(float)) : 0);
  w.maxima = w.wn + (backward ? round256((size_t)d.m * round8(d.F) * sizeof(float)) : 0);
  w.unscale = w.maxima + (backward ? round256((size_t)d.m * elementwise_ctas(d.T, round8(d.F)) * sizeof(float)) : 0);
  w.parts = w.unscale + (backward ? round256((size_t)d.m * sizeof(float)) : 0);
  w.parts_dw = w.parts + (backward ? round256(parts_bytes<DX>(d)) : 0);
  w.total = w.parts_dw + (backward ? parts_bytes<DW>(d) : parts_bytes<FORWARD>(d));
  return w;
}

size_t gated_workspace(const GatedShape& d, bool backward, bool copies) {
  if (!backward && d.T <= kFewTokens) return 0;
  return layout(d, backward, copies).total;
}

bool gated_needs_copies(const GatedShape& d, const GatedOperand& x, const GatedOperand& wg, const GatedOperand& wu) {
  return !tma_ready(x, d.T, d.m) || !tma_ready(wg, d.F, d.m) || !tma_ready(wu, d.F, d.m);
}

cudaError_t launch_gated_forward(GatedForward a, cudaStream_t s) {
  if (a.T <= kFewTokens) return a.f16 ? few<__half>(a, s) : few<__nv_bfloat16>(a, s);
  uint8_t* ws = static_cast<uint8_t*>(a.ws);
  const Workspace at = layout(a, false, gated_needs_copies(a, a.x, a.wg, a.wu));
  const Wanted wanted[] = {{&a.x, a.T}, {&a.wg, a.F}, {&a.wu, a.F}};
  OLSGD_STEP(make_ready(wanted, 3, a.D, a.m, ws, s));
  const Shape sh = shape_for<FORWARD>(product_of(FORWARD, a));
  GatedArgs g = args_for<FORWARD>(a, sh, ws + at.parts);
  g.out_width = store_width(a.h, a.F);
  g.out0 = a.h;
  g.pre = a.pre;
  g.a_rows = loaded_rows(a.T);
  GatedMaps maps;
  const int b_rows = sh.bn / 2;
  if (!make_map16(&maps.a0, a.x, a.D, a.T, a.m, g.a_rows, a.f16) || !make_map16(&maps.b0, a.wg, a.D, a.F, a.m, b_rows, a.f16) ||
      !make_map16(&maps.b1, a.wu, a.D, a.F, a.m, b_rows, a.f16))
    return cudaErrorInvalidValue;
  maps.a1 = maps.a0;
  OLSGD_STEP(launch_product<FORWARD>(sh, maps, g, s));
  return launch_join<FORWARD>(g, s);
}

cudaError_t launch_gated_backward(GatedBackward a, cudaStream_t s) {
  const int64_t pitch = round8(a.F);
  uint8_t* ws = static_cast<uint8_t*>(a.ws);
  const Workspace at = layout(a, true, gated_needs_copies(a, a.x, a.wg, a.wu));
  void *da = ws + at.da, *db = ws + at.db;
  const Wanted wanted[] = {{&a.x, a.T}, {&a.wg, a.F}, {&a.wu, a.F}};   // x for the weights' gradients, the weights for dx
  const int from = a.dwg ? 0 : 1, to = a.dx ? 3 : 1;
  // The element-wise kernel needs none of the copies: where there are any it runs beside them (as the second product
  // does below), on the operands as they were given.  3 workers, 333 tokens, 1021 -> 2035: backward 56.5 -> 54.9 us; one
  // worker, 40 tokens, 333 -> 1003: 12.7 -> 11.9.  relu's norms come ahead of both.
  const GatedBackward given = a;
  const auto floats = [&](size_t offset) { return reinterpret_cast<float*>(ws + offset); };
  if (a.act == OLSGD_ACT_RELU)
    OLSGD_STEP(a.f16 ? row_norms<__half>(a, pitch, floats(at.xn), floats(at.wn), s) : row_norms<__nv_bfloat16>(a, pitch, floats(at.xn), floats(at.wn), s));
  bool copies = false;
  OLSGD_STEP(make_ready(wanted + from, to - from, a.D, a.m, ws, s, &copies));
  GatedGrad grad{};
  grad.da = da;
  grad.db = db;
  grad.pitch = pitch;
  grad.border.xn = floats(at.xn);
  grad.border.wn = floats(at.wn);
  grad.maxima = floats(at.maxima);
  grad.unscale = floats(at.unscale);
  OLSGD_STEP(a.f16 ? elementwise<__half>(given, grad, copies, s) : elementwise<__nv_bfloat16>(given, grad, copies, s));
  const GatedOperand oa{da, a.T * pitch, pitch}, ob{db, a.T * pitch, pitch};
  // Both products read what the element-wise kernel has written, and neither what the other writes.  The
  // second one is launched beside the first: its CTAs may start once all of the first one's have
  // passed their gate (the element-wise kernel, and all before it, have completed then), it takes the
  // multiprocessors as they become free, and at its end it waits for the first.  The joining
  // launches come after both.
  GatedArgs dx{}, dw{};
  if (a.dx) {
    const Shape sh = shape_for<DX>(product_of(DX, a));
    dx = args_for<DX>(a, sh, ws + at.parts);
    dx.out_width = store_width(a.dx, a.D);
    dx.out0 = a.dx;
    dx.unscale = a.f16 ? grad.unscale : nullptr;
    dx.a_rows = loaded_rows(a.T);
    GatedMaps maps;
    if (!make_map16(&maps.a0, oa, a.F, a.T, a.m, dx.a_rows, a.f16) || !make_map16(&maps.a1, ob, a.F, a.T, a.m, dx.a_rows, a.f16) ||
        !make_map16(&maps.b0, a.wg, a.D, a.F, a.m, kBK, a.f16) || !make_map16(&maps.b1, a.wu, a.D, a.F, a.m, kBK, a.f16))
      return cudaErrorInvalidValue;
    OLSGD_STEP(launch_product<DX>(sh, maps, dx, s));
  }
  if (a.dwg) {
    const Shape sh = shape_for<DW>(product_of(DW, a));
    dw = args_for<DW>(a, sh, ws + at.parts_dw);
    dw.beside = a.dx != nullptr;
    const int w0 = store_width(a.dwg, a.D), w1 = store_width(a.dwu, a.D);
    dw.out_width = w0 < w1 ? w0 : w1;
    dw.out0 = a.dwg;
    dw.out1 = a.dwu;
    dw.unscale = a.f16 ? grad.unscale : nullptr;
    GatedMaps maps;
    if (!make_map16(&maps.a0, oa, a.F, a.T, a.m, kBK, a.f16) || !make_map16(&maps.a1, ob, a.F, a.T, a.m, kBK, a.f16) ||
        !make_map16(&maps.b0, a.x, a.D, a.T, a.m, kBK, a.f16))
      return cudaErrorInvalidValue;
    maps.b1 = maps.b0;
    OLSGD_STEP(launch_product<DW>(sh, maps, dw, s));
  }
  if (a.dx) OLSGD_STEP(launch_join<DX>(dx, s));
  if (a.dwg) OLSGD_STEP(launch_join<DW>(dw, s));
  return cudaSuccess;
}

cudaError_t operators_status(int* status, cudaStream_t s) {
  OLSGD_STEP(cudaStreamSynchronize(s));
  OLSGD_STEP(cudaMemcpyFromSymbol(status, g_operator_status, sizeof(int)));
  if (*status != 0) {
    const int zero = 0;
    OLSGD_STEP(cudaMemcpyToSymbol(g_operator_status, &zero, sizeof(int)));
  }
  return cudaSuccess;
}

cudaError_t status_word(int** word) {
  static std::atomic<int*> known[kMaxDevices];   // (the same address, whoever comes first)
  const int dev = current_device();
  if (dev >= 0 && dev < kMaxDevices && (*word = known[dev].load())) return cudaSuccess;
  void* p = nullptr;
  OLSGD_STEP(cudaGetSymbolAddress(&p, g_operator_status));
  *word = static_cast<int*>(p);
  if (dev >= 0 && dev < kMaxDevices) known[dev].store(*word);
  return cudaSuccess;
}

}  // namespace olsgd
