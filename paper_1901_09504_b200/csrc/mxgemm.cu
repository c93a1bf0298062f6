// ocs_qlinear_mx4 / ocs_linear_mx4: the layer on block-scaled 4-bit codes,
//     Y[m][n] = a[m] w[n] sum_k (A[m][k] sa[m][k / B]) (W[n][k] sw[n][k / B]) + bias[n],   B = 32 (E8M0) or 16 (E4M3),
// by tcgen05's block-scaled products: the codes and their scales go to the tensor cores as they are stored, at four times the
// rate of 16-bit operands, and sums are fp32.  The rows' own scales (E4M3, powers of two) and the bias come in the epilogue.
//
// Layout as in the int8 row product: the weights are the rows of the tensor-core tile (128 channels, the lanes of tensor
// memory), the tokens its columns, so that few tokens cost a narrow tile.  A K-block is 256 contraction indices: 128 bytes of
// codes a row (one swizzle span, by TMA) and 2 or 4 pieces of 512 scale bytes per 128 rows, which have to be spread over tensor
// memory ahead of the products that read them.  tcgen05.cp would do that, in order with the products and in the tensor cores'
// time: some 45 cycles a piece, 12 pieces (E4M3, 256 tokens) for 512 cycles of products.  Four warps move them through
// registers instead, while the products before them run.
// Forms: 16, 32, 64 or 128 tokens per CTA, or 256 by a pair of CTAs (256 channels, each CTA stages half the tokens); few tiles:
// 2, 4 or 8 CTAs of a cluster split the contraction and exchange their partial sums through distributed shared memory.
//
// What bounds it (device times by graph replay; the floor is the larger of the bytes at 6.54 TB/s, the measured copy rate, and
// the operations at 6.43 PFLOP/s, four times the measured bf16 rate):
// M x K x N
//   8192 x 8192 x 8192, bf16 out   E4M3 227 us, E8M0 213 us (floor 171): operand tiles; a K-block is 38 (35) KB a CTA, and five
//                                  (six) of them in flight bring 82 GB/s an SM; without any scales 228 and 208 us, and one pair
//                                  alone takes a K-block in 0.36 (0.34) us where its products alone would be 0.28
//   2047 x 4178 x 4096, bf16 out   23.0 us (floor 10.9): two waves of tiles, the second three quarters full
//   128 x 25339 x 4096, fp32 out   21.5 us (floor 9.5): one wave of 128 CTAs with a tile each: start (4 us), exchange and end (4)
//   700 x 663 x 33278, fp32 out    36 us (floor 16): writing (93 MB in this pattern alone take 23 us, 19 where rows start at
//                                  32-byte boundaries; 8 warps and 16 stores a piece are enough for that), and the
//                                  stores and the operand requests share the SM's way out; 20 us without the stores
//   1 x 8192 x 8192, bf16          12.5 us (floor 5.8): HBM after 3 us of start, the exchange and the end
#include <atomic>

#include "mx4.cuh"
#include "ptx.cuh"

namespace ocs {
namespace {

constexpr int TW = 128;        // channels of one CTA's tile
constexpr int KB = 128;        // bytes of a K-block's row: 256 contraction indices
constexpr int kEpiWarps = 8;
constexpr int kFusedBytes = 64 * 1024;             // token codes and scales a CTA can hold beside the ring of weights
constexpr int kTailBytes = 8 * 1024;               // ... and what its rows have behind their last whole block
constexpr int kThreads = 64 + 32 * kEpiWarps + 128;   // copy warp, tensor-core warp, epilogue warps, scale warps
constexpr int kTokenThreads = kThreads - 64;          // that quantize tokens (FUSED): all but the first two

__host__ __device__ constexpr int stage_blocks(int tn) { return tn <= 64 ? 2 : 1; }   // K-blocks of a ring stage

struct MxGemm {
  int M, N, num_st;              // num_st: stages' worth of contraction
  int n_tiles, m_tiles, total, slices;
  const float* a_scales;         // of rows (NULL: 1)
  const float* w_scales;
  const float* bias;
  long long ldy;
  int* dev_status;
  // tokens that are quantized here (FUSED): unquantized rows and what ocs_quantize_mx4 takes
  const void* X;
  long long ldx;
  const int32_t* idx_map;
  int x_type, C, K;
};

// Tensor memory columns: two accumulators, then the scales of two stages.  256 tokens: the accumulators overlap by as many
// columns as the scales need; the epilogue empties those first and says so before it goes on.
template <int GRID, int TN, int CG, bool FUSED>
struct MxSmem {
  static constexpr int kTokens = TN / CG;
  static constexpr int kPieces = GRID == OCS_GRID_E8M0 ? 2 : 4;        // groups of four blocks in a K-block
  static constexpr int kTiles = TN > 128 ? 2 : 1;                       // 128-token scale tiles
  static constexpr int kWBytes = TW * KB, kTBytes = FUSED ? 0 : kTokens * KB;
  static constexpr int kSWBytes = kPieces * kMxTile, kSTBytes = FUSED ? 0 : kTiles * kPieces * kMxTile;
  static constexpr int kSub = stage_blocks(TN);
  static constexpr int kStageBytes = kSub * (kWBytes + kTBytes + kSWBytes + kSTBytes);
  static constexpr int kAtT = kSub * kWBytes, kAtSW = kAtT + kSub * kTBytes, kAtST = kAtSW + kSub * kSWBytes;
  static constexpr int kXBytes = TN == 256 ? 0 : TN * TW * 4;           // partial sums of a K split
  static constexpr bool kXInRing = TN == 128;
  static constexpr int kXExtra = kXInRing ? 0 : kXBytes;
  static constexpr int kWarpTokens = TN < 32 ? 16 : TN / 2;
  static constexpr int kScaleBytes = kEpiWarps * kWarpTokens * 4;
  // FUSED: the codes of all the K-blocks a CTA takes, [K-block][token][128 bytes], their scales, [K-block][32 tokens][16
  // bytes, one per block], a row's maximum and its scale
  static constexpr int kFusedBlocks = FUSED ? kFusedBytes / (TN * KB + kMxTile) : 0, kTokenBytes = FUSED ? kFusedBlocks * (TN * KB + kMxTile) : 0;
  static constexpr int kRowBytes = FUSED ? TN * 8 + kTailBytes : 0;
  static constexpr int kCtrlBytes = 512;
  static constexpr int kBudget = 227 * 1024 - 1024 - kCtrlBytes - kScaleBytes - kXExtra - kTokenBytes - kRowBytes;
  static constexpr int kStages = kBudget / kStageBytes < 8 ? kBudget / kStageBytes : 8;
  static constexpr int kDynBytes = 1024 + kStages * kStageBytes + kTokenBytes + kXExtra + kScaleBytes + kRowBytes + kCtrlBytes;
  static constexpr bool kOverlap = TN == 256;
  static constexpr int kScaleCols = 4 * kPieces * (1 + kTiles), kStageCols = kSub * kScaleCols;   // the weights' scales, then the tokens'
  static constexpr int kAccStride = kOverlap ? 512 - 2 * kStageCols - TN : (TN < 32 ? 32 : TN);
  static constexpr int kShared = kOverlap ? TN - kAccStride : 0;             // columns of both accumulators
  static constexpr int kScaleCol = kAccStride + (kOverlap ? TN : kAccStride);
  static constexpr int kUsedCols = kScaleCol + 2 * kStageCols;
  static constexpr uint32_t kFullTx = kSub * (kWBytes + kTBytes), kScaleTx = kSub * (kSWBytes + kSTBytes);   // a stage's bytes on its two barriers
  static constexpr uint32_t kTmemCols = kUsedCols <= 128 ? 128 : (kUsedCols <= 256 ? 256 : 512);
  static_assert(kStages >= 3 && (!kXInRing || kXBytes <= kStages * kStageBytes) && kStageBytes % 1024 == 0 && kTBytes % 1024 == 0 && (TN * KB) % 1024 == 0 && kUsedCols <= 512, "tile does not fit");
};

// Instruction descriptor of the block-scaled 4-bit products: e2m1 operands, K-major, scales e8m0 or e4m3.  sf: which bytes
// of the scales' 32-bit cells (0, or 2 for the second half where an instruction takes two).
__host__ __device__ constexpr uint32_t mx_instr_desc(int grid, int m, int n, int sf) {
  return ((uint32_t)sf << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(grid == OCS_GRID_E8M0 ? 1 : 0) << 23) | ((uint32_t)(m >> 4) << 24) | ((uint32_t)sf << 29);
}

template <int GRID, int CG>
__device__ __forceinline__ void umma_mx4(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t sa, uint32_t sb, uint32_t accumulate) {
#define OCS_MX4_MMA(cg, kind)                                                                             \
  asm volatile(                                                                                           \
      "{\n\t.reg .pred p;\n\t"                                                                            \
      "setp.ne.b32 p, %6, 0;\n\t"                                                                         \
      "tcgen05.mma.cta_group::" cg "." kind " [%0], %1, %2, %3, [%4], [%5], p;\n\t}"                      \
      ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(sa), "r"(sb), "r"(accumulate) : "memory")
  if constexpr (GRID == OCS_GRID_E8M0) {
    if constexpr (CG == 1) OCS_MX4_MMA("1", "kind::mxf4.block_scale.scale_vec::2X");
    else OCS_MX4_MMA("2", "kind::mxf4.block_scale.scale_vec::2X");
  } else {
    if constexpr (CG == 1) OCS_MX4_MMA("1", "kind::mxf4nvf4.block_scale.scale_vec::4X");
    else OCS_MX4_MMA("2", "kind::mxf4nvf4.block_scale.scale_vec::4X");
  }
#undef OCS_MX4_MMA
}

// N columns of a warp's quarter of the lanes.
template <int N>
__device__ __forceinline__ void tmem_store(uint32_t taddr, const uint32_t* v) {
  static_assert(N == 8 || N == 16, "columns");
  if constexpr (N == 8)
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
  else
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(taddr), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]),
                   "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]) : "memory");
}

__device__ __forceinline__ void tma_load_scales(uint32_t dst, const CUtensorMap* map, uint32_t bar, int piece, int tile) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%3, %4, %5}], [%2];"
      ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(bar), "r"(0), "r"(piece), "r"(tile) : "memory");
}

// The bounded waits for a whole warp: all lanes go on, or all give up.
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag));
}
__device__ __forceinline__ bool warp_wait_cluster(uint32_t bar, uint32_t parity, volatile int* abort_flag) {
  return __all_sync(0xffffffffu, mbar_wait_cluster(bar, parity, abort_flag));
}

// Tile t of the launch: token tiles in groups of eight, all channel tiles of a group before the next group, so that the tiles
// in flight at one time share their operand panels in L2.
__device__ __forceinline__ void tile_of(const MxGemm& p, int t, int* mt, int* nt) {
  const int per_group = 8 * p.n_tiles;
  const int g = t / per_group, in = t - g * per_group;
  const int rows = min(8, p.m_tiles - 8 * g);
  *nt = in / rows;
  *mt = 8 * g + in - *nt * rows;
}

template <typename T> struct Pair;
template <> struct Pair<__half> { static __device__ __forceinline__ uint32_t pack(float a, float b) { __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); } };
template <> struct Pair<__nv_bfloat16> { static __device__ __forceinline__ uint32_t pack(float a, float b) { __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); } };

// One output: the sum times two powers of two (the token's first), plus the bias, rounded once.  The first product is exact
// downward: sums are multiples of 2^-20 and scales at least 2^-117, so it is a multiple of 2^-137.  Upward it stays in fp32's
// range for scales up to kNearScale, as sums are below 2^50 (K < 2^27 products of at most 2688^2); where a warp's tokens have
// larger ones (E4M3 rows of 2^88 and more), near_sums goes before it.
constexpr float kNearScale = 0x1p77f;
__device__ __forceinline__ float one_output(uint32_t acc, float as, float ws, float b) {
  return fmaf(__fmul_rn(__uint_as_float(acc), as), ws, b);
}
// The sums times the channel's scale if that makes them smaller (exact, as above), so that the product with the token's is too
// large for fp32 only where the output is; the scale that is left then: at least 1.  (The smaller scale of the two first in every
// case costs the 16-bit epilogue 4 to 7 %.)
template <int CNT>
__device__ __forceinline__ void near_sums(uint32_t* acc, float ws) {
#pragma unroll
  for (int i = 0; i < CNT; ++i) acc[i] = __float_as_uint(__fmul_rn(__uint_as_float(acc[i]), fminf(ws, 1.0f)));
}
__device__ __forceinline__ float scale_left(float ws) { return fmaxf(ws, 1.0f); }

// CNT consecutive tokens of one channel per lane, rounded to T and stored; the lanes of the warp hold consecutive channels.
// at: the element offset of the lane's channel of the first token; left: tokens that exist, from the first on.  WHOLE: all
// CNT tokens and all 32 channels exist.
template <bool WHOLE, typename T, int CNT>
__device__ __forceinline__ void finish(T* y, long long ldy, const uint32_t* acc, const float* sc, float ws, float b, int left,
                                       bool n_ok, bool pairs) {
  if constexpr (sizeof(T) == 2) {
    if (pairs) {
      // neighbouring lanes swap halves, so that a lane stores two channels of one token in 32 bits
      const int odd = threadIdx.x & 1;
      T* q = y + (odd ? ldy - 1 : 0);
#pragma unroll
      for (int j = 0; j < CNT; j += 2) {
        const uint32_t mine = Pair<T>::pack(one_output(acc[j], sc[j], ws, b), one_output(acc[j + 1], sc[j + 1], ws, b));
        const uint32_t other = __shfl_xor_sync(0xffffffffu, mine, 1);
        const uint32_t out = odd ? __byte_perm(other, mine, 0x7632) : __byte_perm(mine, other, 0x5410);
        if (WHOLE || (j + odd < left && n_ok)) *reinterpret_cast<uint32_t*>(q) = out;
        q += 2 * ldy;
      }
      return;
    }
  }
#pragma unroll
  for (int j = 0; j < CNT; ++j) {
    const float f = one_output(acc[j], sc[j], ws, b);
    if (WHOLE || (j < left && n_ok)) *y = from_f32<T>(f);
    y += ldy;
  }
}
// The epilogue and scale warps quantize the token tile (all of the call's M <= TN tokens) into the operand tiles of stages slice,
// slice + slices, ...; E4M3: after the rows' maxima.  A thread's unit of work is a block of a row.  This code runs once per CTA,
// so that fetching the instructions is what it costs besides the loads' latency: nothing is unrolled over units, and both
// passes go through the same load (20 x 650 in fp32 took 15.5 us in all, with two or four units at a time 15.8 and 16).
template <typename X, int GRID, int TN>
__device__ __forceinline__ void quantize_tokens(const MxGemm& p, int slice, int my_kb, unsigned char* tok, unsigned char* scales,
                                                uint32_t* max_bits, float* row_scale, unsigned char* tails) {
  constexpr int N = mx4_block(GRID), PER = 2 * KB / N, kSub = stage_blocks(TN);   // blocks of a K-block
  const int et = threadIdx.x - 64, nb = (p.K + N - 1) / N;
  if (et < TN) {
    max_bits[et] = 0;
    row_scale[et] = 1.0f;
  }
  // what rows have behind their last whole block (its rest and the duplicated channels): a thread per element, so that indices
  // and values each come in one load.  (Gathered by the threads that have the blocks, they cost every pass 2 us a unit.)
  const int whole = p.C / N, tail = (nb - whole) * N;
  const bool staged = tail > 0 && p.M * tail * (int)sizeof(X) <= kTailBytes;
  X* s_tail = reinterpret_cast<X*>(tails);
  if (staged) {
    for (int e = et; e < p.M * tail; e += kTokenThreads) {
      const int r = e / tail;
      int src = whole * N + e - r * tail;
      X v = from_f32<X>(0.0f);
      if (src < p.K) {
        if (src >= p.C) {
          src = __ldg(p.idx_map + src);
          if ((unsigned)src >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); src = 0; }
        }
        v = static_cast<const X*>(p.X)[r * p.ldx + src];
      }
      s_tail[e] = v;
    }
    if (GRID == OCS_GRID_E8M0) asm volatile("bar.sync 1, %0;" ::"n"(kTokenThreads) : "memory");
  }
#pragma unroll 1
  for (int pass = GRID == OCS_GRID_E4M3 ? 0 : 1; pass < 2; ++pass) {
    if (GRID == OCS_GRID_E4M3) asm volatile("bar.sync 1, %0;" ::"n"(kTokenThreads) : "memory");
    if (GRID == OCS_GRID_E4M3 && pass && et < p.M) {
      row_scale[et] = two_to(mx4_row_exponent(max_bits[et]));
      if (max_bits[et] >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
    }
    const int per_row = pass ? my_kb * PER : (staged ? nb : (p.C + N - 1) / N), units = p.M * per_row;
#pragma unroll 1
    for (int u0 = et & ~31; u0 < units; u0 += kTokenThreads) {   // (whole warps)
      const int u = min(u0 + (et & 31), units - 1);   // (the last one more than once: harmless)
      const int r = u / per_row, at = u - r * per_row, in = at / PER, bb = at % PER;   // this CTA's K-block, block in it
      const int b = pass ? ((slice + in / kSub * p.slices) * kSub + in % kSub) * PER + bb : at;
      const X* x = static_cast<const X*>(p.X) + r * p.ldx;
      Block<X, N> v;
      // (the load reads up to 16 bytes around the block: within the matrix)
      if ((b + 1) * N <= p.C && (r > 0 || b > 0) && (r + 1 < p.M || (b + 2) * N <= p.C)) v.template load<0>(x + b * N);
      else if (staged && b >= whole && b < nb) v.from_shared(s_tail + r * tail + (b - whole) * N);
      else if (b < nb) v.gather(x, b * N, p.C, pass ? p.K : p.C, p.idx_map, p.dev_status);
      else v.clear();
      const uint32_t m = v.max_bits();
      if (GRID == OCS_GRID_E4M3 && !pass) {
        const int first = __shfl_sync(0xffffffffu, r, 0);
        if (__all_sync(0xffffffffu, r == first)) {
          const uint32_t all = __reduce_max_sync(0xffffffffu, m);
          if ((et & 31) == 0) atomicMax(max_bits + first, all);
        } else {
          atomicMax(max_bits + r, m);
        }
        continue;
      }
      if (GRID == OCS_GRID_E8M0 && m >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
      const MxScale s = mx4_scale<GRID, X>(m, GRID == OCS_GRID_E4M3 ? mx4_row_exponent(max_bits[r]) : 0);
      uint32_t c[N / 8];
      v.template codes<GRID>(s, c);
      scales[in * kMxTile + r * 16 + bb] = b < nb ? (unsigned char)s.byte : 0;   // (past the end: anything but NaN)
      unsigned char* row = tok + (in * TN + r) * KB;
      if constexpr (N == 32) *reinterpret_cast<uint4*>(row + ((bb ^ (r & 7)) << 4)) = make_uint4(c[0], c[1], c[2], c[3]);
      else *reinterpret_cast<uint2*>(row + (((bb >> 1) ^ (r & 7)) << 4) + (bb & 1) * 8) = make_uint2(c[0], c[1]);
    }
  }
  fence_proxy_async_smem();   // the tensor cores read what these threads wrote
}

template <typename T, int GRID, int TN, int CG, bool FUSED>
__global__ void __launch_bounds__(kThreads, 1)
mx_gemm_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_t,
               const __grid_constant__ CUtensorMap tm_sw, const __grid_constant__ CUtensorMap tm_st, const MxGemm p, T* __restrict__ Y) {
  using L = MxSmem<GRID, TN, CG, FUSED>;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t raw = smem_u32(smem_dyn);
  const uint32_t base = (raw + 1023u) & ~1023u;
  unsigned char* tiles = smem_dyn + (base - raw);
  unsigned char* tokens = tiles + L::kStages * L::kStageBytes;
  unsigned char* token_scales = tokens + L::kFusedBlocks * TN * KB;
  unsigned char* after = tokens + L::kTokenBytes;
  unsigned char* xbuf = L::kXInRing ? tiles : after;
  float* scale_buf = reinterpret_cast<float*>(after + L::kXExtra);
  uint32_t* row_max = reinterpret_cast<uint32_t*>(after + L::kXExtra + L::kScaleBytes);   // FUSED: [TN] maxima, then scales
  float* row_scale = reinterpret_cast<float*>(row_max + TN);
  unsigned char* tails = reinterpret_cast<unsigned char*>(row_scale + TN);
  uint64_t* bars = reinterpret_cast<uint64_t*>(after + L::kXExtra + L::kScaleBytes + L::kRowBytes);
  auto full_bar = [&](int s) { return smem_u32(bars + s); };
  auto empty_bar = [&](int s) { return smem_u32(bars + L::kStages + s); };
  auto accfull_bar = [&](int a) { return smem_u32(bars + 2 * L::kStages + a); };
  auto accempty_bar = [&](int a) { return smem_u32(bars + 2 * L::kStages + 2 + a); };
  const uint32_t xfull_bar = smem_u32(bars + 2 * L::kStages + 4);
  const uint32_t xready_bar = smem_u32(bars + 2 * L::kStages + 5);
  auto sfull_bar = [&](int s) { return smem_u32(bars + 2 * L::kStages + 6 + s); };            // a stage's scales are here
  auto sready_bar = [&](int b) { return smem_u32(bars + 3 * L::kStages + 6 + b); };           // ... and in tensor memory
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 3 * L::kStages + 8);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((3 * L::kStages + 8) * 8 + 8 <= L::kCtrlBytes, "control block");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int CL = CG * p.slices;
  const int rank = CL > 1 ? (int)cluster_rank() : 0;
  const int half = rank % CG, slice = rank / CG;
  const int cluster = blockIdx.x / CL, n_clusters = gridDim.x / CL;
  const int my_st = (p.num_st - slice + p.slices - 1) / p.slices;

  // Set-up.  Nobody waits for more than it needs (named barriers: 2 = set up, 3 = barriers stand, 4 = tokens in place).  A peer may be written to
  // once all threads of the cluster have arrived; a pair waits for that at once, the others where they first need it.
  if (warp == 0) {
    if (lane == 0) {
      prefetch_tmap(&tm_w);
      prefetch_tmap(&tm_sw);
      if (!FUSED) {
        prefetch_tmap(&tm_t);
        prefetch_tmap(&tm_st);
      }
      for (int s = 0; s < L::kStages; ++s) {
        mbar_init(full_bar(s), 1);     // the leader's producer announces the bytes of both CTAs
        mbar_init(empty_bar(s), 1);    // commit of the products that read the stage
        mbar_init(sfull_bar(s), 1);
      }
      for (int a = 0; a < 2; ++a) {
        mbar_init(accfull_bar(a), 1);
        mbar_init(accempty_bar(a), CG * kEpiWarps);
        mbar_init(sready_bar(a), CG * 4);
      }
      mbar_init(xfull_bar, 1);
      mbar_init(xready_bar, p.slices);
      *abort_flag = 0;
      fence_barrier_init();
      fence_proxy_async_smem();
      if (L::kXBytes && p.slices > 1) mbar_arrive_expect_tx(xfull_bar, (uint32_t)L::kXBytes);
    }
    __syncwarp();
    asm volatile("bar.arrive 3, 64;" ::: "memory");
    asm volatile("bar.arrive 2, %0;" ::"n"(kThreads) : "memory");
    if (CL > 1) cluster_arrive();
  } else if (warp == 1) {
    if (CG == 2) tmem_alloc_pair(smem_u32(tmem_slot), L::kTmemCols);
    else tmem_alloc(smem_u32(tmem_slot), L::kTmemCols);
    tc_fence_before();
    asm volatile("bar.arrive 2, %0;" ::"n"(kThreads) : "memory");
    if (CL > 1) cluster_arrive();
    asm volatile("bar.sync 3, 64;" ::: "memory");
  } else {
    if (CL > 1) cluster_arrive();
    if (FUSED) {
      // they need nothing of the set-up
      if (p.x_type == OCS_F32) quantize_tokens<float, GRID, TN>(p, slice, my_st * L::kSub, tokens, token_scales, row_max, row_scale, tails);
      else if (p.x_type == OCS_F16) quantize_tokens<__half, GRID, TN>(p, slice, my_st * L::kSub, tokens, token_scales, row_max, row_scale, tails);
      else quantize_tokens<__nv_bfloat16, GRID, TN>(p, slice, my_st * L::kSub, tokens, token_scales, row_max, row_scale, tails);
      if (warp < 2 + kEpiWarps) asm volatile("bar.arrive 4, %0;" ::"n"(kThreads - 32) : "memory");   // this warp's codes are in place
    }
    asm volatile("bar.sync 2, %0;" ::"n"(kThreads) : "memory");
  }
  if (CG == 2) cluster_wait();
  tc_fence_after();
  const uint32_t tmem_base = warp == 0 ? 0u : *reinterpret_cast<volatile uint32_t*>(tmem_slot);

  if (warp == 0) {
    // ---------------------------------------------------------------- copies
    if (lane == 0) {
      const uint32_t lead = CG == 2 ? (uint32_t)(rank & ~1) : 0;
      int it = 0;
      bool ok = true;
      int ahead = 0, mt, nt;
      auto bar_of = [&](int s) { return CG == 2 ? peer_addr(full_bar(s), lead) : full_bar(s); };
      auto load_w = [&](int s, int st) {
        const uint32_t at = base + s * L::kStageBytes, bar = bar_of(s);
#pragma unroll
        for (int u = 0; u < L::kSub; ++u) {
          const int kb = st * L::kSub + u, row = (nt * CG + half) * TW;
          if (CG == 2) tma_load_2d_pair(at + u * L::kWBytes, &tm_w, bar, kb * KB, row);
          else tma_load_2d(at + u * L::kWBytes, &tm_w, bar, kb * KB, row);
          tma_load_scales(at + L::kAtSW + u * L::kSWBytes, &tm_sw, sfull_bar(s), kb * L::kPieces, nt * CG + half);
        }
      };
      auto load_t = [&](int s, int st) {
        const uint32_t at = base + s * L::kStageBytes, bar = bar_of(s);
#pragma unroll
        for (int u = 0; u < L::kSub; ++u) {
          const int kb = st * L::kSub + u, row = mt * TN + half * L::kTokens;
          if (CG == 2) tma_load_2d_pair(at + L::kAtT + u * L::kTBytes, &tm_t, bar, kb * KB, row);
          else tma_load_2d(at + L::kAtT + u * L::kTBytes, &tm_t, bar, kb * KB, row);
#pragma unroll
          for (int i = 0; i < L::kTiles; ++i)   // (both CTAs of a pair need the scales of all the tile's tokens)
            tma_load_scales(at + L::kAtST + u * L::kSTBytes + i * L::kSWBytes, &tm_st, sfull_bar(s), kb * L::kPieces, mt * TN / 128 + i);
        }
      };
      auto announce = [&](int s) {
        if (half == 0) mbar_arrive_expect_tx(full_bar(s), CG * L::kFullTx);
        mbar_arrive_expect_tx(sfull_bar(s), L::kScaleTx);
      };
      // weights do not depend on the kernel before: the first ring of them is requested before waiting for it
      if (cluster < p.total) {
        tile_of(p, cluster, &mt, &nt);
        ahead = min(L::kStages, my_st);
        for (int i = 0; i < ahead; ++i) {
          announce(i);
          load_w(i, slice + i * p.slices);
        }
      }
      if (!FUSED) grid_wait_previous();
      for (int t = cluster; ok && t < p.total; t += n_clusters) {
        tile_of(p, t, &mt, &nt);
        for (int i = 0; i < my_st; ++i, ++it) {
          const int s = it % L::kStages;
          if (it >= ahead) {
            if (!mbar_wait(empty_bar(s), (uint32_t)((it / L::kStages) & 1) ^ 1u, abort_flag)) { ok = false; break; }
            announce(s);
            load_w(s, slice + i * p.slices);
          }
          if (!FUSED) load_t(s, slice + i * p.slices);
        }
      }
      // every commit has arrived (also those the other CTA of a pair sends here) before the CTA may leave
      for (int i = 0; ok && i < L::kStages; ++i, ++it)
        ok = mbar_wait(empty_bar(it % L::kStages), (uint32_t)((it / L::kStages) & 1) ^ 1u, abort_flag);
      if (*abort_flag)   // copies that are still in flight land before the CTA's shared memory is released
        for (int i = 0; i < 2000; ++i) __nanosleep(100);
    }
    __syncwarp();
    if (CL > 1 && CG == 1) cluster_wait();
  } else if (warp == 1) {
    // ---------------------------------------------------------------- tensor cores
    if (FUSED) asm volatile("bar.sync 4, %0;" ::"n"(kThreads - 32) : "memory");   // the tokens' codes are in place
    if (lane == 0 && half == 0) {
      constexpr uint32_t kDescM = TW * CG;
      const uint16_t mask = (uint16_t)(3u << (rank & ~1));
      const uint64_t w_desc0 = smem_desc_sw128(base), t_desc0 = smem_desc_sw128(FUSED ? smem_u32(tokens) : base + L::kAtT);
      int j = 0, s = 0;
      uint32_t phase = 0, n = 0;   // n: stages so far
      bool ok = true;
      for (int t = cluster; ok && t < p.total; t += n_clusters, ++j) {
        int mt, nt;
        tile_of(p, t, &mt, &nt);
        const int acc = j & 1;
        const uint32_t half_col = TN == 64 ? (mt & 1) * 2 : 0;   // the columns of this half of the 128 tokens
        if (L::kOverlap) {
          if (j && !mbar_wait_relaxed(accempty_bar(0), (uint32_t)(j - 1) & 1u, abort_flag)) break;
        } else {
          if (!mbar_wait_relaxed(accempty_bar(acc), (((uint32_t)j >> 1) & 1u) ^ 1u, abort_flag)) break;
        }
        tc_fence_after();
        const uint32_t d = tmem_base + (uint32_t)(acc * L::kAccStride);
        uint32_t more = 0;
        for (int i = 0; i < my_st; ++i) {
          if (!mbar_wait(full_bar(s), phase, abort_flag) || !mbar_wait_relaxed(sready_bar(n & 1), (n >> 1) & 1u, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint32_t o = (uint32_t)(s * (L::kStageBytes >> 4));
          const uint64_t t_desc = t_desc0 + (FUSED ? (uint32_t)(i * L::kSub * (TN * KB >> 4)) : o);
#pragma unroll
          for (int u = 0; u < L::kSub; ++u) {
            const uint32_t sw_col = tmem_base + L::kScaleCol + (n & 1) * L::kStageCols + u * L::kScaleCols;
            const uint32_t st_col = sw_col + 4 * L::kPieces + half_col;
#pragma unroll
            for (int k = 0; k < 4; ++k) {   // 64 contraction indices: 32 bytes on, 2 in the descriptors' units of 16
              constexpr int kPer = 4 / L::kPieces;   // products per piece of scales
              const int c = k / kPer, sf = k % kPer * 2;
              umma_mx4<GRID, CG>(d, w_desc0 + o + u * (L::kWBytes >> 4) + 2 * k, t_desc + u * ((FUSED ? TN * KB : L::kTBytes) >> 4) + 2 * k,
                                 mx_instr_desc(GRID, kDescM, TN, sf), sw_col + 4 * c, st_col + 4 * c * L::kTiles, u + k == 0 ? more : 1u);
            }
          }
          more = 1;
          ++n;
          if (CG == 2) umma_commit_pair(empty_bar(s), mask);
          else umma_commit(empty_bar(s));
          if (++s == L::kStages) { s = 0; phase ^= 1; }
        }
        if (!ok) break;
        if (CG == 2) umma_commit_pair(accfull_bar(acc), mask);
        else umma_commit(accfull_bar(acc));
      }
    }
    __syncwarp();
    if (CL > 1 && CG == 1) cluster_wait();
  } else if (warp >= 2 + kEpiWarps) {
    // ---------------------------------------------------------------- scales (of the CTA's own shared memory and lanes)
    const uint32_t q = warp & 3, lead = (uint32_t)(rank & ~(CG - 1));
    const uint32_t lanes = tmem_base + ((q * 32) << 16) + L::kScaleCol;
    if (FUSED) asm volatile("bar.sync 4, %0;" ::"n"(kThreads - 32) : "memory");   // the tokens' scales are in place
    int s = 0, s_before = 0;               // s_before: the stage before the last one
    uint32_t phase = 0, phase_before = 0, n = 0;
    bool ok = true;
    for (int t = cluster; ok && t < p.total; t += n_clusters) {
      for (int i = 0; i < my_st; ++i, ++n) {
        if (!warp_wait(sfull_bar(s), phase, abort_flag)) { ok = false; break; }
        const unsigned char* st = tiles + s * L::kStageBytes + lane * 16;
        constexpr int kAll = L::kPieces * (1 + L::kTiles);
        uint32_t v[L::kSub][4 * kAll];
#pragma unroll
        for (int u = 0; u < L::kSub; ++u) {
          if (FUSED) {   // a lane's token: four scales for the first column of each piece
            const uint4 w = *reinterpret_cast<const uint4*>(token_scales + (i * L::kSub + u) * kMxTile + lane * 16);
            const uint32_t c[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int e = 0; e < 4 * L::kPieces; ++e) v[u][4 * L::kPieces + e] = c[e / 4];
          }
#pragma unroll
          for (int e = 0; e < (FUSED ? L::kPieces : kAll); ++e) {   // the weights' pieces, then for each group of blocks the tokens' tiles
            const int c = (e - L::kPieces) / L::kTiles, k = (e - L::kPieces) % L::kTiles;
            const uint4 w = *reinterpret_cast<const uint4*>(
                st + (e < L::kPieces ? L::kAtSW + u * L::kSWBytes + e * kMxTile : L::kAtST + u * L::kSTBytes + k * L::kSWBytes + c * kMxTile));
            v[u][4 * e] = w.x; v[u][4 * e + 1] = w.y; v[u][4 * e + 2] = w.z; v[u][4 * e + 3] = w.w;
          }
        }
        if (n >= 2) {                      // the products that read this buffer are done
          if (!warp_wait(empty_bar(s_before), phase_before, abort_flag)) { ok = false; break; }
          tc_fence_after();
          if (++s_before == L::kStages) { s_before = 0; phase_before ^= 1u; }
        }
        __syncwarp();
#pragma unroll
        for (int u = 0; u < L::kSub; ++u)
#pragma unroll
          for (int e = 0; e < 4 * kAll; e += 4 * L::kPieces)
            tmem_store<4 * L::kPieces>(lanes + (n & 1) * L::kStageCols + u * L::kScaleCols + e, v[u] + e);
        asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (CG == 2) mbar_arrive_peer_relaxed(peer_addr(sready_bar(n & 1), lead));
          else mbar_arrive(sready_bar(n & 1));
        }
        if (++s == L::kStages) { s = 0; phase ^= 1u; }
      }
    }
    __syncwarp();
    if (CL > 1 && CG == 1) cluster_wait();
  } else {
    // ---------------------------------------------------------------- epilogue
    constexpr int EC = 16;                              // accumulator columns (tokens) moved at a time
    const int ew = warp - 2, q = warp & 3, part = ew >> 2;   // lanes 32q.. of tensor memory; two warps share a quadrant
    float* sc = scale_buf + ew * L::kWarpTokens;
    const bool pairs = sizeof(T) == 2 && (p.ldy % 2 == 0) && (p.N % 2 == 0) && (reinterpret_cast<uintptr_t>(Y) & 3) == 0;
    if (!FUSED) grid_wait_previous();
    if (CL > 1 && CG == 1) cluster_wait();
    auto token_scale = [&](int m) {
      if (m >= p.M) return 0.0f;
      if (FUSED) return row_scale[m];
      return p.a_scales ? __ldcg(p.a_scales + m) : 1.0f;
    };
    // the scales of this warp's `count` tokens; whether any is beyond kNearScale
    auto fetch_scales = [&](int count, auto token) {
      bool far = false;
      for (int i = lane; i < count; i += 32) {
        const float f = token_scale(token(i));
        sc[i] = f;
        far |= f > kNearScale;
      }
      far = GRID == OCS_GRID_E4M3 && __any_sync(0xffffffffu, far);
      __syncwarp();
      return far;
    };
    int j = 0;
    for (int t = cluster; t < p.total; t += n_clusters, ++j) {
      int mt, nt;
      tile_of(p, t, &mt, &nt);
      const int acc = j & 1;
      const int n = (nt * CG + half) * TW + q * 32 + lane;
      const float ws = n < p.N && p.w_scales ? __ldg(p.w_scales + n) : 1.0f;
      const float b = p.bias && n < p.N ? __ldg(p.bias + n) : 0.0f;
      if (p.slices > 1) {
        // K split: owner o of the tile's slices finishes tokens [o * own, (o + 1) * own).  Every CTA sends the columns
        // another one owns into that one's buffer, cells of 16 bytes [sender][four tokens][channel], counted as
        // transaction bytes on the owner's barrier; they are added in the order of the senders.
        if constexpr (L::kXBytes > 0) {
          const int own = TN / p.slices, groups = own / 4;
          __syncwarp();
          const bool far = fetch_scales(own, [&](int i) { return mt * TN + slice * own + i; });
          const float ws_left = far ? scale_left(ws) : ws;
          if (!warp_wait(accfull_bar(acc), ((uint32_t)j >> 1) & 1u, abort_flag)) break;
          tc_fence_after();
          if (L::kXInRing) {
            // this CTA's tensor cores are done with its ring: it may be written to; and so are all the others'
            if (ew == 0 && lane == 0)
              for (int o = 0; o < p.slices; ++o) mbar_arrive_peer(peer_addr(xready_bar, (uint32_t)o));
            if (!warp_wait_cluster(xready_bar, 0u, abort_flag)) break;
          }
          const uint32_t mine = smem_u32(xbuf) + (uint32_t)(slice * groups * TW + q * 32 + lane) * 16u;
          const uint32_t addr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * L::kAccStride);
          uint32_t v[2][16];
          constexpr int kPieces = TN >= 32 ? TN / 32 : 1;
          if (part * 16 < TN) {
            __syncwarp();
            tmem_ld_async<16>(addr + part * 16, v[0]);
#pragma unroll
            for (int i = 0; i < kPieces; ++i) {
              tmem_wait_ld16(v[i & 1]);
              if (i + 1 < kPieces) tmem_ld_async<16>(addr + part * 16 + 32 * (i + 1), v[(i + 1) & 1]);
              const uint32_t* w = v[i & 1];
#pragma unroll
              for (int e = 0; e < 16; e += 4) {
                const int col = part * 16 + 32 * i + e;
                const int owner = col / own, g = (col - owner * own) / 4;
                const uint32_t peer = (uint32_t)owner;
                st_async_v4(peer_addr(mine + (uint32_t)g * (TW * 16u), peer), make_uint4(w[e], w[e + 1], w[e + 2], w[e + 3]),
                            peer_addr(xfull_bar, peer));
              }
            }
          }
          if (!warp_wait_cluster(xfull_bar, 0u, abort_flag)) break;
          const int m_own = mt * TN + slice * own;
          T* y = Y + (long long)m_own * p.ldy + n;
          const uint32_t slot = (uint32_t)groups * TW * 16u;   // from one sender's cells to the next one's
          for (int g = part; g < groups; g += 2) {
            const unsigned char* cell = xbuf + (size_t)(g * TW + q * 32 + lane) * 16;
            float4 a = *reinterpret_cast<const float4*>(cell);
#pragma unroll 4
            for (int sl = 1; sl < p.slices; ++sl) {
              const float4 b4 = *reinterpret_cast<const float4*>(cell + sl * slot);
              a.x = __fadd_rn(a.x, b4.x); a.y = __fadd_rn(a.y, b4.y); a.z = __fadd_rn(a.z, b4.z); a.w = __fadd_rn(a.w, b4.w);
            }
            uint32_t av[4] = {__float_as_uint(a.x), __float_as_uint(a.y), __float_as_uint(a.z), __float_as_uint(a.w)};
            if (far) near_sums<4>(av, ws);
            const float4 s4 = *reinterpret_cast<const float4*>(sc + 4 * g);
            const float sv[4] = {s4.x, s4.y, s4.z, s4.w};
            finish<false, T, 4>(y + 4 * g * p.ldy, p.ldy, av, sv, ws_left, b, p.M - m_own - 4 * g, n < p.N, pairs);
          }
        }
        break;   // a K split is used only where every cluster has one tile
      }
      // the token scales of this warp's columns: fetched while the main loop runs
      __syncwarp();
      const bool far = fetch_scales(L::kWarpTokens, [&](int i) { return mt * TN + (i / EC) * 2 * EC + part * EC + i % EC; });
      const float ws_left = far ? scale_left(ws) : ws;
      if (!warp_wait(accfull_bar(acc), ((uint32_t)j >> 1) & 1u, abort_flag)) break;
      tc_fence_after();
      // Pieces of EC columns; the next one's way out of tensor memory overlaps this one's arithmetic and stores.  Overlapping
      // accumulators: from the end that the next tile's products write to (the first one's last columns, the second one's
      // first); once those are out, the next tile may start.
      constexpr int kPieces = TN >= 2 * EC ? TN / (2 * EC) : 1;
      const bool down = L::kOverlap && acc == 0;
      const uint32_t addr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * L::kAccStride + part * EC);
      const bool n_all = (nt * CG + half) * TW + q * 32 + 32 <= p.N;
      const int m_first = mt * TN + part * EC;
      auto emptied = [&](int a) {
        tc_fence_before();
        __syncwarp();
        if (lane == 0) {
          if (CG == 2) mbar_arrive_peer_relaxed(peer_addr(accempty_bar(a), (uint32_t)(rank & ~1)));
          else mbar_arrive(accempty_bar(a));
        }
      };
      uint32_t v[2][EC];
      if (part * EC < TN) {
        if (far)   // in tensor memory, so that the loop below stays as short as it is
#pragma unroll 1
          for (int i = 0; i < kPieces; ++i) {
            tmem_ld_async<EC>(addr + 2 * EC * i, v[0]);
            tmem_wait_ld16(v[0]);
            near_sums<EC>(v[0], ws);
            tmem_store<EC>(addr + 2 * EC * i, v[0]);
            asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
          }
        auto piece = [&](int i) { return down ? kPieces - 1 - i : i; };
        tmem_ld_async<EC>(addr + 2 * EC * piece(0), v[0]);
#pragma unroll 2
        for (int i = 0; i < kPieces; ++i) {   // (no more than the two buffers ask for: what runs should stay in the instruction cache)
          tmem_wait_ld16(v[i & 1]);
          if (L::kOverlap && i == (L::kShared + 2 * EC - 1) / (2 * EC) - 1) emptied(0);
          if (i + 1 < kPieces) tmem_ld_async<EC>(addr + 2 * EC * piece(i + 1), v[(i + 1) & 1]);
          const int at = 2 * EC * piece(i), left = p.M - m_first - at;   // tokens from this piece's first on
          if (left <= 0) continue;               // the same for the whole warp
          float s[EC];
#pragma unroll
          for (int e = 0; e < EC; e += 4) {
            const float4 f = *reinterpret_cast<const float4*>(sc + at / 2 + e);
            s[e] = f.x; s[e + 1] = f.y; s[e + 2] = f.z; s[e + 3] = f.w;
          }
          T* y = Y + (long long)(m_first + at) * p.ldy + n;
          if (n_all && left >= EC) finish<true, T, EC>(y, p.ldy, v[i & 1], s, ws_left, b, left, true, pairs);
          else finish<false, T, EC>(y, p.ldy, v[i & 1], s, ws_left, b, left, n < p.N, pairs);
        }
      }
      if (!L::kOverlap) emptied(acc);
    }
    tc_fence_before();
  }

  __syncthreads();
  if (CL > 1) cluster_sync_all();   // no CTA leaves while a peer may still store into it or arrive on its barriers
  if (warp == 1) {
    __syncwarp();
    tc_fence_after();
    if (CG == 2) tmem_dealloc_pair(tmem_base, L::kTmemCols);
    else tmem_dealloc(tmem_base, L::kTmemCols);
  }
  if (threadIdx.x == 0 && *abort_flag) flag(p.dev_status, OCS_DEV_TIMEOUT);
}

// ------------------------------------------------------------------------------------------------ host
struct MxPlan {
  int tn, cg, slices;
};

// Test hook (ocs_selftest_force_mx4_plan), in one word: tn << 8 | cg << 4 | slices, 0 for none.
std::atomic<int> g_forced_plan{0};

// CTAs resident at once, one per SM, for cluster sizes 1, 2, 4, 8 (a cluster lies inside one GPC)
int cluster_capacity(int cl) { return cl <= 2 ? 148 : (cl == 4 ? 132 : 120); }

int stages_of(int tn, int num_kb) { return (num_kb + stage_blocks(tn) - 1) / stage_blocks(tn); }

// Scales come in groups of 128 tokens, of which a product takes an aligned half or the first part: tiles of fewer than 64
// tokens are for calls with no more tokens than that.
bool tile_fits(int tn, int M) { return tn >= 64 || M <= tn; }

bool split_fits(int tn, int cg, int slices, long long tiles, int stages) {
  if (slices == 1) return true;
  return cg == 1 && tn < 256 && tn / slices >= 4 && slices <= stages && tiles * slices <= cluster_capacity(slices);
}

// The plan by a time model in microseconds, fitted to 1545 measurements (M 1..8192, K 64..25088, N 64..33278, both grids, fp32
// and 16-bit outputs, every plan that fits): root mean square error 7.4 %; the plan it picks is 0.7 % slower than the best
// measured one on average, 11 % at worst.  A tile costs its K-blocks and its epilogue; a K split adds the exchange; the bytes
// take their time at 4.9 TB/s; of the two the longer one counts most (root of the sum of squares); 3.7 us pass before the first
// and after the last tile.
MxPlan choose_plan(int M, int N, int K, ocs_grid grid, int out_bytes) {
  struct Form { int tn, cg; double block_us, epilogue_us; };
  static const Form forms[5] = {{16, 1, 0.256, 0.60}, {32, 1, 0.257, 0.57}, {64, 1, 0.273, 0.63}, {128, 1, 0.331, 1.31}, {256, 2, 0.352, 2.56}};
  const int num_kb = (K + 2 * KB - 1) / (2 * KB);
  auto tiles_of = [&](int tn, int cg) {
    return (long long)((M + (long long)tn - 1) / tn) * ((N + (long long)TW * cg - 1) / (TW * cg));
  };
  if (const int forced = g_forced_plan.load()) {
    MxPlan r{forced >> 8, forced >> 4 & 15, forced & 15};
    while (!tile_fits(r.tn, M)) r.tn *= 2;
    while (r.slices > 1 && !split_fits(r.tn, r.cg, r.slices, tiles_of(r.tn, r.cg), stages_of(r.tn, num_kb))) r.slices /= 2;
    return r;
  }
  const double row = K * (grid == OCS_GRID_E4M3 ? 0.5625 : 0.53125);   // bytes of a row's codes and scales
  const double bytes_us = (((double)N + M) * row + (double)M * N * out_bytes) / 4.94e6;
  MxPlan best{64, 1, 1};
  double best_us = 1e300;   // squared
  for (const Form& f : forms) {
    if (!tile_fits(f.tn, M)) continue;
    const long long tiles = tiles_of(f.tn, f.cg);
    for (int s = 1; s <= 8; s *= 2) {
      if (!split_fits(f.tn, f.cg, s, tiles, stages_of(f.tn, num_kb))) continue;
      const long long slots = cluster_capacity(f.cg * s) / (f.cg * s);
      const double waves = (double)((tiles + slots - 1) / slots);
      const int blocks = (stages_of(f.tn, num_kb) + s - 1) / s * stage_blocks(f.tn);
      double us = waves * (blocks * f.block_us * (grid == OCS_GRID_E4M3 ? 1.034 : 1.0) + f.epilogue_us * (out_bytes == 4 ? 0.87 : 1.0));
      if (s > 1) us += 3.61 * f.tn / 128.0 + 0.35;
      us = us * us + bytes_us * bytes_us;   // (its root, plus a constant)
      if (us < best_us) { best_us = us; best = MxPlan{f.tn, f.cg, s}; }
    }
  }
  return best;
}

struct Product {
  const uint8_t* A;
  const uint8_t* A_scales;
  const float* a_rows;
  const uint8_t* W;
  const uint8_t* W_scales;
  const float* w_rows;
  const float* bias;
  int M, N, K;
  long long lda, ldw, ldy;
  ocs_grid grid;
  void* Y;
  ocs_dtype y_type;
  int* dev_status;
  // not quantized yet (A = NULL)
  const void* X = nullptr;
  long long ldx = 0;
  const int32_t* idx_map = nullptr;
  ocs_dtype x_type = OCS_F32;
  int C = 0;
};

// Whether ocs_linear_mx4 quantizes inside the product's kernel: every CTA quantizes all tokens itself, those of its share of
// the contraction.  That saves a launch and the workspace, 4 to 6 us of the host's 17, which is what bounds an eager call of
// this size.  The host decides here: on the device the fused form is even up to some 500 blocks and slower beyond, since its code
// is cold and few warps run it.  us by graph replay, fused against two launches: E4M3 (M, C, N) = (1, 8192, 8192), 512 blocks:
// 14.8 against 13.5 to 15.5; (20, 650, 2600) in fp32, 820 blocks: 12.5 against 6.5; (8, 4096, 4096), 2048 blocks: 11.4 against 7.6;
// E8M0 (16, 1024, 4096), 512 blocks: 7.3 against 6.4; (2, 300, 500): 6.3 against 7.8; (24, 2000, 2000), 1512 blocks: 8.4
// against 7.3.  A caller that replays graphs takes ocs_quantize_mx4 and ocs_qlinear_mx4 instead, which give the same bits.
// Blocks are those of all K channels, duplicated ones too: each is quantized.
bool fuse_tokens(const MxPlan& plan, int M, int K, ocs_grid grid) {
  if (plan.tn > 32) return false;
  const int num_kb = (K + 2 * KB - 1) / (2 * KB), n = mx4_block(grid);
  const int my_kb = (stages_of(plan.tn, num_kb) + plan.slices - 1) / plan.slices * stage_blocks(plan.tn);
  return my_kb <= kFusedBytes / (plan.tn * KB + kMxTile) && (long long)M * ((K + n - 1) / n) <= (grid == OCS_GRID_E4M3 ? 1024 : 2048);
}

template <typename T, int GRID, int TN, int CG, bool FUSED = false>
ocs_status launch_tiles(const Product& g, int slices, bool overlap, cudaStream_t stream) {
  using L = MxSmem<GRID, TN, CG, FUSED>;
  static std::atomic<unsigned long long> ready{0};   // devices whose copy of the kernel has its attribute set
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return OCS_ERR_CUDA;
  if (dev >= 64 || !(ready.load() >> dev & 1)) {
    if (cudaFuncSetAttribute(mx_gemm_kernel<T, GRID, TN, CG, FUSED>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynBytes) != cudaSuccess)
      return OCS_ERR_CUDA;
    if (dev < 64) ready.fetch_or(1ull << dev);
  }
  MxGemm p{};
  p.M = g.M; p.N = g.N; p.num_st = stages_of(TN, (g.K + 2 * KB - 1) / (2 * KB));
  p.a_scales = g.a_rows; p.w_scales = g.w_rows; p.bias = g.bias; p.ldy = g.ldy;
  p.dev_status = g.dev_status;
  p.n_tiles = (g.N + TW * CG - 1) / (TW * CG);
  p.m_tiles = (g.M + TN - 1) / TN;
  const long long total = (long long)p.n_tiles * p.m_tiles;
  if (total > 0x3fffffff) return OCS_ERR_UNSUPPORTED;
  p.total = (int)total;
  p.slices = slices;
  CUtensorMap tm_w, tm_t, tm_sw, tm_st;
  const cuuint64_t row = (cuuint64_t)(g.K + 1) / 2;
  const cuuint64_t wd[2] = {row, (cuuint64_t)g.N}, ws[1] = {(cuuint64_t)g.ldw};
  const cuuint64_t td[2] = {row, (cuuint64_t)g.M}, ts[1] = {(cuuint64_t)g.lda};
  const cuuint32_t wb[2] = {KB, TW}, tb[2] = {KB, (cuuint32_t)L::kTokens};
  if (!encode_u8(&tm_w, g.W, 2, wd, ws, wb)) return OCS_ERR_CUDA;
  const int n = mx4_block(GRID), pieces = ((g.K + n - 1) / n + 3) / 4;
  if (!encode_mx4_scales(&tm_sw, g.W_scales, pieces, (g.N + 127) / 128, L::kPieces)) return OCS_ERR_CUDA;
  if (FUSED) {
    tm_t = tm_st = tm_w;   // unused
    p.X = g.X; p.ldx = g.ldx; p.idx_map = g.idx_map; p.x_type = g.x_type; p.C = g.C; p.K = g.K;
  } else if (!encode_u8(&tm_t, g.A, 2, td, ts, tb) || !encode_mx4_scales(&tm_st, g.A_scales, pieces, (g.M + 127) / 128, L::kPieces)) {
    return OCS_ERR_CUDA;
  }
  const int cl = CG * slices;
  const long long slots = cluster_capacity(cl) / cl;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((total < slots ? total : slots) * cl), 1, 1);
  cfg.blockDim = dim3(kThreads, 1, 1);
  cfg.dynamicSmemBytes = L::kDynBytes;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  int n_attr = 0;
  if (cl > 1) {
    attr[n_attr].id = cudaLaunchAttributeClusterDimension;
    attr[n_attr].val.clusterDim.x = cl; attr[n_attr].val.clusterDim.y = 1; attr[n_attr].val.clusterDim.z = 1;
    ++n_attr;
  }
  if (overlap) {
    attr[n_attr].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n_attr].val.programmaticStreamSerializationAllowed = 1;
    ++n_attr;
  }
  cfg.attrs = attr; cfg.numAttrs = n_attr;
  LaunchScope scope(FUSED ? "mx_gemm_kernel(fused)" : "mx_gemm_kernel", stream);
  if (cudaLaunchKernelEx(&cfg, mx_gemm_kernel<T, GRID, TN, CG, FUSED>, tm_w, tm_t, tm_sw, tm_st, p, static_cast<T*>(g.Y)) != cudaSuccess) return OCS_ERR_CUDA;
  return launch_status();
}

template <typename T, int GRID>
ocs_status run_product(const Product& g, const MxPlan& plan, bool overlap, cudaStream_t stream) {
  if (!g.A) {
    if (plan.tn == 16) return launch_tiles<T, GRID, 16, 1, true>(g, plan.slices, false, stream);
    return launch_tiles<T, GRID, 32, 1, true>(g, plan.slices, false, stream);
  }
  switch (plan.tn) {
    case 16: return launch_tiles<T, GRID, 16, 1>(g, plan.slices, overlap, stream);
    case 32: return launch_tiles<T, GRID, 32, 1>(g, plan.slices, overlap, stream);
    case 64: return launch_tiles<T, GRID, 64, 1>(g, plan.slices, overlap, stream);
    case 128: return launch_tiles<T, GRID, 128, 1>(g, plan.slices, overlap, stream);
    default: return launch_tiles<T, GRID, 256, 2>(g, plan.slices, overlap, stream);
  }
}
template <typename T>
ocs_status run_product(const Product& g, const MxPlan& plan, bool overlap, cudaStream_t stream) {
  return g.grid == OCS_GRID_E8M0 ? run_product<T, OCS_GRID_E8M0>(g, plan, overlap, stream)
                                 : run_product<T, OCS_GRID_E4M3>(g, plan, overlap, stream);
}
ocs_status run_product(const Product& g, const MxPlan& plan, bool overlap, cudaStream_t stream) {
  switch (g.y_type) {
    case OCS_F16: return run_product<__half>(g, plan, overlap, stream);
    case OCS_BF16: return run_product<__nv_bfloat16>(g, plan, overlap, stream);
    default: return run_product<float>(g, plan, overlap, stream);
  }
}

// Everything but the tokens, which ocs_linear_mx4 has in another form.
ocs_status check_product(const Product& g) {
  if (!g.W || !g.W_scales || !g.Y || (g.grid == OCS_GRID_E4M3 && !g.w_rows)) return OCS_ERR_INVALID_ARG;
  if (g.M >= (1 << 30) || g.K >= kMxMaxK || g.N > 0x7fffffff - 512) return OCS_ERR_UNSUPPORTED;
  if (g.ldw < (g.K + 1) / 2 || g.ldw % 16 != 0 || !aligned(g.W, 16) || !aligned(g.W_scales, 16)) return OCS_ERR_SHAPE;
  if (g.ldy < g.N || !aligned(g.Y, elem_bytes(g.y_type)) || !aligned(g.w_rows, 4) || !aligned(g.bias, 4)) return OCS_ERR_SHAPE;
  return OCS_OK;
}

}  // namespace
}  // namespace ocs

using namespace ocs;

extern "C" ocs_status ocs_qlinear_mx4(const uint8_t* A_codes, const uint8_t* A_scales, const float* a_row_scales, int M, int K,
                                      int64_t lda, const uint8_t* W_codes, const uint8_t* W_scales, const float* w_row_scales,
                                      int N, int64_t ldw, ocs_grid grid, const float* bias, void* Y, ocs_dtype y_type,
                                      int64_t ldy, int* dev_status, void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!valid_dtype(y_type) || !mx4_grid(grid)) return OCS_ERR_INVALID_ARG;
  if (M < 0 || K <= 0 || N <= 0) return OCS_ERR_SHAPE;
  if (M == 0) return OCS_OK;
  if (!A_codes || !A_scales || (grid == OCS_GRID_E4M3 && !a_row_scales)) return OCS_ERR_INVALID_ARG;
  const bool rows = grid == OCS_GRID_E4M3;
  const Product g{A_codes, A_scales, rows ? a_row_scales : nullptr, W_codes, W_scales, rows ? w_row_scales : nullptr, bias,
                  M, N, K, lda, ldw, ldy, grid, Y, y_type, dev_status};
  ocs_status st = check_product(g);
  if (st != OCS_OK) return st;
  if (lda < (K + 1) / 2 || lda % 16 != 0 || !aligned(A_codes, 16) || !aligned(A_scales, 16) || !aligned(g.a_rows, 4)) return OCS_ERR_SHAPE;
  if ((st = check_device()) != OCS_OK) return st;
  return run_product(g, choose_plan(M, N, K, grid, elem_bytes(y_type)), false, stream);
}

namespace {
// Where ocs_linear_mx4 keeps the tokens' codes, scales and row scales in its workspace.
struct TokenSpace {
  int64_t lda;
  size_t scales, rows, bytes;
};
TokenSpace token_space(int M, int K, ocs_grid grid) {
  TokenSpace t;
  t.lda = (int64_t)align_up((size_t)(K + 1) / 2, 16);
  t.scales = align_up((size_t)M * t.lda, 256);
  t.rows = t.scales + align_up((size_t)ocs_mx4_scale_bytes(M, K, grid), 256);
  t.bytes = t.rows + (grid == OCS_GRID_E4M3 ? align_up((size_t)M * 4, 256) : 0);
  return t;
}
// The plan of an ocs_linear_mx4 call, chosen once, and whether its tokens are quantized inside the product's kernel.
struct LinearCall {
  MxPlan plan;
  bool fused;
};
LinearCall linear_plan(int M, int K, int N, ocs_grid grid, ocs_dtype y_type) {
  const MxPlan plan = choose_plan(M, N, K, grid, elem_bytes(y_type));
  return {plan, fuse_tokens(plan, M, K, grid)};
}
}  // namespace

extern "C" size_t ocs_linear_mx4_workspace_bytes(int M, int C, int S, ocs_grid grid, int N, ocs_dtype y_type) {
  if (M <= 0 || C <= 0 || S < 0 || N <= 0 || !mx4_grid(grid) || !valid_dtype(y_type) || (int64_t)C + S >= kMxMaxK) return 0;
  if (linear_plan(M, C + S, N, grid, y_type).fused) return 0;
  return token_space(M, C + S, grid).bytes;
}

extern "C" ocs_status ocs_linear_mx4(const void* X, ocs_dtype x_type, int M, int C, int64_t ldx, int S, const int32_t* idx_map,
                                     ocs_grid grid, const uint8_t* W_codes, const uint8_t* W_scales, const float* w_row_scales,
                                     int N, int64_t ldw, const float* bias, void* Y, ocs_dtype y_type, int64_t ldy, void* ws,
                                     size_t ws_bytes, int* dev_status, void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!valid_dtype(x_type) || !valid_dtype(y_type) || !mx4_grid(grid) || S < 0) return OCS_ERR_INVALID_ARG;
  if (M < 0 || C <= 0 || N <= 0) return OCS_ERR_SHAPE;
  if (M == 0) return OCS_OK;
  if (!X || (S > 0 && !idx_map)) return OCS_ERR_INVALID_ARG;
  if ((int64_t)C + S >= kMxMaxK) return OCS_ERR_UNSUPPORTED;
  const int K = C + S;
  const LinearCall call = linear_plan(M, K, N, grid, y_type);
  const TokenSpace t = token_space(M, K, grid);
  if (!call.fused && (!ws || !aligned(ws, 256) || ws_bytes < t.bytes)) return OCS_ERR_WORKSPACE;
  const bool rows = grid == OCS_GRID_E4M3;
  Product g{nullptr, nullptr, nullptr, W_codes, W_scales, rows ? w_row_scales : nullptr, bias,
            M, N, K, t.lda, ldw, ldy, grid, Y, y_type, dev_status, X, ldx, idx_map, x_type, C};
  ocs_status st = check_product(g);
  if (st != OCS_OK) return st;
  if (ldx < C || !aligned(X, elem_bytes(x_type)) || (S > 0 && !aligned(idx_map, 4))) return OCS_ERR_SHAPE;
  if ((st = check_device()) != OCS_OK) return st;
  if (!call.fused) {
    uint8_t* codes = static_cast<uint8_t*>(ws);
    float* a_rows = rows ? reinterpret_cast<float*>(codes + t.rows) : nullptr;
    if ((st = ocs_quantize_mx4(X, x_type, M, C, ldx, S, idx_map, grid, codes, t.lda, codes + t.scales, a_rows, dev_status, stream_)) != OCS_OK)
      return st;
    g.A = codes; g.A_scales = codes + t.scales; g.a_rows = a_rows;
  }
  return run_product(g, call.plan, true, stream);
}

// Test hook: the next ocs_qlinear_mx4 / ocs_linear_mx4 calls of this process use the given plan; tn = 0 gives the choice back.
extern "C" ocs_status ocs_selftest_force_mx4_plan(int tn, int cg, int slices) {
  if (tn != 0 && ((tn != 16 && tn != 32 && tn != 64 && tn != 128 && tn != 256) || cg != (tn == 256 ? 2 : 1) ||
                  (slices != 1 && slices != 2 && slices != 4 && slices != 8)))
    return OCS_ERR_INVALID_ARG;
  g_forced_plan.store(tn ? tn << 8 | cg << 4 | slices : 0);
  return OCS_OK;
}
