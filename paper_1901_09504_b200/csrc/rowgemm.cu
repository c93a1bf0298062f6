// ocs_qlinear_rows / ocs_linear_rows: the int8 layer with a scale per token and per output channel,
//     Y[m][n] = (float(sum_k A[m][k] * W[n][k]) * a[m]) * w[n] + bias[n].
// The contraction is exact in int32 whatever its order, so tiles and splits are free; only the epilogue rounds.
//
// Layout: the weights are the rows of the tensor-core tile (128 channels = the lanes of tensor memory) and the tokens its
// columns.  The instruction's row count is fixed and its column count is free in steps of 16, and a layer always has many
// channels but often few tokens: one decoded token costs a 16-column tile, not 128 rows of padding.  An epilogue lane then
// holds one channel of many tokens, so w[n] and bias[n] are registers and a[m] a broadcast from shared memory.
// Forms: 16, 32, 64, 128 or 256 tokens per CTA, or 256 by a pair of CTAs (256 channels, each CTA stages half the tokens);
// 128-byte swizzled K-blocks come by TMA into a ring that a copy warp keeps full, one thread issues the MMAs, eight warps
// empty one of two accumulators while the other fills.  Few tiles: 2, 4 or 8 CTAs of a cluster split the contraction, send
// each other their partial sums as 16-byte cells through distributed shared memory, and finish a share of the tokens each.
//
// What bounds it (device times; the floor is the larger of the bytes at 6.54 TB/s, the measured copy rate, and the operations
// at 3.35 int8 POPS, twice the measured bf16 rate):
// M x K x N
//   8192 x 8192 x 8192, bf16 out   331 us (floor 328): the tensor pipe (93 % busy at 4096 x 8192 x 8192)
//   2047 x 4178 x 4096, bf16 out   28.7 us (floor 20.9): the tensor pipe, in two waves of which the second is not full
//   128 x 25339 x 4096, fp32 out   27.5 us (floor 16.7): one wave of 128 CTAs with one tile each, whose start (4 us), exchange
//                                  (4) and epilogue (1; the plan model's terms) have no other tile's loads beside them
//   700 x 663 x 33278, fp32 out    36.3 us (floor 17.7): 225 MB of operand tiles from L2 (a token tile again for every channel
//                                  tile) and the stores of the output (93 MB, straight from registers) share the SMs' way to
//                                  L2; 23.3 us without the stores
//   1 x 8192 x 8192, quantized here, bf16   16.5 us (floor 10.3): HBM, and 6 us of start, quantization, exchange and end
//   1 x 16384 x 16384, bf16        46 us: HBM at 5.8 TB/s (quantized by a launch of its own: its codes do not fit beside the ring)
#include <atomic>

#include "elem.cuh"
#include "ptx.cuh"

namespace ocs {
namespace {

// K-blocks of one ring stage.  A stage costs the tensor-core thread about 0.2 us of waiting, issuing and committing
// whatever it holds, which bounds the narrow forms: with two K-blocks a stage the 64-token form takes 89 instead of 110 us
// at (M, K, N) = (1024, 8192, 8192), the 16-token form 46.0 instead of 48.0 at (1, 16384, 16384); the wide forms are even
// (128 tokens) or slower (256: 344 instead of 331 at 8192 cubed) with half as many stages.
__host__ __device__ constexpr int stage_blocks(int tn) { return tn <= 64 ? 2 : 1; }

constexpr int TW = 128;        // channels (weight rows) of one CTA's tile: the lanes of tensor memory
constexpr int KB = 128;        // contraction bytes of a K-block: one 128-byte swizzle span
constexpr int UK = 32;         // contraction indices of one tcgen05.mma.kind::i8
constexpr int kThreads = 320;  // copy warp, tensor-core warp, 8 epilogue warps
constexpr int kEpiWarps = 8;
constexpr int kFusedCodes = 64 * 1024;         // token codes a CTA can hold beside the ring of weights

struct RowGemm {
  int M, N, num_kb, t_signed;     // num_kb: stages' worth of contraction (K-blocks, or pairs of them)
  int n_tiles, m_tiles, total;   // channel tiles (TW * CG), token tiles (TN)
  int slices;                    // CTAs (pairs) that share a tile and split its K-blocks
  const float* a_scales;
  const float* w_scales;
  const float* bias;
  long long ldy;
  int* dev_status;
  // tokens that are quantized here (FUSED): unquantized rows and what ocs_quantize_rows takes
  const void* X;
  long long ldx;
  const int32_t* idx_map;
  int x_type, x_align, C, K;
  float hi;
};

// TN tokens, CG CTAs per tensor-core tile
template <int TN, int CG, bool FUSED>
struct RowSmem {
  static constexpr int kTokens = TN / CG;                       // token rows this CTA stages
  static constexpr int kWBytes = TW * KB, kTBytes = kTokens * KB;
  static constexpr int kSub = stage_blocks(TN);
  static constexpr int kStageBytes = kSub * (FUSED ? kWBytes : kWBytes + kTBytes);
  // FUSED: the codes of all the K-blocks a CTA takes stay in a region of their own
  static constexpr int kTokenBytes = FUSED ? kFusedCodes : 0;
  // partial sums of this CTA's share (K split): a buffer of their own, or the operand ring where it would cost the ring
  // too many stages
  static constexpr int kXBytes = TN == 256 ? 0 : TN * TW * 4;
  static constexpr bool kXInRing = TN == 128;
  static constexpr int kXExtra = kXInRing ? 0 : kXBytes;
  static constexpr int kWarpTokens = TN < 32 ? 16 : TN / 2;      // columns an epilogue warp finishes
  static constexpr int kScaleBytes = kEpiWarps * kWarpTokens * 4;
  static constexpr int kCtrlBytes = 512;
  static constexpr int kRowBytes = FUSED ? TN * 12 : 0;            // a row's maximum, scale and 1 / step
  static constexpr int kBudget = 227 * 1024 - 1024 - kCtrlBytes - kScaleBytes - kRowBytes - kTokenBytes;
  static constexpr int kStagesFit = (kBudget - kXExtra) / kStageBytes;
  static constexpr int kStages = kStagesFit < 8 ? kStagesFit : 8;
  static constexpr int kDynBytes = 1024 + kStages * kStageBytes + kTokenBytes + kXExtra + kScaleBytes + kRowBytes + kCtrlBytes;
  static constexpr int kAccStride = TN < 32 ? 32 : TN;
  static constexpr uint32_t kTmemCols = 2 * kAccStride;
  static_assert(kStages >= 3 && (!kXInRing || kXBytes <= kStages * kStageBytes) && kDynBytes <= 227 * 1024 && kTBytes % 1024 == 0, "tile does not fit");
};

__host__ __device__ constexpr uint32_t row_instr_desc(int m, int n, int b_signed) {
  return (2u << 4)                               // accumulator S32
         | (1u << 7)                             // A (weights): int8
         | ((uint32_t)(b_signed ? 1 : 0) << 10)  // B (tokens): uint8 / int8
         | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

// Tile t of the launch: token tiles in groups of eight, all channel tiles of a group before the next group, so that
// the tiles in flight at one time share their operand panels in L2.
__device__ __forceinline__ void tile_of(const RowGemm& p, int t, int* mt, int* nt) {
  const int per_group = 8 * p.n_tiles;
  const int g = t / per_group, in = t - g * per_group;
  const int rows = min(8, p.m_tiles - 8 * g);
  *nt = in / rows;
  *mt = 8 * g + in - *nt * rows;
}

template <typename T> struct Pair;
template <> struct Pair<__half> { static __device__ __forceinline__ uint32_t pack(float a, float b) { __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); } };
template <> struct Pair<__nv_bfloat16> { static __device__ __forceinline__ uint32_t pack(float a, float b) { __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<uint32_t*>(&h); } };

// One output: (float(acc) * a_scale) * w_scale + bias; the conversion, the first product and the fused rest round once each.
// (The accumulator comes first: the two scales' product alone may leave fp32's normal range for rows of tiny values.)
__device__ __forceinline__ float one_output(int acc, float as, float ws, float b) {
  return fmaf(__fmul_rn(__int2float_rn(acc), as), ws, b);
}

// CNT consecutive tokens of one channel per lane, rounded to T and stored; the lanes of the warp hold consecutive
// channels.  y: the lane's channel of the first token; left: tokens of the tile that exist, from the first on.
// WHOLE: all CNT tokens and all 32 channels exist.
template <bool WHOLE, typename T, int CNT>
__device__ __forceinline__ void finish(T* y, long long ldy, const int* acc, const float* sc, float ws, float b, int left,
                                       bool n_ok, bool pairs) {
  if constexpr (sizeof(T) == 2) {
    if (pairs) {
      // neighbouring lanes swap halves, so that a lane stores two channels of one token in 32 bits: the even lane token j,
      // channels n and n + 1, the odd lane token j + 1, channels n - 1 and n
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

// Four consecutive elements of a row, 8-byte aligned (wide: 16-byte).
template <typename T>
struct Four {
  uint32_t w[sizeof(T)];
  __device__ __forceinline__ void load(const T* x, bool wide) {
    if constexpr (sizeof(T) == 2) {
      const uint2 v = __ldg(reinterpret_cast<const uint2*>(x));
      w[0] = v.x; w[1] = v.y;
    } else if (wide) {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(x));
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else {
      const uint2 v = __ldg(reinterpret_cast<const uint2*>(x)), u = __ldg(reinterpret_cast<const uint2*>(x) + 1);
      w[0] = v.x; w[1] = v.y; w[2] = u.x; w[3] = u.y;
    }
  }
  __device__ __forceinline__ float operator[](int i) const { return to_f32(reinterpret_cast<const T*>(w)[i]); }
};

// One value's code: ocs_quantize_rows' arithmetic for a row with maximum bits `max_bits`.
__device__ __forceinline__ int token_code(float x, float inv, uint32_t max_bits, int is_signed) {
  const float v = __uint_as_float(max_bits) < 0x1p-100f ? __fmul_rn(x, 0x1p64f) : x;
  return is_signed ? row_code<true>(v, inv) : row_code<false>(v, inv);
}

// The epilogue warps quantize the token tile that starts at row m0 straight into the operand tiles of stages slice,
// slice + slices, ...: first the rows' maxima, 512 elements per warp and step, then the codes, one row of a K-block per
// warp and step.  What does not come in whole fours of channels goes one by one: a row's last C % 4 channels and the
// duplicated ones (item u: contraction index C4 + u / rows of row u % rows; the first item's value is on its way from the
// start).  The latency of the loads is what this costs, so those of several steps are issued before the first is used.
template <typename X, int TN>
__device__ __forceinline__ void quantize_tokens(const RowGemm& p, const X* x0, int m0, int slice, int my_kb, unsigned char* tok,
                                                uint32_t* max_bits, float* scale, float* inv) {
  constexpr int B = 4, D = 4;   // steps whose loads are under way together
  const int et = threadIdx.x - 64, warp = et >> 5, lane = et & 31;
  const int rows = min(TN, p.M - m0), C4 = p.C & ~3, n_items = rows * (p.K - C4);
  const bool wide = p.x_align >= 16;
  // where the code of item (contraction index k, row r) goes; -1: not in this CTA's share
  auto place = [&](int k, int r) {
    constexpr int kSub = stage_blocks(TN);
    const int st = k / (kSub * KB), i = st / p.slices, in = k % KB;
    return st - i * p.slices == slice ? ((i * kSub + k / KB % kSub) * TN + r) * KB + (((in >> 4) ^ (r & 7)) << 4) + (in & 15) : -1;
  };
  int src = 0, at = -1, item_row = 0, item_k = 0;
  if (et < n_items) {
    item_k = et / rows;
    item_row = et - item_k * rows;
    src = item_k += C4;
    if (src >= p.C) src = __ldg(p.idx_map + src);
    at = place(item_k, item_row);
  }
  if (et < TN) max_bits[et] = 0;
  asm volatile("bar.sync 1, 256;" ::: "memory");
  const int chunks = (C4 + 511) / 512, units = rows * chunks;
  for (int u0 = warp; u0 < units; u0 += B * kEpiWarps) {
    Four<X> f[B][4];
    int rr[B];
#pragma unroll
    for (int b = 0; b < B; ++b) {
      const int u = min(u0 + b * kEpiWarps, units - 1), r = u / chunks, c = (u - r * chunks) * 512 + lane * 4;
      rr[b] = r;
#pragma unroll
      for (int j = 0; j < 4; ++j) f[b][j].load(x0 + r * p.ldx + min(c + 128 * j, C4 - 4), wide);   // (twice at the end: harmless)
    }
#pragma unroll
    for (int b = 0; b < B; ++b) {
      uint32_t m = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) m = max(m, __float_as_uint(f[b][j][i]) & 0x7fffffffu);
      m = __reduce_max_sync(0xffffffffu, m);
      if (lane == 0) atomicMax(max_bits + rr[b], m);
    }
  }
  float value = 0.0f;
  if (et < n_items) {
    if ((unsigned)src >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); src = 0; }
    value = to_f32(x0[item_row * p.ldx + src]);
    if (item_k < p.C) atomicMax(max_bits + item_row, __float_as_uint(value) & 0x7fffffffu);   // (all of these are first items)
  }
  asm volatile("bar.sync 1, 256;" ::: "memory");
  if (et < rows) {
    const float alpha = __uint_as_float(max_bits[et]);
    scale[et] = __fdiv_rn(alpha, p.hi);
    inv[et] = row_grid(alpha, p.hi).inv;
    if (max_bits[et] >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
  }
  asm volatile("bar.sync 1, 256;" ::: "memory");
  if (at >= 0) tok[at] = (unsigned char)token_code(value, inv[item_row], max_bits[item_row], p.t_signed);
  constexpr int kSub = stage_blocks(TN);
  const int steps = C4 > 0 ? my_kb * kSub * rows : 0;
  for (int u0 = warp; u0 < steps; u0 += D * kEpiWarps) {
    Four<X> f[D];
    int rr[D], to[D];
#pragma unroll
    for (int b = 0; b < D; ++b) {
      const int u = u0 + b * kEpiWarps, i = u / rows, r = u - i * rows, k = ((slice + i / kSub * p.slices) * kSub + i % kSub) * KB + lane * 4;
      rr[b] = u < steps ? r : 0;
      // past the last contraction index the weights' tile is zero
      to[b] = u < steps && k < C4 ? (i * TN + r) * KB + (((lane >> 2) ^ (r & 7)) << 4) + (lane & 3) * 4 : -1;
      f[b].load(x0 + rr[b] * p.ldx + (to[b] >= 0 ? k : 0), wide);
    }
#pragma unroll
    for (int b = 0; b < D; ++b) {
      int c[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) c[e] = token_code(f[b][e], inv[rr[b]], max_bits[rr[b]], p.t_signed);
      if (to[b] >= 0) *reinterpret_cast<uint32_t*>(tok + to[b]) = pack4(c[0], c[1], c[2], c[3]);
    }
  }
  for (int u = et + 256; u < n_items; u += 256) {
    const int d = u / rows, r = u - d * rows, to = place(C4 + d, r);
    if (to < 0) continue;
    src = __ldg(p.idx_map + C4 + d);
    if ((unsigned)src >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); src = 0; }
    tok[to] = (unsigned char)token_code(to_f32(x0[r * p.ldx + src]), inv[r], max_bits[r], p.t_signed);
  }
  fence_proxy_async_smem();   // the tensor cores read what these threads wrote
}

template <typename T, int TN, int CG, bool FUSED>
__global__ void __launch_bounds__(kThreads, 1)
row_gemm_kernel(const __grid_constant__ CUtensorMap tm_w, const __grid_constant__ CUtensorMap tm_t, const RowGemm p,
                T* __restrict__ Y) {
  using L = RowSmem<TN, CG, FUSED>;
  extern __shared__ unsigned char smem_dyn[];
  const uint32_t raw = smem_u32(smem_dyn);
  const uint32_t base = (raw + 1023u) & ~1023u;
  unsigned char* tiles = smem_dyn + (base - raw);
  unsigned char* tokens = tiles + L::kStages * L::kStageBytes;
  unsigned char* after = tokens + L::kTokenBytes;
  unsigned char* xbuf = L::kXInRing ? tiles : after;
  float* scale_buf = reinterpret_cast<float*>(after + L::kXExtra);
  uint32_t* row_max = reinterpret_cast<uint32_t*>(after + L::kXExtra + L::kScaleBytes);   // FUSED: [TN] maxima, scales, inv
  float* row_scale = reinterpret_cast<float*>(row_max + TN);
  uint64_t* bars = reinterpret_cast<uint64_t*>(after + L::kXExtra + L::kScaleBytes + L::kRowBytes);
  auto full_bar = [&](int s) { return smem_u32(bars + s); };
  auto empty_bar = [&](int s) { return smem_u32(bars + L::kStages + s); };
  auto accfull_bar = [&](int a) { return smem_u32(bars + 2 * L::kStages + a); };
  auto accempty_bar = [&](int a) { return smem_u32(bars + 2 * L::kStages + 2 + a); };
  const uint32_t xfull_bar = smem_u32(bars + 2 * L::kStages + 4);
  const uint32_t xready_bar = smem_u32(bars + 2 * L::kStages + 5);
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(bars + 2 * L::kStages + 6);
  volatile int* abort_flag = reinterpret_cast<volatile int*>(tmem_slot + 1);
  static_assert((2 * L::kStages + 6) * 8 + 8 <= L::kCtrlBytes, "control block");

  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int CL = CG * p.slices;
  const int rank = CL > 1 ? (int)cluster_rank() : 0;
  const int half = rank % CG, slice = rank / CG;
  const int cluster = blockIdx.x / CL, n_clusters = gridDim.x / CL;
  const int my_kb = (p.num_kb - slice + p.slices - 1) / p.slices;

  // Set-up.  Nobody waits for more than it needs: the copy warp asks for the first weights as soon as its own barriers
  // stand, the tensor-core warp needs these barriers, the epilogue warps the address in tensor memory as well -- after
  // they have quantized the tokens, where that is theirs to do.  (Named barriers: 2 = set up, 3 = barriers stand, 4 =
  // tokens in place.)  A peer may be written to once all threads of the cluster have arrived; a pair waits for that at
  // once, the others where they first need it.
  if (warp == 0) {
    if (lane == 0) {
      prefetch_tmap(&tm_w);
      if (!FUSED) prefetch_tmap(&tm_t);
      for (int s = 0; s < L::kStages; ++s) {
        mbar_init(full_bar(s), 1);     // the leader's producer announces the bytes of both CTAs
        mbar_init(empty_bar(s), 1);    // commit of the MMAs that read the stage
      }
      for (int a = 0; a < 2; ++a) {
        mbar_init(accfull_bar(a), 1);
        mbar_init(accempty_bar(a), CG * kEpiWarps);
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
    asm volatile("bar.arrive 2, 320;" ::: "memory");
    if (CL > 1) cluster_arrive();
  } else if (warp == 1) {
    if (CG == 2) tmem_alloc_pair(smem_u32(tmem_slot), L::kTmemCols);
    else tmem_alloc(smem_u32(tmem_slot), L::kTmemCols);
    tc_fence_before();
    asm volatile("bar.arrive 2, 320;" ::: "memory");
    if (CL > 1) cluster_arrive();
    asm volatile("bar.sync 3, 64;" ::: "memory");
  } else {
    if (CL > 1) cluster_arrive();
    if (FUSED) {
      // every tile of this CTA has the same tokens; they need nothing of the set-up
      int mt, nt;
      tile_of(p, cluster, &mt, &nt);
      const long long at = (long long)mt * TN * p.ldx;
      float* inv = row_scale + TN;
      if (p.x_type == OCS_F32) quantize_tokens<float, TN>(p, static_cast<const float*>(p.X) + at, mt * TN, slice, my_kb, tokens, row_max, row_scale, inv);
      else if (p.x_type == OCS_F16) quantize_tokens<__half, TN>(p, static_cast<const __half*>(p.X) + at, mt * TN, slice, my_kb, tokens, row_max, row_scale, inv);
      else quantize_tokens<__nv_bfloat16, TN>(p, static_cast<const __nv_bfloat16*>(p.X) + at, mt * TN, slice, my_kb, tokens, row_max, row_scale, inv);
      asm volatile("bar.arrive 4, 288;" ::: "memory");   // this warp's codes are in place
    }
    asm volatile("bar.sync 2, 320;" ::: "memory");
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
      // weights do not depend on the kernel before: the first ring of them is requested before waiting for it
      int ahead = 0;
      int mt, nt;
      auto load_w = [&](int s, int kb) {
#pragma unroll
        for (int u = 0; u < L::kSub; ++u) {
          const uint32_t dst = base + s * L::kStageBytes + u * L::kWBytes;
          const int x = (kb * L::kSub + u) * KB;
          if (CG == 2) tma_load_2d_pair(dst, &tm_w, peer_addr(full_bar(s), lead), x, (nt * CG + half) * TW);
          else tma_load_2d(dst, &tm_w, full_bar(s), x, nt * TW);
        }
      };
      auto load_t = [&](int s, int kb) {
#pragma unroll
        for (int u = 0; u < L::kSub; ++u) {
          const uint32_t dst = base + s * L::kStageBytes + L::kSub * L::kWBytes + u * L::kTBytes;
          const int x = (kb * L::kSub + u) * KB;
          if (CG == 2) tma_load_2d_pair(dst, &tm_t, peer_addr(full_bar(s), lead), x, mt * TN + half * L::kTokens);
          else tma_load_2d(dst, &tm_t, full_bar(s), x, mt * TN);
        }
      };
      if (cluster < p.total) {
        tile_of(p, cluster, &mt, &nt);
        ahead = min(L::kStages, my_kb);
        for (int i = 0; i < ahead; ++i) {
          if (half == 0) mbar_arrive_expect_tx(full_bar(i), CG * L::kStageBytes);
          load_w(i, slice + i * p.slices);
        }
      }
      if (!FUSED) grid_wait_previous();
      for (int t = cluster; ok && t < p.total; t += n_clusters) {
        tile_of(p, t, &mt, &nt);
        for (int i = 0; i < my_kb; ++i, ++it) {
          const int s = it % L::kStages;
          if (it >= ahead) {
            if (!mbar_wait(empty_bar(s), (uint32_t)((it / L::kStages) & 1) ^ 1u, abort_flag)) { ok = false; break; }
            if (half == 0) mbar_arrive_expect_tx(full_bar(s), CG * L::kStageBytes);
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
    if (FUSED) asm volatile("bar.sync 4, 288;" ::: "memory");   // the tokens' codes are in place
    if (lane == 0 && half == 0) {
      constexpr uint32_t kDescM = TW * CG;
      const uint32_t idesc = row_instr_desc(kDescM, TN, p.t_signed);
      const uint16_t mask = (uint16_t)(3u << (rank & ~1));
      // This thread's instructions between two K-blocks are what bounds the narrow forms, so the loop carries a stage's
      // addresses along instead of working them out.
      const uint64_t w_desc0 = smem_desc_sw128(base), t_desc0 = smem_desc_sw128(FUSED ? smem_u32(tokens) : base + L::kSub * L::kWBytes);
      int j = 0, s = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int t = cluster; ok && t < p.total; t += n_clusters, ++j) {
        const int acc = j & 1;
        if (!mbar_wait_cluster(accempty_bar(acc), (((uint32_t)j >> 1) & 1u) ^ 1u, abort_flag)) break;
        tc_fence_after();
        const uint32_t d = tmem_base + (uint32_t)(acc * L::kAccStride);
        uint32_t more = 0;
        uint64_t t_desc = t_desc0;   // FUSED: one token tile after the other
        for (int i = 0; i < my_kb; ++i) {
          if (!mbar_wait(full_bar(s), phase, abort_flag)) { ok = false; break; }
          tc_fence_after();
          const uint64_t w_desc = w_desc0 + (uint32_t)(s * (L::kStageBytes >> 4));
          if (!FUSED) t_desc = t_desc0 + (uint32_t)(s * (L::kStageBytes >> 4));
#pragma unroll
          for (int k = 0; k < L::kSub * KB / UK; ++k) {   // 32 bytes on, 2 in the descriptors' units of 16
            const int u = k / (KB / UK), in = k % (KB / UK);
            const uint64_t w = w_desc + u * (L::kWBytes >> 4) + 2 * in, x = t_desc + u * (L::kTBytes >> 4) + 2 * in;
            if (CG == 2) umma_i8_pair(d, w, x, idesc, k == 0 ? more : 1u);
            else umma_i8(d, w, x, idesc, k == 0 ? more : 1u);
          }
          more = 1;
          if (FUSED) t_desc += L::kSub * (L::kTBytes >> 4);
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
  } else {
    // ---------------------------------------------------------------- epilogue
    constexpr int EC = 16;                              // accumulator columns (tokens) moved at a time
    const int ew = warp - 2, q = warp & 3, part = ew >> 2;   // lanes 32q.. of tensor memory; two warps share a quadrant
    float* sc = scale_buf + ew * L::kWarpTokens;
    const bool pairs = sizeof(T) == 2 && (p.ldy % 2 == 0) && (p.N % 2 == 0) && (reinterpret_cast<uintptr_t>(Y) & 3) == 0;
    if (!FUSED) grid_wait_previous();
    if (CL > 1 && CG == 1) cluster_wait();
    int j = 0;
    for (int t = cluster; t < p.total; t += n_clusters, ++j) {
      int mt, nt;
      tile_of(p, t, &mt, &nt);
      const int acc = j & 1;
      const int n = (nt * CG + half) * TW + q * 32 + lane;
      const float ws = n < p.N ? __ldg(p.w_scales + n) : 0.0f;
      const float b = p.bias && n < p.N ? __ldg(p.bias + n) : 0.0f;
      if (p.slices > 1) {
        // K split: owner o of the tile's slices finishes tokens [o * own, (o + 1) * own).  Every CTA sends the columns
        // another one owns into that one's buffer, cells of 16 bytes [sender][four tokens][channel], counted as
        // transaction bytes on the owner's barrier.
        if constexpr (L::kXBytes > 0) {
          const int own = TN / p.slices, groups = own / 4;
          // the scales of the tokens this CTA finishes, while the main loop runs
          __syncwarp();
          for (int i = lane; i < own; i += 32) {
            const int m = mt * TN + slice * own + i;
            sc[i] = m < p.M ? (FUSED ? row_scale[slice * own + i] : __ldcg(p.a_scales + m)) : 0.0f;
          }
          __syncwarp();
          if (!mbar_wait(accfull_bar(acc), ((uint32_t)j >> 1) & 1u, abort_flag)) break;
          tc_fence_after();
          if (L::kXInRing) {
            // this CTA's tensor cores are done with its ring: it may be written to; and so are all the others'
            if (ew == 0 && lane == 0)
              for (int o = 0; o < p.slices; ++o) mbar_arrive_peer(peer_addr(xready_bar, (uint32_t)o));
            if (!mbar_wait_cluster(xready_bar, 0u, abort_flag)) break;
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
          if (!mbar_wait_cluster(xfull_bar, 0u, abort_flag)) break;
          const int m_own = mt * TN + slice * own;
          T* y = Y + (long long)m_own * p.ldy + n;
          const uint32_t slot = (uint32_t)groups * TW * 16u;   // from one sender's cells to the next one's
          for (int g = part; g < groups; g += 2) {
            const unsigned char* cell = xbuf + (size_t)(g * TW + q * 32 + lane) * 16;
            int4 a = *reinterpret_cast<const int4*>(cell);
#pragma unroll 4
            for (int sl = 1; sl < p.slices; ++sl) {
              const int4 b4 = *reinterpret_cast<const int4*>(cell + sl * slot);
              a.x += b4.x; a.y += b4.y; a.z += b4.z; a.w += b4.w;
            }
            const int av[4] = {a.x, a.y, a.z, a.w};
            const float4 s4 = *reinterpret_cast<const float4*>(sc + 4 * g);
            const float sv[4] = {s4.x, s4.y, s4.z, s4.w};
            finish<false, T, 4>(y + 4 * g * p.ldy, p.ldy, av, sv, ws, b, p.M - m_own - 4 * g, n < p.N, pairs);
          }
        }
        break;   // a K split is used only where every cluster has one tile
      }
      // the token scales of this warp's columns: fetched while the main loop runs
      __syncwarp();
      for (int i = lane; i < L::kWarpTokens; i += 32) {
        const int col = (i / EC) * 2 * EC + part * EC + i % EC, m = mt * TN + col;
        sc[i] = m < p.M ? (FUSED ? row_scale[col] : __ldcg(p.a_scales + m)) : 0.0f;
      }
      __syncwarp();
      if (!mbar_wait(accfull_bar(acc), ((uint32_t)j >> 1) & 1u, abort_flag)) break;
      tc_fence_after();
      // pieces of EC columns; the next one's way out of tensor memory overlaps this one's arithmetic and stores
      constexpr int kPieces = TN >= 2 * EC ? TN / (2 * EC) : 1;
      const uint32_t addr = tmem_base + ((uint32_t)(q * 32) << 16) + (uint32_t)(acc * L::kAccStride + part * EC);
      const bool n_all = (nt * CG + half) * TW + q * 32 + 32 <= p.N;
      T* y = Y + (long long)(mt * TN + part * EC) * p.ldy + n;
      int left = p.M - mt * TN - part * EC;   // tokens from this piece's first on
      uint32_t v[2][EC];
      if (part * EC < TN && left > 0) {
        tmem_ld_async<EC>(addr, v[0]);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
          if (left <= 0) break;               // the same for the whole warp
          tmem_wait_ld16(v[i & 1]);
          if (i + 1 < kPieces && left > 2 * EC) tmem_ld_async<EC>(addr + 2 * EC * (i + 1), v[(i + 1) & 1]);
          float s[EC];
#pragma unroll
          for (int e = 0; e < EC; e += 4) {
            const float4 f = *reinterpret_cast<const float4*>(sc + i * EC + e);
            s[e] = f.x; s[e + 1] = f.y; s[e + 2] = f.z; s[e + 3] = f.w;
          }
          const int* av = reinterpret_cast<const int*>(v[i & 1]);
          if (n_all && left >= EC) finish<true, T, EC>(y, p.ldy, av, s, ws, b, left, true, pairs);
          else finish<false, T, EC>(y, p.ldy, av, s, ws, b, left, n < p.N, pairs);
          y += 2 * EC * p.ldy;
          left -= 2 * EC;
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        if (CG == 2) mbar_arrive_peer(peer_addr(accempty_bar(acc), (uint32_t)(rank & ~1)));
        else mbar_arrive(accempty_bar(acc));
      }
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
// Bytes of a token tile, unquantized, that a CTA may read itself (min(M, tokens per tile) rows).  The host decides here: at
// these sizes an eager call is bound by it, and one launch takes 12 to 14 us of it, two take 17.  On the device the fused
// form is even up to 16 KB and slower beyond, since every CTA reads its rows twice before its first product.  us by graph
// replay, fused against two launches: (M, C, N) = (1, 4096, 4096), 8 KB: 8.7 against 8.6; (1, 8192, 8192), 16 KB: 16.5 against
// 16.6; (16, 1024, 4096), 32 KB: 6.5 against 5.6; (20, 650, 2600) in fp32, 41.6 KB a tile: 8.0 against 5.9.  At (4, 8192,
// 8192), 64 KB, the device is the slower side: 20.2 against 17.0.  A caller that replays graphs takes ocs_quantize_rows and
// ocs_qlinear_rows instead, which give the same bits.
constexpr long long kFuseBytes = 48 * 1024;

struct RowPlan {
  int tn, cg, slices;
};

// Test hook (ocs_selftest_force_row_plan): the plan of the following calls where it is valid for the problem, in one word
// so that a call in another thread sees a whole plan: tn << 8 | cg << 4 | slices, 0 for none.
std::atomic<int> g_forced_plan{0};

// CTAs resident at once, one per SM, for cluster sizes 1, 2, 4, 8 (a cluster lies inside one GPC)
int cluster_capacity(int cl) { return cl <= 2 ? 148 : (cl == 4 ? 132 : 120); }

int stages_of(int tn, int num_kb) { return (num_kb + stage_blocks(tn) - 1) / stage_blocks(tn); }

bool split_fits(int tn, int cg, int slices, long long tiles, int stages) {
  if (slices == 1) return true;
  return cg == 1 && tn < 256 && tn / slices >= 4 && slices <= stages && tiles * slices <= cluster_capacity(slices);
}

// The plan by a time model in microseconds, fitted to 806 measurements (M 1..4096, K 300..25339, N 1024..33278, fp32 and
// 16-bit outputs, every plan that fits): root mean square error 5.5 %; the plan it picks is 0.4 % slower than the best
// measured one on average, 10 % at worst.  A tile costs its K-blocks and its epilogue, which adds to them instead of hiding
// behind them (the stores and the next tile's operand requests share the SM's way out), and 0.29 us; a K split adds the
// exchange; the bytes take their time at 6.2 TB/s; of the two the longer one counts most (root of the sum of squares); and
// 3.9 us pass before the first and after the last tile.
RowPlan choose_plan(int M, int N, int num_kb, int out_bytes) {
  struct Form { int tn, cg; double block_us, epilogue_us; };
  static const Form forms[6] = {{16, 1, 0.18, 0.0},  {32, 1, 0.18, 0.01},  {64, 1, 0.18, 0.27},
                                {128, 1, 0.23, 0.91}, {256, 1, 0.33, 2.17}, {256, 2, 0.27, 3.02}};
  auto tiles_of = [&](int tn, int cg) {
    return (long long)((M + (long long)tn - 1) / tn) * ((N + (long long)TW * cg - 1) / (TW * cg));
  };
  if (const int forced = g_forced_plan.load()) {
    RowPlan r{forced >> 8, forced >> 4 & 15, forced & 15};
    while (r.slices > 1 && !split_fits(r.tn, r.cg, r.slices, tiles_of(r.tn, r.cg), stages_of(r.tn, num_kb))) r.slices /= 2;
    return r;
  }
  const double K = (double)num_kb * KB;
  const double bytes_us = ((double)N * K + (double)M * K + (double)M * N * out_bytes) / 6.22e6;
  RowPlan best{16, 1, 1};
  double best_us = 1e300;   // squared
  for (const Form& f : forms) {
    const long long tiles = tiles_of(f.tn, f.cg);
    for (int s = 1; s <= 8; s *= 2) {
      if (!split_fits(f.tn, f.cg, s, tiles, stages_of(f.tn, num_kb))) continue;
      const long long slots = cluster_capacity(f.cg * s) / (f.cg * s);
      const double waves = (double)((tiles + slots - 1) / slots);
      const int blocks = (stages_of(f.tn, num_kb) + s - 1) / s * stage_blocks(f.tn);
      double us = waves * (blocks * f.block_us + f.epilogue_us * (out_bytes == 4 ? 1.2 : 1.0) + 0.29);
      if (s > 1) us += 3.85 * f.tn / 128.0;
      us = us * us + bytes_us * bytes_us;   // (its root, plus a constant)
      if (us < best_us) { best_us = us; best = RowPlan{f.tn, f.cg, s}; }
    }
  }
  return best;
}

template <typename T, int TN, int CG, bool FUSED = false>
ocs_status launch_tiles(RowGemm p, int slices, const void* A, long long lda, const int8_t* W, long long ldw, int K, T* Y,
                        bool overlap, cudaStream_t stream) {
  using L = RowSmem<TN, CG, FUSED>;
  static std::atomic<unsigned long long> ready{0};   // devices whose copy of the kernel has its attribute set
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return OCS_ERR_CUDA;
  if (dev >= 64 || !(ready.load() >> dev & 1)) {
    if (cudaFuncSetAttribute(row_gemm_kernel<T, TN, CG, FUSED>, cudaFuncAttributeMaxDynamicSharedMemorySize, L::kDynBytes) != cudaSuccess)
      return OCS_ERR_CUDA;
    if (dev < 64) ready.fetch_or(1ull << dev);
  }
  p.n_tiles = (p.N + TW * CG - 1) / (TW * CG);
  p.m_tiles = (p.M + TN - 1) / TN;
  const long long total = (long long)p.n_tiles * p.m_tiles;
  if (total > 0x3fffffff) return OCS_ERR_UNSUPPORTED;
  p.total = (int)total;
  p.slices = slices;
  CUtensorMap tm_w, tm_t;
  const cuuint64_t wd[2] = {(cuuint64_t)K, (cuuint64_t)p.N}, ws[1] = {(cuuint64_t)ldw};
  const cuuint64_t td[2] = {(cuuint64_t)K, (cuuint64_t)p.M}, ts[1] = {(cuuint64_t)lda};
  const cuuint32_t wb[2] = {KB, TW}, tb[2] = {KB, (cuuint32_t)L::kTokens};
  if (!encode_u8(&tm_w, W, 2, wd, ws, wb)) return OCS_ERR_CUDA;
  if (FUSED) tm_t = tm_w;   // unused
  else if (!encode_u8(&tm_t, A, 2, td, ts, tb)) return OCS_ERR_CUDA;
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
  LaunchScope scope(FUSED ? "row_gemm_kernel(fused)" : "row_gemm_kernel", stream);
  if (cudaLaunchKernelEx(&cfg, row_gemm_kernel<T, TN, CG, FUSED>, tm_w, tm_t, p, Y) != cudaSuccess) return OCS_ERR_CUDA;
  return launch_status();
}

// Whether ocs_linear_rows quantizes inside the product's kernel: every CTA quantizes its token tile itself.  That saves a
// launch, but each CTA reads the whole rows, so it is for few tokens.
bool fuse_tokens(const RowPlan& plan, int M, int N, int C, int num_kb, int x_bytes, int x_align) {
  if (plan.tn > 32 || plan.cg != 1 || x_align < 8) return false;
  const long long m_tiles = (M + plan.tn - 1) / plan.tn, tiles = m_tiles * ((N + (long long)TW - 1) / TW);
  const int my_kb = (stages_of(plan.tn, num_kb) + plan.slices - 1) / plan.slices * stage_blocks(plan.tn);
  if ((long long)my_kb * plan.tn * KB > kFusedCodes) return false;                                // the codes have to fit
  if (m_tiles > 1 && tiles > cluster_capacity(plan.slices) / plan.slices) return false;           // one token tile per CTA
  return (long long)(M < plan.tn ? M : plan.tn) * C * x_bytes <= kFuseBytes;
}

struct Product {
  const void* A;
  const float* a_scales;
  const int8_t* W;
  const float* w_scales;
  const float* bias;
  int M, N, K, a_signed;
  long long lda, ldw, ldy;
  int* dev_status;
  // not quantized yet (A = a_scales = NULL)
  const void* X;
  long long ldx;
  const int32_t* idx_map;
  ocs_dtype x_type;
  int x_align, C;
  float hi;
};

template <typename T>
ocs_status launch_product(const Product& g, const RowPlan& plan, void* Y_, bool overlap, cudaStream_t stream) {
  RowGemm p{};
  p.M = g.M; p.N = g.N; p.t_signed = g.a_signed;
  p.a_scales = g.a_scales; p.w_scales = g.w_scales; p.bias = g.bias; p.ldy = g.ldy; p.dev_status = g.dev_status;
  const int num_kb = (g.K + KB - 1) / KB;
  p.num_kb = stages_of(plan.tn, num_kb);
  T* Y = static_cast<T*>(Y_);
  if (!g.A) {
    p.X = g.X; p.ldx = g.ldx; p.idx_map = g.idx_map; p.x_type = g.x_type; p.C = g.C; p.K = g.K; p.hi = g.hi;
    p.x_align = g.x_align;
    if (plan.tn == 16) return launch_tiles<T, 16, 1, true>(p, plan.slices, nullptr, 16, g.W, g.ldw, g.K, Y, false, stream);
    return launch_tiles<T, 32, 1, true>(p, plan.slices, nullptr, 16, g.W, g.ldw, g.K, Y, false, stream);
  }
  switch (plan.tn * 2 + plan.cg - 1) {
    case 32: return launch_tiles<T, 16, 1>(p, plan.slices, g.A, g.lda, g.W, g.ldw, g.K, Y, overlap, stream);
    case 64: return launch_tiles<T, 32, 1>(p, plan.slices, g.A, g.lda, g.W, g.ldw, g.K, Y, overlap, stream);
    case 128: return launch_tiles<T, 64, 1>(p, plan.slices, g.A, g.lda, g.W, g.ldw, g.K, Y, overlap, stream);
    case 256: return launch_tiles<T, 128, 1>(p, plan.slices, g.A, g.lda, g.W, g.ldw, g.K, Y, overlap, stream);
    case 512: return launch_tiles<T, 256, 1>(p, plan.slices, g.A, g.lda, g.W, g.ldw, g.K, Y, overlap, stream);
    default: return launch_tiles<T, 256, 2>(p, plan.slices, g.A, g.lda, g.W, g.ldw, g.K, Y, overlap, stream);
  }
}

ocs_status run_product(const Product& p, const RowPlan& plan, void* Y, ocs_dtype y_type, bool overlap, cudaStream_t stream) {
  switch (y_type) {
    case OCS_F16: return launch_product<__half>(p, plan, Y, overlap, stream);
    case OCS_BF16: return launch_product<__nv_bfloat16>(p, plan, Y, overlap, stream);
    default: return launch_product<float>(p, plan, Y, overlap, stream);
  }
}

ocs_status check_product(int a_signed, int M, int K, int64_t lda, const void* A, const int8_t* W, int N, int64_t ldw,
                         const float* bias, const void* Y, ocs_dtype y_type, int64_t ldy, const float* w_scales) {
  if (!W || !w_scales || !Y) return OCS_ERR_INVALID_ARG;
  if (lda < K || lda % 16 != 0 || !aligned(A, 16)) return OCS_ERR_SHAPE;
  if (ldw < K || ldw % 16 != 0 || !aligned(W, 16)) return OCS_ERR_SHAPE;
  if (ldy < N || !aligned(Y, elem_bytes(y_type)) || !aligned(w_scales, 4) || (bias && !aligned(bias, 4))) return OCS_ERR_SHAPE;
  if ((int64_t)K * 128 * (a_signed ? 128 : 255) > 2147483647ll || M >= (1 << 30) || N > 0x7fffffff - 512)
    return OCS_ERR_UNSUPPORTED;
  return OCS_OK;
}

}  // namespace
}  // namespace ocs

using namespace ocs;

extern "C" ocs_status ocs_qlinear_rows(const void* A_codes, int a_signed, const float* a_scales, int M, int K,
                                       int64_t lda, const int8_t* W_codes, const float* w_scales, int N, int64_t ldw,
                                       const float* bias, void* Y, ocs_dtype y_type, int64_t ldy, int* dev_status,
                                       void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!valid_dtype(y_type)) return OCS_ERR_INVALID_ARG;
  if (M < 0 || K <= 0 || N <= 0) return OCS_ERR_SHAPE;
  if (M == 0) return OCS_OK;
  if (!A_codes || !a_scales) return OCS_ERR_INVALID_ARG;
  ocs_status st = check_product(a_signed, M, K, lda, A_codes, W_codes, N, ldw, bias, Y, y_type, ldy, w_scales);
  if (st != OCS_OK) return st;
  if (!aligned(a_scales, 4)) return OCS_ERR_SHAPE;
  if ((st = check_device()) != OCS_OK) return st;
  Product p{A_codes, a_scales, W_codes, w_scales, bias, M, N, K, a_signed ? 1 : 0,
            lda, ldw, ldy, dev_status, nullptr, 0, nullptr, OCS_F32, 0, 0, 0.0f};
  return run_product(p, choose_plan(M, N, (K + KB - 1) / KB, elem_bytes(y_type)), Y, y_type, false, stream);
}

namespace {
// The plan of an ocs_linear_rows call, chosen once (the two forms of the call and their kernels have to agree on it), and the
// bytes of codes and scales it keeps in the workspace (0: quantized inside the product's kernel).
struct RowsCall {
  RowPlan plan;
  size_t ws_bytes;
};
int row_align(const void* X, int M, int64_t ldx, ocs_dtype x_type) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(X) | (M > 1 ? (uintptr_t)(ldx * elem_bytes(x_type)) : 0);
  return a % 16 == 0 ? 16 : (a % 8 == 0 ? 8 : 1);
}
RowsCall linear_rows_plan(const void* X, int M, int C, int64_t ldx, int S, int N, ocs_dtype x_type, ocs_dtype y_type) {
  const int K = C + S, num_kb = (K + KB - 1) / KB;
  const RowPlan plan = choose_plan(M, N, num_kb, elem_bytes(y_type));
  if (fuse_tokens(plan, M, N, C, num_kb, elem_bytes(x_type), row_align(X, M, ldx, x_type))) return {plan, 0};
  return {plan, align_up((size_t)M * align_up((size_t)K, 16), 256) + align_up((size_t)M * 4, 256)};
}
}  // namespace

extern "C" size_t ocs_linear_rows_workspace_bytes(const void* X, ocs_dtype x_type, int M, int C, int64_t ldx, int S, int N,
                                                  ocs_dtype y_type) {
  if (M <= 0 || C <= 0 || S < 0 || N <= 0 || !valid_dtype(x_type) || !valid_dtype(y_type) || (int64_t)C + S >= (1 << 30)) return 0;
  return linear_rows_plan(X, M, C, ldx, S, N, x_type, y_type).ws_bytes;
}

extern "C" ocs_status ocs_linear_rows(const void* X, ocs_dtype x_type, int M, int C, int64_t ldx, int S,
                                      const int32_t* idx_map, int bits, int is_signed, const int8_t* W_codes,
                                      const float* w_scales, int N, int64_t ldw, const float* bias, void* Y,
                                      ocs_dtype y_type, int64_t ldy, void* ws, size_t ws_bytes, int* dev_status,
                                      void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!valid_dtype(x_type) || !valid_dtype(y_type) || S < 0 || bits < 2 || bits > 8) return OCS_ERR_INVALID_ARG;
  if (M < 0 || C <= 0 || N <= 0) return OCS_ERR_SHAPE;
  if (M == 0) return OCS_OK;
  if (!X || (S > 0 && !idx_map)) return OCS_ERR_INVALID_ARG;
  if ((int64_t)C + S >= (1 << 30)) return OCS_ERR_UNSUPPORTED;
  const int K = C + S;
  const int64_t lda = (int64_t)align_up((size_t)K, 16);
  const RowsCall call = linear_rows_plan(X, M, C, ldx, S, N, x_type, y_type);
  const size_t need = call.ws_bytes;
  if (need && (!ws || !aligned(ws, 256) || ws_bytes < need)) return OCS_ERR_WORKSPACE;
  ocs_status st = check_product(is_signed, M, K, lda, nullptr, W_codes, N, ldw, bias, Y, y_type, ldy, w_scales);
  if (st != OCS_OK) return st;
  if (ldx < C || !aligned(X, elem_bytes(x_type)) || (S > 0 && !aligned(idx_map, 4))) return OCS_ERR_SHAPE;
  if ((st = check_device()) != OCS_OK) return st;
  Product p{nullptr, nullptr, W_codes, w_scales, bias, M, N, K, is_signed ? 1 : 0, lda, ldw, ldy, dev_status,
            X, ldx, idx_map, x_type, row_align(X, M, ldx, x_type), C, (float)(is_signed ? (1 << (bits - 1)) - 1 : (1 << bits) - 1)};
  if (need) {
    int8_t* codes = static_cast<int8_t*>(ws);
    float* scales = reinterpret_cast<float*>(codes + align_up((size_t)M * lda, 256));
    st = ocs_quantize_rows(X, x_type, M, C, ldx, S, idx_map, bits, is_signed, codes, lda, scales, dev_status, stream_);
    if (st != OCS_OK) return st;
    p.A = codes; p.a_scales = scales;
  }
  return run_product(p, call.plan, Y, y_type, true, stream);
}

// Test hook: the next ocs_qlinear_rows / ocs_linear_rows calls of this process use the given plan; tn = 0 gives the
// choice back.
extern "C" ocs_status ocs_selftest_force_row_plan(int tn, int cg, int slices) {
  if (tn != 0 && ((tn != 16 && tn != 32 && tn != 64 && tn != 128 && tn != 256) || (cg != 1 && !(cg == 2 && tn == 256)) ||
                  (slices != 1 && slices != 2 && slices != 4 && slices != 8)))
    return OCS_ERR_INVALID_ARG;
  g_forced_plan.store(tn ? tn << 8 | cg << 4 | slices : 0);
  return OCS_OK;
}
