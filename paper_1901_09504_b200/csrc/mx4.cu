// ocs_quantize_mx4 / ocs_dequantize_mx4: rows to block-scaled 4-bit codes, the duplicated channels of a split layer appended,
// and back.
#include "mx4.cuh"
#include "ptx.cuh"

namespace ocs {
namespace {

struct MxRows {
  long long rows, ldx, ld_codes;
  int C, K, nb, chunks;          // own channels, all channels, blocks, groups of four blocks
  const int32_t* idx_map;
  int code_align;                // bytes that all rows of codes are aligned to (16, 8, 4 or 1)
  uint8_t* codes;
  uint8_t* scales;
  float* row_scales;
  int* dev_status;
};

// A thread's unit of work: a piece of 32 (E4M3) or 64 bytes (E8M0) of a row, which is a block or half of one (kLanes
// neighbouring threads have the block).
template <typename T, int GRID>
struct Piece {
  static constexpr int N = (GRID == OCS_GRID_E8M0 ? 64 : 32) / (int)sizeof(T), kLanes = mx4_block(GRID) / N, BYTES = N / 2;
  static_assert(kLanes >= 1, "a block is at least a piece");
};

// Bits of the largest magnitude of the block that a thread's piece belongs to.
template <typename T, int GRID>
__device__ __forceinline__ uint32_t block_max(uint32_t m) {
#pragma unroll
  for (int o = 1; o < Piece<T, GRID>::kLanes; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  return m;
}

// Piece j of row r: codes, and by the block's first thread its scale.
template <typename T, int GRID>
__device__ __forceinline__ void store_piece(const MxRows& p, uint8_t* codes, uint8_t* scales, int j, const MxScale& s, const uint32_t* c) {
  using P = Piece<T, GRID>;
  if (j % P::kLanes == 0) {
    const int b = j / P::kLanes;
    uint8_t* at = scales + (b >> 2) * kMxTile + (b & 3);
    *at = (uint8_t)s.byte;
    if (b == p.nb - 1)
      for (int i = b + 1; i & 3; ++i) at[i - b] = 0;     // the group's blocks past the row's end
  }
  uint8_t* dst = codes + j * P::BYTES;
  const int left = (p.K + 1) / 2 - j * P::BYTES;          // bytes of the row from here on
  if (left >= P::BYTES && p.code_align >= P::BYTES) {
    if constexpr (P::BYTES == 16) *reinterpret_cast<uint4*>(dst) = make_uint4(c[0], c[1], c[2], c[3]);
    else if constexpr (P::BYTES == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(c[0], c[1]);
    else *reinterpret_cast<uint32_t*>(dst) = c[0];
  } else {
#pragma unroll
    for (int i = 0; i < P::BYTES; ++i)
      if (i < left) dst[i] = (uint8_t)(c[i / 4] >> (8 * (i & 3)));
  }
}

// Whether piece j of row r can be read by Block::load: all its elements are the row's own, and where rows start anywhere
// (ALIGN 0), what it reads around them lies in the matrix too (in neighbouring rows, or between them).
template <int N, int ALIGN>
__device__ __forceinline__ bool whole_piece(const MxRows& p, long long r, int j) {
  if ((j + 1) * N > p.C) return false;
  return ALIGN || ((r > 0 || j > 0) && (r + 1 < p.rows || (j + 2) * N <= p.C));
}

// The row's tail, from the first piece on that is not all its own, into shared memory by G threads, zeros up to the last
// piece's end: a thread per element, so that the indices come in one load and the values in another.
constexpr int kTailBytes = 8192;
template <typename T, int N>
__device__ __forceinline__ void stage_tail(const MxRows& p, const T* x, int first, int pieces, T* s, int tx, int G) {
  for (int e = tx; e < pieces * N; e += G) {
    int src = first + e;
    T v = from_f32<T>(0.0f);
    if (src < p.K) {
      if (src >= p.C) {
        src = __ldg(p.idx_map + src);
        if ((unsigned)src >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); src = 0; }
      }
      v = x[src];
    }
    s[e] = v;
  }
}

constexpr int kRowThreads = 512;
constexpr int kRowPieces = 4;       // most pieces per thread

// What bounds it: instructions beside HBM.  8192 x 8192 bf16 (134 MB in, 38 out, floor 26 us): E4M3 34 us, issue slots two
// thirds full at 12 instructions an element, E8M0 28 us; 333 x 5000 with 50 duplicated channels 3.1 us.  Rows that start anywhere
// read 48 bytes where they need 32 and shift them: 4085 x 7279 bf16 E4M3 23.0 us, E8M0 18.8 (4085 x 7296: 17.3 and 13.5, floor 11.6
// and 11.5).  40 registers a thread hold all but 4 to 28 bytes (spilled) of the 16-bit forms.
// G = blockDim.x threads (a power of two below 32, or whole warps) and NV pieces each for one row, or (E8M0, whose blocks need
// nothing of their row) a part of one: blockIdx.y.  blockDim.y rows per CTA.  E4M3: a row's scale is that of its largest
// magnitude, so the row waits in registers for it.
template <typename T, int GRID, int ALIGN, int NV>
__global__ void __launch_bounds__(kRowThreads, NV * Block<T, Piece<T, GRID>::N>::W > 16 ? 2 : 3) mx4_rows_kernel(const T* __restrict__ X, const MxRows p, int tail_room) {
  constexpr int N = Piece<T, GRID>::N;
  __shared__ uint32_t s_max[16];
  __shared__ __align__(16) unsigned char s_tail[kTailBytes];
  grid_launch_dependents();
  const int G = blockDim.x, tx = threadIdx.x, lane = (threadIdx.y * G + tx) & 31;
  const long long r = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  const bool live = r < p.rows;
  const T* x = X + (live ? r : 0) * p.ldx;
  const int lo = GRID == OCS_GRID_E8M0 ? (int)blockIdx.y * G * NV : 0, hi = min(lo + G * NV, p.nb * Piece<T, GRID>::kLanes);
  const int t0 = max(p.C / N, lo), tail = hi - t0;            // the tail's pieces in this part
  const bool staged = tail > 0 && tail <= tail_room;
  T* my_tail = reinterpret_cast<T*>(s_tail) + threadIdx.y * tail_room * N;
  Block<T, N> v[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int j = lo + tx + i * G;
    if (j >= hi || !live) v[i].clear();
    else if (whole_piece<N, ALIGN>(p, r, j)) v[i].template load<ALIGN>(x + j * N);
    else if (!staged || j < t0) v[i].template gather<(N > 16 ? 8 : N)>(x, j * N, p.C, p.K, p.idx_map, p.dev_status);
  }
  if (staged) {
    if (live) stage_tail<T, N>(p, x, t0 * N, tail, my_tail, tx, G);
    if (G > 32) __syncthreads();
    else __syncwarp();
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = lo + tx + i * G;
      if (j >= t0 && j < hi && live) v[i].from_shared(my_tail + (j - t0) * N);
    }
  }
  uint32_t mine[NV], m = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    mine[i] = block_max<T, GRID>(v[i].max_bits());
    m = max(m, mine[i]);
  }
  int k = 0;
  if constexpr (GRID == OCS_GRID_E4M3) {
    if (G >= 32) m = __reduce_max_sync(0xffffffffu, m);
    else
      for (int o = 1; o < G; o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (G > 32) {
      const int per = G >> 5, first = threadIdx.y * per;
      if (lane == 0) s_max[first + (tx >> 5)] = m;
      __syncthreads();
      m = __reduce_max_sync(0xffffffffu, lane < per ? s_max[first + lane] : 0u);
    }
    k = mx4_row_exponent(m);
    if (tx == 0 && live) p.row_scales[r] = two_to(k);
  }
  if (!live) return;
  if (m >= 0x7f800000u && (GRID == OCS_GRID_E8M0 || tx == 0)) flag(p.dev_status, OCS_DEV_NONFINITE);
  uint8_t* codes = p.codes + r * p.ld_codes;
  uint8_t* scales = p.scales + mx4_scale_at(r, 0, p.chunks);
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int j = lo + tx + i * G;
    if (j >= hi) break;
    const MxScale s = mx4_scale<GRID, T>(mine[i], k);
    uint32_t c[N / 8];
    v[i].template codes<GRID>(s, c);
    store_piece<T, GRID>(p, codes, scales, j, s, c);
  }
}

// E4M3, many long rows that start at 16-byte boundaries: one CTA per SM walks over them.  A row comes by one bulk copy into
// a ring of shared-memory buffers, moves into registers (which frees its buffer), and is quantized from there while the next
// rows are on their way.  4096 x 25088 fp32: 91 us (floor 72; read twice instead, the second time from L2: 102 us, in one go
// by CTAs of 1024 threads whose loads and stores take turns 151 us).
constexpr int kStagedThreads = 1024, kStagedRing = 4;
constexpr size_t kStagedBytes = 224 * 1024;
template <typename T>
__global__ void __launch_bounds__(kStagedThreads, 1) mx4_staged_rows_kernel(const T* __restrict__ X, const MxRows p, int ring) {
  constexpr int GRID = OCS_GRID_E4M3, N = Piece<T, GRID>::N, NV = kRowPieces;
  extern __shared__ __align__(128) unsigned char smem[];   // [ring] rows
  __shared__ __align__(8) uint64_t bars[kStagedRing];
  __shared__ uint32_t s_max[2][32];
  __shared__ int abort_flag;
  const int tx = threadIdx.x, lane = tx & 31, pieces = p.nb * Piece<T, GRID>::kLanes;
  const uint32_t row_bytes = (uint32_t)p.C * (uint32_t)sizeof(T);
  grid_launch_dependents();
  auto request = [&](long long r, int slot) {   // one thread
    const uint32_t bar = smem_u32(bars + slot);
    mbar_arrive_expect_tx(bar, row_bytes);
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];"
                 ::"r"(smem_u32(smem) + (uint32_t)slot * row_bytes), "l"(X + r * p.ldx), "r"(row_bytes), "r"(bar) : "memory");
  };
  if (tx == 0) {
    for (int i = 0; i < ring; ++i) mbar_init(smem_u32(bars + i), 1);
    abort_flag = 0;
    fence_barrier_init();
    fence_proxy_async_smem();
    for (int i = 0; i < ring; ++i)
      if (blockIdx.x + (long long)i * gridDim.x < p.rows) request(blockIdx.x + (long long)i * gridDim.x, i);
  }
  __syncthreads();
  int it = 0, slot = 0;
  uint32_t phase = 0;
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x, ++it) {
    const bool ok = mbar_wait(smem_u32(bars + slot), phase, &abort_flag);
    const T* row = reinterpret_cast<const T*>(smem + (size_t)slot * row_bytes);
    Block<T, N> v[NV];
    uint32_t mine[NV], m = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = tx + i * kStagedThreads;
      if ((j + 1) * N <= p.C) v[i].from_shared(row + j * N);
      else {
        v[i].clear();
        if (j < pieces)
#pragma unroll
          for (int e = 0; e < N; ++e) {
            int src = j * N + e;
            if (src < p.K) {
              if (src >= p.C) {
                src = __ldg(p.idx_map + src);
                if ((unsigned)src >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); src = 0; }
              }
              if constexpr (sizeof(T) == 4) v[i].w[e] = reinterpret_cast<const uint32_t*>(row)[src];
              else v[i].w[e / 2] |= (uint32_t)reinterpret_cast<const uint16_t*>(row)[src] << (16 * (e & 1));
            }
          }
      }
      mine[i] = v[i].max_bits();
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      mine[i] = block_max<T, GRID>(mine[i]);
      m = max(m, mine[i]);
    }
    m = __reduce_max_sync(0xffffffffu, m);
    if (lane == 0) s_max[it & 1][tx >> 5] = m;
    if (!__syncthreads_and(ok)) break;          // the row is in registers
    const long long next = r + (long long)ring * gridDim.x;
    if (tx == 0 && next < p.rows) request(next, slot);
    m = __reduce_max_sync(0xffffffffu, s_max[it & 1][lane]);
    const int k = mx4_row_exponent(m);
    if (tx == 0) {
      p.row_scales[r] = two_to(k);
      if (m >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
    }
    uint8_t* codes = p.codes + r * p.ld_codes;
    uint8_t* scales = p.scales + mx4_scale_at(r, 0, p.chunks);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = tx + i * kStagedThreads;
      if (j >= pieces) break;
      const MxScale s = mx4_scale<GRID, T>(mine[i], k);
      uint32_t c[N / 8];
      v[i].template codes<GRID>(s, c);
      store_piece<T, GRID>(p, codes, scales, j, s, c);
    }
    if (++slot == ring) { slot = 0; phase ^= 1u; }
  }
  if (abort_flag && tx == 0) {
    for (int i = 0; i < 2000; ++i) __nanosleep(100);   // copies still in flight land before the CTA leaves
    flag(p.dev_status, OCS_DEV_TIMEOUT);
  }
  __syncthreads();
}

// E4M3, other rows that no CTA's registers hold: read twice, the second time from L2 (2377 x 33001 fp32: 117 us, floor 55;
// at most 84 bytes a thread are spilled in 16 bits).
template <typename T, int ALIGN>
__global__ void __launch_bounds__(kRowThreads, 3) mx4_long_rows_kernel(const T* __restrict__ X, const MxRows p) {
  constexpr int GRID = OCS_GRID_E4M3, N = Piece<T, GRID>::N;
  __shared__ uint32_t s_max[2][16];
  __shared__ __align__(16) unsigned char s_tail[kTailBytes];
  grid_launch_dependents();
  const int tx = threadIdx.x, lane = tx & 31;
  const int pieces = p.nb * Piece<T, GRID>::kLanes, t0 = p.C / N, tail = pieces - t0;
  const bool staged = tail * N * (int)sizeof(T) <= kTailBytes;
  T* my_tail = reinterpret_cast<T*>(s_tail);
  int odd = 0;
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x, odd ^= 1) {
    const T* x = X + r * p.ldx;
    if (staged) {
      __syncthreads();
      stage_tail<T, N>(p, x, t0 * N, tail, my_tail, tx, kRowThreads);
      __syncthreads();
    }
    auto load = [&](Block<T, N>& v, int j) {
      if (whole_piece<N, ALIGN>(p, r, j)) v.template load<ALIGN>(x + j * N);
      else if (staged && j >= t0) v.from_shared(my_tail + (j - t0) * N);
      else v.gather(x, j * N, p.C, p.K, p.idx_map, p.dev_status);
    };
    uint32_t m = 0;
#pragma unroll 4
    for (int j = tx; j < pieces; j += kRowThreads) {
      Block<T, N> v;
      load(v, j);
      m = max(m, v.max_bits());
    }
    m = __reduce_max_sync(0xffffffffu, m);
    if (lane == 0) s_max[odd][tx >> 5] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, s_max[odd][lane & 15]);
    const int k = mx4_row_exponent(m);
    if (tx == 0) {
      p.row_scales[r] = two_to(k);
      if (m >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
    }
    uint8_t* codes = p.codes + r * p.ld_codes;
    uint8_t* scales = p.scales + mx4_scale_at(r, 0, p.chunks);
#pragma unroll 2
    for (int j0 = 0; j0 < pieces; j0 += kRowThreads) {   // (whole warps stay: they share blocks)
      const int j = j0 + tx;
      Block<T, N> v;
      v.clear();
      if (j < pieces) load(v, j);
      const MxScale s = mx4_scale<GRID, T>(block_max<T, GRID>(v.max_bits()), k);
      uint32_t c[N / 8];
      v.template codes<GRID>(s, c);
      if (j < pieces) store_piece<T, GRID>(p, codes, scales, j, s, c);
    }
  }
}

template <typename T, int GRID, int ALIGN>
ocs_status launch_rows(const T* X, const MxRows& p, cudaStream_t stream) {
  constexpr int N = Piece<T, GRID>::N;
  const int pieces = p.nb * Piece<T, GRID>::kLanes;
  if (GRID == OCS_GRID_E4M3 && pieces > kRowPieces * kRowThreads) {
    const size_t row_bytes = (size_t)p.C * sizeof(T);
    if (ALIGN && p.rows >= 2 * kNumSMs && pieces <= kRowPieces * kStagedThreads && row_bytes % 16 == 0 && 2 * row_bytes <= kStagedBytes) {
      const int ring = (int)(kStagedBytes / row_bytes < kStagedRing ? kStagedBytes / row_bytes : kStagedRing);
      if (cudaFuncSetAttribute(mx4_staged_rows_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kStagedBytes) != cudaSuccess)
        return OCS_ERR_CUDA;
      LaunchScope ls("mx4_staged_rows_kernel", stream);
      mx4_staged_rows_kernel<T><<<kNumSMs, kStagedThreads, ring * row_bytes, stream>>>(X, p, ring);
      return launch_status();
    }
    const long long most = 3 * kNumSMs;
    LaunchScope ls("mx4_long_rows_kernel", stream);
    mx4_long_rows_kernel<T, ALIGN><<<(unsigned)(p.rows < most ? p.rows : most), kRowThreads, 0, stream>>>(X, p);
    return launch_status();
  }
  // few rows: a thread for every piece, as far as a CTA has them; many: two pieces each, or four (E8M0: one, twice the size)
  // fewer threads have more of a row's common work: 8192 x 8192 bf16 33.7 us with four pieces, 36 with two; rows that start
  // anywhere need the registers for loads: 4085 x 7279 29 and 26
  int nv = GRID == OCS_GRID_E4M3 && p.rows > kNumSMs && pieces > 32 ? (ALIGN == 32 && pieces > 128 ? 4 : 2) : 1;
  if (GRID == OCS_GRID_E4M3)
    while (pieces > nv * kRowThreads) nv *= 2;
  const int part = (pieces + nv - 1) / nv;
  int G = 4;
  while (G < part && G < 32) G *= 2;
  if (part > 32) G = part < kRowThreads ? (part + 31) / 32 * 32 : kRowThreads;
  const int y = GRID == OCS_GRID_E8M0 ? (part + G - 1) / G : 1;
  const int R = G <= 128 && p.rows * G > 32 * kNumSMs ? 256 / G : (G < 32 ? 32 / G : 1);
  const long long ctas = (p.rows + R - 1) / R;
  if (ctas > 0x7fffffff || y > 65535) return OCS_ERR_UNSUPPORTED;
  const dim3 grid((unsigned)ctas, (unsigned)y), block(G, R);
  const int room = kTailBytes / (R * N * (int)sizeof(T));
  LaunchScope ls("mx4_rows_kernel", stream);
  if (nv == 1) mx4_rows_kernel<T, GRID, ALIGN, 1><<<grid, block, 0, stream>>>(X, p, room);
  else if constexpr (GRID == OCS_GRID_E4M3) {
    if (nv == 2) mx4_rows_kernel<T, GRID, ALIGN, 2><<<grid, block, 0, stream>>>(X, p, room);
    else mx4_rows_kernel<T, GRID, ALIGN, 4><<<grid, block, 0, stream>>>(X, p, room);
  }
  return launch_status();
}
template <typename T, int ALIGN>
ocs_status launch_quantize(const T* X, const MxRows& p, ocs_grid grid, cudaStream_t stream) {
  return grid == OCS_GRID_E8M0 ? launch_rows<T, OCS_GRID_E8M0, ALIGN>(X, p, stream) : launch_rows<T, OCS_GRID_E4M3, ALIGN>(X, p, stream);
}

template <typename T>
ocs_status launch_quantize(const void* X_, const MxRows& p, ocs_grid grid, cudaStream_t stream) {
  const T* X = static_cast<const T*>(X_);
  const uintptr_t a = reinterpret_cast<uintptr_t>(X) | (p.rows > 1 ? (uintptr_t)(p.ldx * (int64_t)sizeof(T)) : 0);
  if (a % 32 == 0) return launch_quantize<T, 32>(X, p, grid, stream);
  if (a % 16 == 0) return launch_quantize<T, 16>(X, p, grid, stream);
  return launch_quantize<T, 0>(X, p, grid, stream);
}

// ---- codes to values: a thread stores NS times 32 aligned bytes of a row; blockDim.x threads and gridDim.y CTAs per row,
// blockDim.y rows per CTA.  SHIFTED: rows start anywhere, so a thread's elements are `ahead` behind a multiple of their number:
// their codes are shifted out of the words around them, and each 32 bytes of them may have two scales.  HBM bounds it: 4096 x
// 25088 to fp32 73 us (6.4 TB/s), 8192 x 8192 to bf16 28 us (6.1); 4085 x
// 7279, whose rows start anywhere, 19 (7296: 13).
template <typename T, int GRID, bool SHIFTED, int NS>
__global__ void __launch_bounds__(256) mx4_values_kernel(const MxRows p, T* __restrict__ Y, long long ldy) {
  constexpr int E = 32 / (int)sizeof(T), SHIFT = GRID == OCS_GRID_E8M0 ? 5 : 4, NW = NS * E / 8;
  const long long r = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  if (r >= p.rows) return;
  T* y = Y + r * ldy;
  const int ahead = SHIFTED ? (int)((reinterpret_cast<uintptr_t>(y) & 31) / sizeof(T)) : 0;
  const int c0 = (int)(blockIdx.y * blockDim.x + threadIdx.x) * (E * NS) - ahead;    // (negative: from the first element on)
  if (c0 >= p.K) return;
  const uint8_t* src = p.codes + r * p.ld_codes;
  const uint8_t* scales = p.scales + mx4_scale_at(r, 0, p.chunks);
  const float row = GRID == OCS_GRID_E4M3 ? __ldg(p.row_scales + r) : 1.0f;
  y += c0;
  uint32_t w[NW + 1];
  const int w0 = c0 >> 3, bytes = (p.K + 1) / 2;
  const bool inside = c0 >= 0 && c0 + NS * E <= p.K;
  if (!SHIFTED && inside && p.code_align >= 4 * NW) {
    if constexpr (NW == 4) { const uint4 v = __ldg(reinterpret_cast<const uint4*>(src + 4 * w0)); w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w; }
    else if constexpr (NW == 2) { const uint2 v = __ldg(reinterpret_cast<const uint2*>(src + 4 * w0)); w[0] = v.x; w[1] = v.y; }
    else w[0] = __ldg(reinterpret_cast<const uint32_t*>(src + 4 * w0));
  } else {
#pragma unroll
    for (int i = 0; i < NW + (SHIFTED ? 1 : 0); ++i) {
      const int at = 4 * (w0 + i);
      w[i] = 0;
      if (at < 0) continue;
      if (p.code_align >= 4 && at + 4 <= bytes) w[i] = __ldg(reinterpret_cast<const uint32_t*>(src + at));
      else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (at + j < bytes) w[i] |= (uint32_t)__ldg(src + at + j) << (8 * j);
      }
    }
    if (SHIFTED) {
#pragma unroll
      for (int i = 0; i < NW; ++i) w[i] = __funnelshift_r(w[i], w[i + 1], (c0 & 7) * 4);
    }
  }
  auto unit_of = [&](int b) {
    const uint32_t byte = __ldg(scales + (b >> 2) * kMxTile + (b & 3));
    return GRID == OCS_GRID_E8M0 ? e8m0_value(byte) : __fmul_rn(e4m3_value(byte), row);
  };
#pragma unroll
  for (int n = 0; n < NS; ++n) {
    const int c = c0 + n * E;
    if (n && c >= p.K) break;
    const int first = max(c, 0) >> SHIFT;
    const float u0 = unit_of(first), u1 = SHIFTED ? unit_of((min(c + E, p.K) - 1) >> SHIFT) : u0;
    const int split = SHIFTED ? ((first + 1) << SHIFT) - c : E;            // elements from here on have the second scale
    const unsigned long long u00 = pack_f32x2(u0, u0);
    T out[E];
#pragma unroll
    for (int i = 0; i < E / 8; ++i) {
      __half2 h[4];
      e2m1_values(w[n * (E / 8) + i], h);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float2 f = __half22float2(h[e]);
        const int at = 8 * i + 2 * e;
        float v0, v1;
        if (SHIFTED) { v0 = __fmul_rn(f.x, at < split ? u0 : u1); v1 = __fmul_rn(f.y, at + 1 < split ? u0 : u1); }
        else unpack_f32x2(mul_f32x2(pack_f32x2(f.x, f.y), u00), v0, v1);
        out[at] = from_f32<T>(v0);
        out[at + 1] = from_f32<T>(v1);
      }
    }
    if (inside || (c >= 0 && c + E <= p.K)) store32(reinterpret_cast<uint32_t*>(y + n * E), reinterpret_cast<const uint32_t*>(out));
    else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (c + i >= 0 && c + i < p.K) y[n * E + i] = out[i];
    }
  }
}

template <typename T, int GRID, bool SHIFTED>
ocs_status launch_values(const MxRows& p, T* Y, long long ldy, cudaStream_t stream) {
  constexpr int NS = 2, E = 32 / (int)sizeof(T) * NS;
  const int per = (p.K + (SHIFTED ? E - 1 : 0) + E - 1) / E;   // threads that a row may need
  int G = 4;
  while (G < per && G < 32) G *= 2;
  if (per > 32) G = per < 256 ? (per + 31) / 32 * 32 : 256;
  const int R = 256 / G;
  const long long ctas = (p.rows + R - 1) / R, y = (per + G - 1) / G;
  if (ctas > 0x7fffffff || y > 65535) return OCS_ERR_UNSUPPORTED;
  LaunchScope ls("mx4_values_kernel", stream);
  mx4_values_kernel<T, GRID, SHIFTED, NS><<<dim3((unsigned)ctas, (unsigned)y), dim3(G, R), 0, stream>>>(p, Y, ldy);
  return launch_status();
}
template <typename T>
ocs_status launch_values(const MxRows& p, ocs_grid grid, void* Y_, long long ldy, cudaStream_t stream) {
  T* Y = static_cast<T*>(Y_);
  const uintptr_t a = reinterpret_cast<uintptr_t>(Y) | (p.rows > 1 ? (uintptr_t)(ldy * (int64_t)sizeof(T)) : 0);
  if (grid == OCS_GRID_E8M0)
    return a % 32 ? launch_values<T, OCS_GRID_E8M0, true>(p, Y, ldy, stream) : launch_values<T, OCS_GRID_E8M0, false>(p, Y, ldy, stream);
  return a % 32 ? launch_values<T, OCS_GRID_E4M3, true>(p, Y, ldy, stream) : launch_values<T, OCS_GRID_E4M3, false>(p, Y, ldy, stream);
}

int align_of(const void* base, int64_t rows, int64_t ld) {
  const uintptr_t a = reinterpret_cast<uintptr_t>(base) | (rows > 1 ? (uintptr_t)ld : 0);
  return a % 16 == 0 ? 16 : (a % 8 == 0 ? 8 : (a % 4 == 0 ? 4 : 1));
}

}  // namespace
}  // namespace ocs

using namespace ocs;

extern "C" int64_t ocs_mx4_scale_bytes(int64_t rows, int K, ocs_grid grid) {
  if (rows < 0 || K <= 0 || !mx4_grid(grid)) return 0;
  const int64_t nb = ((int64_t)K + mx4_block(grid) - 1) / mx4_block(grid);
  return (rows + 127) / 128 * ((nb + 3) / 4) * kMxTile;
}

extern "C" ocs_status ocs_quantize_mx4(const void* X, ocs_dtype x_type, int64_t rows, int C, int64_t ldx, int S,
                                       const int32_t* idx_map, ocs_grid grid, uint8_t* codes, int64_t ld_codes,
                                       uint8_t* scales, float* row_scales, int* dev_status, void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!valid_dtype(x_type) || !mx4_grid(grid) || S < 0) return OCS_ERR_INVALID_ARG;
  if (rows < 0 || C <= 0) return OCS_ERR_SHAPE;
  if (rows == 0) return OCS_OK;
  if (!X || !codes || !scales || (grid == OCS_GRID_E4M3 && !row_scales) || (S > 0 && !idx_map)) return OCS_ERR_INVALID_ARG;
  if ((int64_t)C + S >= kMxMaxK) return OCS_ERR_UNSUPPORTED;
  const int K = C + S, n = mx4_block(grid), nb = (K + n - 1) / n;
  if (ldx < C || ld_codes < (K + 1) / 2) return OCS_ERR_SHAPE;
  if (!aligned(X, elem_bytes(x_type)) || !aligned(scales, 16) || !aligned(row_scales, 4) || (S > 0 && !aligned(idx_map, 4)))
    return OCS_ERR_SHAPE;
  const ocs_status st = check_device();
  if (st != OCS_OK) return st;
  const MxRows p{rows, ldx, ld_codes, C, K, nb, (nb + 3) / 4, idx_map, align_of(codes, rows, ld_codes), codes, scales,
                 row_scales, dev_status};
  switch (x_type) {
    case OCS_F16: return launch_quantize<__half>(X, p, grid, stream);
    case OCS_BF16: return launch_quantize<__nv_bfloat16>(X, p, grid, stream);
    default: return launch_quantize<float>(X, p, grid, stream);
  }
}

extern "C" ocs_status ocs_dequantize_mx4(const uint8_t* codes, int64_t ld_codes, const uint8_t* scales, const float* row_scales,
                                         int64_t rows, int K, ocs_grid grid, void* Y, ocs_dtype y_type, int64_t ldy,
                                         void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!valid_dtype(y_type) || !mx4_grid(grid)) return OCS_ERR_INVALID_ARG;
  if (rows < 0 || K <= 0) return OCS_ERR_SHAPE;
  if (rows == 0) return OCS_OK;
  if (!codes || !scales || !Y || (grid == OCS_GRID_E4M3 && !row_scales)) return OCS_ERR_INVALID_ARG;
  if (K >= kMxMaxK) return OCS_ERR_UNSUPPORTED;
  if (ld_codes < (K + 1) / 2 || ldy < K) return OCS_ERR_SHAPE;
  if (!aligned(Y, elem_bytes(y_type)) || !aligned(scales, 16) || !aligned(row_scales, 4)) return OCS_ERR_SHAPE;
  const ocs_status st = check_device();
  if (st != OCS_OK) return st;
  const int n = mx4_block(grid), nb = (K + n - 1) / n;
  const MxRows p{rows, 0, ld_codes, K, K, nb, (nb + 3) / 4, nullptr, align_of(codes, rows, ld_codes),
                 const_cast<uint8_t*>(codes), const_cast<uint8_t*>(scales), const_cast<float*>(row_scales), nullptr};
  switch (y_type) {
    case OCS_F16: return launch_values<__half>(p, grid, Y, ldy, stream);
    case OCS_BF16: return launch_values<__nv_bfloat16>(p, grid, Y, ldy, stream);
    default: return launch_values<float>(p, grid, Y, ldy, stream);
  }
}
