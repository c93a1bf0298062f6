// ocs_quantize_rows: linear quantization with one grid per row (a token's activations, or an output
// channel's split weights), the duplicated channels of a split layer appended to the codes.
//     alpha = max |x|,  scale = alpha / L,  code = rint(x * (L / alpha))
// The codes need the whole row's maximum first.  HBM bounds it as long as a row is read once, so the row waits on chip for its
// maximum: in one CTA's registers, in a cluster's, or (many long rows) in shared memory.
#include <type_traits>

#include "elem.cuh"
#include "ptx.cuh"

namespace ocs {
namespace {

struct RowsParams {
  long long rows, ldx, ld_codes;
  int C, S;
  const int32_t* idx_map;
  float hi;
  int is_signed;
  int code_vec;          // a thread's codes leave in one store (alignment of codes and ld_codes)
  int8_t* codes;
  float* scales;
  int* dev_status;
};

// VB bytes of a row (32 or 16, aligned) in registers
template <typename T, int VB>
struct Piece {
  static constexpr int VE = VB / (int)sizeof(T), W = VB / 4;
  uint32_t w[W];
  __device__ __forceinline__ void load(const T* x) {
    if constexpr (VB == 32) {
      asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                   : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(x));
    } else {
      const uint4 v = __ldg(reinterpret_cast<const uint4*>(x));
      w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    }
  }
  // elements [from, to), zeros around them
  __device__ __forceinline__ void load_part(const T* x, int from, int to) {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0;
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (e >= from && e < to) {
        if constexpr (sizeof(T) == 4) w[e] = __ldg(reinterpret_cast<const uint32_t*>(x) + e);
        else w[e / 2] |= (uint32_t)__ldg(reinterpret_cast<const uint16_t*>(x) + e) << (16 * (e & 1));
      }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0;
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    else return __half2float(__ushort_as_half((unsigned short)(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu)));
  }
  // Largest magnitude as bits (magnitudes order like their bit patterns, and so does what is not finite): of fp32, or of
  // both 16-bit halves side by side.
  __device__ __forceinline__ uint32_t max_bits(uint32_t m) const {
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if constexpr (sizeof(T) == 4) m = max(m, w[i] & 0x7fffffffu);
      else asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i] & 0x7fff7fffu));
    }
    return m;
  }
};
// ... as the bits of the fp32 value
template <typename T>
__device__ __forceinline__ uint32_t bits_f32(uint32_t m) {
  if constexpr (sizeof(T) == 4) return m;
  const uint32_t h = max(m & 0xffffu, m >> 16);
  if constexpr (std::is_same<T, __nv_bfloat16>::value) return h << 16;
  else return __float_as_uint(__half2float(__ushort_as_half((unsigned short)h)));
}

template <bool SIGNED, typename T, int VB>
__device__ __forceinline__ void codes_of(const Piece<T, VB>& p, const RowGrid& g, int* c) {
  constexpr int VE = Piece<T, VB>::VE;
  if (g.up == 1.0f) {
#pragma unroll
    for (int e = 0; e < VE; ++e) c[e] = row_code<SIGNED>(p[e], g.inv);
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) c[e] = row_code<SIGNED>(__fmul_rn(p[e], g.up), g.inv);
  }
}
// all codes of a piece, VE-byte aligned
template <int VE>
__device__ __forceinline__ void put_codes(void* dst, const int* c) {
  uint32_t w[VE / 4];
#pragma unroll
  for (int i = 0; i < VE / 4; ++i) w[i] = pack4(c[4 * i], c[4 * i + 1], c[4 * i + 2], c[4 * i + 3]);
  if constexpr (VE == 16) *reinterpret_cast<uint4*>(dst) = make_uint4(w[0], w[1], w[2], w[3]);
  else if constexpr (VE == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(w[0], w[1]);
  else *reinterpret_cast<uint32_t*>(dst) = w[0];
}

template <bool SIGNED, typename T, int VB>
__device__ __forceinline__ void store_codes(const Piece<T, VB>& p, const RowGrid& g, int8_t* dst, int n, bool vec) {
  constexpr int VE = Piece<T, VB>::VE;
  int c[VE];
  codes_of<SIGNED>(p, g, c);
  if (vec && n >= VE) {
    put_codes<VE>(dst, c);
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (e < n) dst[e] = (int8_t)c[e];
  }
}

constexpr int kRowThreads = 512;    // threads of a CTA with two pieces each (1024 with one)
constexpr int kRowCluster = 8;      // CTAs that may share a row
constexpr int kStagedRing = 4;      // rows of the staged form that are on chip or on their way
constexpr size_t kStagedBytes = 226 * 1024;

// One row per threadIdx.y and cluster, blockDim.x threads of each CTA on it, NV pieces of 32 bytes per thread: the row is
// read once and stays in registers between the maximum and the codes.  CLUSTER: the CTAs of a cluster take consecutive
// parts of the row and exchange their maxima through shared memory.  Three CTAs of 512 threads fit an SM, so that one
// row's loads cover another's maximum and stores: 8192 x 8192 bf16 (201 MB) takes 31.6 us, 6.4 TB/s.  With pieces of 16
// instead of 32 bytes and maxima of single elements instead of packed pairs it took 62 us: instructions bounded it.
template <typename T, int NV, bool CLUSTER, bool SHIFTED>
__global__ void __launch_bounds__(NV == 1 ? 1024 : kRowThreads, NV == 1 ? 1 : 3) rows_kernel(const T* __restrict__ X, const RowsParams p) {
  constexpr int VE = Piece<T, 32>::VE;
  __shared__ uint32_t s_max[32], s_part[kRowCluster];
  __shared__ __align__(16) unsigned char s_codes[SHIFTED ? 1024 * VE + 16 : 16];
  grid_launch_dependents();
  const int CL = CLUSTER ? (int)cluster_size() : 1, rank = CLUSTER ? (int)cluster_rank() : 0;
  if (CLUSTER) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");   // every CTA runs before its memory is written to
  const int G = blockDim.x, tx = threadIdx.x, lane = tx & 31;
  const long long r = CLUSTER ? blockIdx.x / CL : (long long)blockIdx.x * blockDim.y + threadIdx.y;
  if (!CLUSTER && r >= p.rows) return;   // (blocks of several rows have one warp on each)
  const T* x = X + r * p.ldx;
  const int ahead = SHIFTED ? (int)((reinterpret_cast<uintptr_t>(x) & 31) / sizeof(T)) : 0;
  const int n_vec = (p.C + ahead + VE - 1) / VE, per = (n_vec + CL - 1) / CL;
  const int lo = min(rank * per, n_vec), hi = min(lo + per, n_vec);
  Piece<T, 32> v[NV];
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int j = lo + tx + i * G, c = j * VE - ahead;
    if (j >= hi) v[i].clear();
    else if (c >= 0 && c + VE <= p.C) v[i].load(x + c);
    else v[i].load_part(x + c, -c, p.C - c);
  }
  // the first duplicated channels' values: fetched while the row is on its way
  const int s0 = rank * G + tx;
  float dup = 0.0f;
  if (s0 < p.S) {
    int c = __ldg(p.idx_map + p.C + s0);
    if ((unsigned)c >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); c = 0; }
    dup = to_f32(x[c]);
  }
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) m = v[i].max_bits(m);
  m = __reduce_max_sync(0xffffffffu, bits_f32<T>(m));
  if (G > 32) {
    if (lane == 0) s_max[tx >> 5] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, lane < (G >> 5) ? s_max[lane] : 0u);
  }
  if (CLUSTER) {
    asm volatile("barrier.cluster.wait;" ::: "memory");
    if (tx < CL) asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(peer_addr(smem_u32(s_part + rank), (uint32_t)tx)), "r"(m) : "memory");
    __syncwarp();
    cluster_arrive();
    cluster_wait();
    for (int i = 0; i < CL; ++i) m = max(m, s_part[i]);
  }
  const float alpha = __uint_as_float(m);
  const RowGrid g = row_grid(alpha, p.hi);
  if (tx == 0 && rank == 0) {
    p.scales[r] = __fdiv_rn(alpha, p.hi);
    if (m >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
  }
  int8_t* dst = p.codes + r * p.ld_codes;
  if constexpr (SHIFTED) {
    // through shared memory, from where they leave in aligned words
    unsigned char* buf = s_codes + threadIdx.y * (NV * 32 * VE);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = tx + i * G;
      int c[VE];
      if (p.is_signed) codes_of<true>(v[i], g, c);
      else codes_of<false>(v[i], g, c);
      if (lo + j < hi) put_codes<VE>(buf + j * VE, c);
    }
    if (G > 32) __syncthreads();
    else __syncwarp();
    const int at0 = lo * VE - ahead;                          // the element that buf starts with
    const int from = max(at0, 0), to = min(hi * VE - ahead, p.C);
    const int lead = min((int)(-reinterpret_cast<uintptr_t>(dst + from) & 3), max(to - from, 0));
    const int words = max(to - from - lead, 0) / 4, o = from + lead - at0, sh = (o & 3) * 8;
    const uint32_t* w = reinterpret_cast<const uint32_t*>(buf) + (o >> 2);
    uint32_t* out = reinterpret_cast<uint32_t*>(dst + from + lead);
    for (int i = tx; i < words; i += G) out[i] = __funnelshift_r(w[i], w[i + 1], sh);
    if (tx < lead) dst[from + tx] = (int8_t)buf[from + tx - at0];
    const int tail = from + lead + 4 * words + tx;
    if (tx < 4 && tail < to) dst[tail] = (int8_t)buf[tail - at0];
  } else {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = lo + tx + i * G, c = j * VE;
      if (j < hi) {
        if (p.is_signed) store_codes<true>(v[i], g, dst + c, p.C - c, p.code_vec);
        else store_codes<false>(v[i], g, dst + c, p.C - c, p.code_vec);
      }
    }
  }
  for (int s = s0; s < p.S; s += G * CL) {
    if (s != s0) {
      int c = __ldg(p.idx_map + p.C + s);
      if ((unsigned)c >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); c = 0; }
      dup = to_f32(x[c]);
    }
    const float f = g.up == 1.0f ? dup : __fmul_rn(dup, g.up);
    dst[p.C + s] = (int8_t)(p.is_signed ? row_code<true>(f, g.inv) : row_code<false>(f, g.inv));
  }
}

// Many long rows (whole 16-byte pieces): one CTA per SM, or two with half the threads, walk over them.  A row comes by
// one bulk copy into a ring of shared-memory buffers, moves into registers (which frees its buffer for the row after
// next), and is quantized from there while the next rows are on their way.  One barrier per row.  4096 x 25088 fp32 (514
// MB): 78.1 us, 6.6 TB/s, the measured copy rate; in clusters of four CTAs 124 us, since a cluster's three meetings per
// row leave its SMs without loads.
template <typename T, int NV, int THREADS>
__global__ void __launch_bounds__(THREADS, 1024 / THREADS) staged_rows_kernel(const T* __restrict__ X, const RowsParams p, int ring) {
  constexpr int VE = 16 / (int)sizeof(T);
  extern __shared__ __align__(128) unsigned char smem[];   // [ring] rows
  __shared__ __align__(8) uint64_t bars[kStagedRing];
  __shared__ uint32_t s_max[2][32];
  __shared__ int abort_flag;
  const int tx = threadIdx.x, lane = tx & 31, warp = tx >> 5;
  const uint32_t row_bytes = (uint32_t)p.C * (uint32_t)sizeof(T);
  const int n_vec = (int)(row_bytes / 16);
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
  int src = 0;
  if (tx < p.S) {
    src = __ldg(p.idx_map + p.C + tx);
    if ((unsigned)src >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); src = 0; }
  }
  __syncthreads();
  int it = 0, slot = 0;
  uint32_t phase = 0;
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x, ++it) {
    bool ok = mbar_wait(smem_u32(bars + slot), phase, &abort_flag);
    const unsigned char* buf = smem + (size_t)slot * row_bytes;
    Piece<T, 16> v[NV];
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = tx + i * THREADS;
      v[i].clear();
      if (j < n_vec) {
        const uint4 w = *reinterpret_cast<const uint4*>(buf + (size_t)j * 16);
        v[i].w[0] = w.x; v[i].w[1] = w.y; v[i].w[2] = w.z; v[i].w[3] = w.w;
      }
      m = v[i].max_bits(m);
    }
    float dup = tx < p.S ? to_f32(reinterpret_cast<const T*>(buf)[src]) : 0.0f;
    m = __reduce_max_sync(0xffffffffu, bits_f32<T>(m));
    if (lane == 0) s_max[it & 1][warp] = m;
    if (!__syncthreads_and(ok)) break;          // the row is in registers
    const long long next = r + (long long)ring * gridDim.x;
    if (tx == 0 && next < p.rows) request(next, slot);
    m = __reduce_max_sync(0xffffffffu, lane < THREADS / 32 ? s_max[it & 1][lane] : 0u);
    const float alpha = __uint_as_float(m);
    const RowGrid g = row_grid(alpha, p.hi);
    if (tx == 0) {
      p.scales[r] = __fdiv_rn(alpha, p.hi);
      if (m >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
    }
    int8_t* dst = p.codes + r * p.ld_codes;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int j = tx + i * THREADS;
      if (j < n_vec) {
        if (p.is_signed) store_codes<true>(v[i], g, dst + j * VE, VE, p.code_vec);
        else store_codes<false>(v[i], g, dst + j * VE, VE, p.code_vec);
      }
    }
    const T* x = X + r * p.ldx;
    for (int s = tx; s < p.S; s += THREADS) {
      if (s != tx) {
        int c = __ldg(p.idx_map + p.C + s);
        if ((unsigned)c >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); c = 0; }
        dup = to_f32(x[c]);
      }
      const float f = g.up == 1.0f ? dup : __fmul_rn(dup, g.up);
      dst[p.C + s] = (int8_t)(p.is_signed ? row_code<true>(f, g.inv) : row_code<false>(f, g.inv));
    }
    if (++slot == ring) { slot = 0; phase ^= 1u; }
  }
  if (abort_flag && tx == 0) {
    for (int i = 0; i < 2000; ++i) __nanosleep(100);   // copies still in flight land before the CTA leaves
    flag(p.dev_status, OCS_DEV_TIMEOUT);
  }
  __syncthreads();
}

// Rows too long for the registers of a cluster: read twice, the second time from L2.
template <typename T>
__global__ void __launch_bounds__(1024, 1) long_rows_kernel(const T* __restrict__ X, const RowsParams p) {
  using P = Piece<T, 32>;
  constexpr int VE = P::VE;
  __shared__ uint32_t s_max[32];
  grid_launch_dependents();
  const int tx = threadIdx.x, lane = tx & 31;
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T* x = X + r * p.ldx;
    const int past = (int)((reinterpret_cast<uintptr_t>(x) & 31) / sizeof(T));
    const int head = past ? min(VE - past, p.C) : 0;             // elements before the first aligned piece
    const int full = (p.C - head) / VE, body = head + full * VE;
    uint32_t m = 0;
#pragma unroll 4
    for (int i = tx; i < full; i += 1024) {
      P v;
      v.load(x + head + (long long)i * VE);
      m = v.max_bits(m);
    }
    m = bits_f32<T>(m);
    if (tx < head) m = max(m, __float_as_uint(to_f32(x[tx])) & 0x7fffffffu);
    if (tx < p.C - body) m = max(m, __float_as_uint(to_f32(x[body + tx])) & 0x7fffffffu);
    m = __reduce_max_sync(0xffffffffu, m);
    if (lane == 0) s_max[tx >> 5] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, s_max[lane]);
    const float alpha = __uint_as_float(m);
    const RowGrid g = row_grid(alpha, p.hi);
    if (tx == 0) {
      p.scales[r] = __fdiv_rn(alpha, p.hi);
      if (m >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
    }
    int8_t* dst = p.codes + r * p.ld_codes;
    // codes: in pieces where their stores are aligned too, else in aligned words (2 x 140009 bf16: 13.6 us, byte by byte 52)
    const bool vec = p.code_vec && head == 0;
    const int lead = vec ? 0 : min((int)(-reinterpret_cast<uintptr_t>(dst) & 3), p.C);
    const int units = vec ? full : (p.C - lead) / 4, done = units * (vec ? VE : 4);
#pragma unroll 4
    for (int i = tx; i < units; i += 1024) {
      if (vec) {
        P v;
        v.load(x + (long long)i * VE);
        if (p.is_signed) store_codes<true>(v, g, dst + (long long)i * VE, VE, true);
        else store_codes<false>(v, g, dst + (long long)i * VE, VE, true);
      } else {
        int c[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float f = __fmul_rn(to_f32(x[lead + 4 * i + e]), g.up);
          c[e] = p.is_signed ? row_code<true>(f, g.inv) : row_code<false>(f, g.inv);
        }
        put_codes<4>(dst + lead + 4 * i, c);
      }
    }
    for (int i = tx; i < p.C + p.S - done; i += 1024) {          // the ends of the row and the duplicated channels
      const int c = i < lead ? i : i + done;
      int src = c;
      if (c >= p.C) {
        src = __ldg(p.idx_map + c);
        if ((unsigned)src >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); src = 0; }
      }
      const float f = __fmul_rn(to_f32(x[src]), g.up);
      dst[c] = (int8_t)(p.is_signed ? row_code<true>(f, g.inv) : row_code<false>(f, g.inv));
    }
    __syncthreads();
  }
}

template <typename T, int NV, int THREADS>
ocs_status launch_staged(const T* X, const RowsParams& p, cudaStream_t stream) {
  const size_t row_bytes = (size_t)p.C * sizeof(T), budget = kStagedBytes * THREADS / 1024;
  const int ring = (int)(budget / row_bytes < kStagedRing ? budget / row_bytes : kStagedRing);
  if (cudaFuncSetAttribute(staged_rows_kernel<T, NV, THREADS>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)budget) != cudaSuccess)
    return OCS_ERR_CUDA;
  LaunchScope ls("staged_rows_kernel", stream);
  staged_rows_kernel<T, NV, THREADS><<<kNumSMs * 1024 / THREADS, THREADS, ring * row_bytes, stream>>>(X, p, ring);
  return launch_status();
}

template <typename T, bool SHIFTED>
ocs_status launch_rows(const T* X, RowsParams p, bool bulk, cudaStream_t stream) {
  constexpr int VE = Piece<T, 32>::VE;
  p.code_vec = aligned(p.codes, VE) && p.ld_codes % VE == 0;
  const int n_vec = (p.C + VE - 1 + (SHIFTED ? VE - 1 : 0)) / VE;   // at most
  // Many rows that are too long for one CTA's registers are staged: two CTAs of 512 threads per SM (whose rows overlap) as
  // long as their registers hold a row, else one of 1024.  Against the same rows in clusters, us: fp32 [4096][25088] 78.5
  // / 124.5; fp32 [4096][10000] 37.4 / 49.8 (47.3 with one CTA per SM); bf16 [2000][33280] 35.8 / 51.3; at 300 rows they
  // are even (13.1 / 12.3), and rows that fit one CTA's registers are as fast unstaged (bf16 [8192][8192] 31.7, staged 40;
  // bf16 [8192][8200] 47.3, staged 60.7).
  const size_t row_bytes = (size_t)p.C * sizeof(T);
  if (bulk && n_vec > 2 * kRowThreads && p.rows >= 2 * kNumSMs && row_bytes % 16 == 0 && 2 * row_bytes <= kStagedBytes) {
    if (row_bytes <= 6 * 512 * 16) return launch_staged<T, 6, 512>(X, p, stream);
    if (row_bytes <= 10 * 512 * 16) return launch_staged<T, 10, 512>(X, p, stream);
    return launch_staged<T, 8, 1024>(X, p, stream);
  }
  int cl = 1;   // CTAs on a row: as few as hold it in registers
  while (cl < kRowCluster && n_vec > 2 * kRowThreads * cl) cl *= 2;
  LaunchScope ls("rows_kernel", stream);
  if (n_vec > 2 * kRowThreads * cl || p.rows * cl >= 0x7fffffff) {
    const int grid = (int)(p.rows < 2 * kNumSMs ? p.rows : 2 * kNumSMs);
    long_rows_kernel<T><<<grid, 1024, 0, stream>>>(X, p);
    return launch_status();
  }
  // few rows: a thread for every piece; many: two pieces each, and rows of one warp share a CTA
  const int part = (n_vec + cl - 1) / cl;
  const bool one = cl == 1 && p.rows <= kNumSMs;
  const int G = ((one ? part : (part + 1) / 2) + 31) / 32 * 32, R = G == 32 ? 8 : 1;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((p.rows * cl + R - 1) / R), 1, 1);
  cfg.blockDim = dim3(G, R, 1);
  cfg.stream = stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cl; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr; cfg.numAttrs = cl > 1 ? 1 : 0;
  cudaError_t e;
  if (cl > 1) e = cudaLaunchKernelEx(&cfg, rows_kernel<T, 2, true, SHIFTED>, X, p);
  else if (one) e = cudaLaunchKernelEx(&cfg, rows_kernel<T, 1, false, SHIFTED>, X, p);
  else e = cudaLaunchKernelEx(&cfg, rows_kernel<T, 2, false, SHIFTED>, X, p);
  if (e != cudaSuccess) return OCS_ERR_CUDA;
  return launch_status();
}

template <typename T>
ocs_status launch_rows(const void* X_, const RowsParams& p, cudaStream_t stream) {
  const T* X = static_cast<const T*>(X_);
  // Rows that do not all start at a 32-byte boundary are read in aligned pieces all the same, and their codes shifted into
  // place.  Against pieces of the width that the rows' alignment allows, us: bf16 [4085][7279] 25.8 / 219, [13541][506] 10.4
  // / 14.8; fp32 [13152][1334] 21.0 / 34.5; 16-byte aligned fp32 [4000][4004] 16.9 / 20.3; a single row is even (2.1 / 2.0).
  // Against the bytes (13.6 us for [4085][7279]) the shift through shared memory costs: instructions are issued on 71 % of
  // the cycles, and a row's warps meet once more between its codes and their stores.
  const uintptr_t a = reinterpret_cast<uintptr_t>(X) | (p.rows > 1 ? (uintptr_t)(p.ldx * (int64_t)sizeof(T)) : 0);
  if (a % 32 == 0) return launch_rows<T, false>(X, p, true, stream);
  return launch_rows<T, true>(X, p, a % 16 == 0, stream);
}

}  // namespace
}  // namespace ocs

using namespace ocs;

extern "C" ocs_status ocs_quantize_rows(const void* X, ocs_dtype x_type, int64_t rows, int C, int64_t ldx, int S,
                                        const int32_t* idx_map, int bits, int is_signed, int8_t* codes,
                                        int64_t ld_codes, float* scales, int* dev_status, void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!valid_dtype(x_type) || bits < 2 || bits > 8 || S < 0) return OCS_ERR_INVALID_ARG;
  if (rows < 0 || C <= 0) return OCS_ERR_SHAPE;
  if (rows == 0) return OCS_OK;
  if (!X || !codes || !scales || (S > 0 && !idx_map)) return OCS_ERR_INVALID_ARG;
  if ((int64_t)C + S >= (1 << 30)) return OCS_ERR_UNSUPPORTED;
  if (ldx < C || ld_codes < (int64_t)C + S) return OCS_ERR_SHAPE;
  if (!aligned(X, elem_bytes(x_type)) || !aligned(scales, 4) || (S > 0 && !aligned(idx_map, 4))) return OCS_ERR_SHAPE;
  const ocs_status st = check_device();
  if (st != OCS_OK) return st;
  const float hi = (float)(is_signed ? (1 << (bits - 1)) - 1 : (1 << bits) - 1);
  const RowsParams p{rows, ldx, ld_codes, C, S, idx_map, hi, is_signed ? 1 : 0, 0, codes, scales, dev_status};
  switch (x_type) {
    case OCS_F16: return launch_rows<__half>(X, p, stream);
    case OCS_BF16: return launch_rows<__nv_bfloat16>(X, p, stream);
    default: return launch_rows<float>(X, p, stream);
  }
}
