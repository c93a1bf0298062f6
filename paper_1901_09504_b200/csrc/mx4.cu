// ocs_quantize_mx4 / ocs_dequantize_mx4: rows to block-scaled 4-bit codes, the duplicated channels of a split layer appended,
// and back.  A thread has one block of a row: its scale needs no one else.
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

template <int GRID>
__device__ __forceinline__ void store_block(const MxRows& p, long long r, int b, const MxScale& s, const uint32_t* c) {
  constexpr int N = mx4_block(GRID), BYTES = N / 2;
  uint8_t* at = p.scales + mx4_scale_at(r, b, p.chunks);
  *at = (uint8_t)s.byte;
  if (b == p.nb - 1)
    for (int i = b + 1; i & 3; ++i) at[i - b] = 0;     // the group's blocks past the row's end
  uint8_t* dst = p.codes + r * p.ld_codes + (long long)b * BYTES;
  const int left = (p.K + 1) / 2 - b * BYTES;          // bytes of the row from here on
  if (left >= BYTES && p.code_align >= BYTES) {
    if constexpr (BYTES == 16) *reinterpret_cast<uint4*>(dst) = make_uint4(c[0], c[1], c[2], c[3]);
    else *reinterpret_cast<uint2*>(dst) = make_uint2(c[0], c[1]);
  } else if (left >= BYTES && p.code_align >= 4) {
#pragma unroll
    for (int i = 0; i < BYTES / 4; ++i) reinterpret_cast<uint32_t*>(dst)[i] = c[i];
  } else {
#pragma unroll
    for (int i = 0; i < BYTES; ++i)
      if (i < left) dst[i] = (uint8_t)(c[i / 4] >> (8 * (i & 3)));
  }
}

// E8M0: blocks know nothing of their row; thread g has block g % nb of row g / nb.
template <typename T, int ALIGN>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 4 : 3) mx4_blocks_kernel(const T* __restrict__ X, const MxRows p) {
  grid_launch_dependents();
  const unsigned long long g = (unsigned long long)blockIdx.x * 256 + threadIdx.x;
  const long long r = g >> 32 ? (long long)(g / (unsigned)p.nb) : (long long)((unsigned)g / (unsigned)p.nb);
  if (r >= p.rows) return;
  const int b = (int)(g - (unsigned long long)r * p.nb);
  Block<T, 32> v;
  v.template load_block<ALIGN>(X + r * p.ldx, b, p.C, p.K, p.idx_map, p.dev_status);
  const uint32_t m = v.max_bits();
  if (m >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
  const MxScale s = mx4_scale<OCS_GRID_E8M0, T>(m, 0);
  uint32_t c[4];
  v.template codes<OCS_GRID_E8M0>(s, c);
  store_block<OCS_GRID_E8M0>(p, r, b, s, c);
}

constexpr int kRowThreads = 512;

// E4M3: a row's scale is that of its largest magnitude, so the row waits in registers: blockDim.x threads with NV blocks each,
// blockDim.y rows per CTA.
template <typename T, int ALIGN, int NV>
__global__ void __launch_bounds__(kRowThreads, NV == 1 || sizeof(T) == 4 ? 2 : 3) mx4_rows_kernel(const T* __restrict__ X, const MxRows p) {
  __shared__ uint32_t s_max[32];
  grid_launch_dependents();
  const int G = blockDim.x, tx = threadIdx.x, lane = tx & 31;
  const long long r = (long long)blockIdx.x * blockDim.y + threadIdx.y;
  const bool live = r < p.rows;
  const T* x = X + (live ? r : 0) * p.ldx;
  Block<T, 16> v[NV];
  uint32_t mine[NV], m = 0;
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int b = tx + i * G;
    if (b >= p.nb || !live) v[i].clear();
    else v[i].template load_block<ALIGN>(x, b, p.C, p.K, p.idx_map, p.dev_status);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    mine[i] = v[i].max_bits();
    m = max(m, mine[i]);
  }
  m = __reduce_max_sync(0xffffffffu, m);
  if (G > 32) {
    const int per = G >> 5, first = threadIdx.y * per;
    if (lane == 0) s_max[first + (tx >> 5)] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, lane < per ? s_max[first + lane] : 0u);
  }
  if (!live) return;
  const int k = mx4_row_exponent(m);
  if (tx == 0) {
    p.row_scales[r] = two_to(k);
    if (m >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
  }
#pragma unroll
  for (int i = 0; i < NV; ++i) {
    const int b = tx + i * G;
    if (b >= p.nb) break;
    const MxScale s = mx4_scale<OCS_GRID_E4M3, T>(mine[i], k);
    uint32_t c[2];
    v[i].template codes<OCS_GRID_E4M3>(s, c);
    store_block<OCS_GRID_E4M3>(p, r, b, s, c);
  }
}

// E4M3, rows that no CTA's registers hold: read twice, the second time from L2.
template <typename T, int ALIGN>
__global__ void __launch_bounds__(kRowThreads, 2) mx4_long_rows_kernel(const T* __restrict__ X, const MxRows p) {
  __shared__ uint32_t s_max[2][16];
  grid_launch_dependents();
  const int tx = threadIdx.x, lane = tx & 31;
  int odd = 0;
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x, odd ^= 1) {
    const T* x = X + r * p.ldx;
    uint32_t m = 0;
#pragma unroll 2
    for (int b = tx; b < p.nb; b += kRowThreads) {
      Block<T, 16> v;
      v.template load_block<ALIGN>(x, b, p.C, p.K, p.idx_map, p.dev_status);
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
#pragma unroll 2
    for (int b = tx; b < p.nb; b += kRowThreads) {
      Block<T, 16> v;
      v.template load_block<ALIGN>(x, b, p.C, p.K, p.idx_map, p.dev_status);
      const MxScale s = mx4_scale<OCS_GRID_E4M3, T>(v.max_bits(), k);
      uint32_t c[2];
      v.template codes<OCS_GRID_E4M3>(s, c);
      store_block<OCS_GRID_E4M3>(p, r, b, s, c);
    }
  }
}

template <typename T, int ALIGN>
ocs_status launch_quantize(const T* X, const MxRows& p, ocs_grid grid, cudaStream_t stream) {
  if (grid == OCS_GRID_E8M0) {
    const long long ctas = (p.rows * p.nb + 255) / 256;
    if (ctas > 0x7fffffff) return OCS_ERR_UNSUPPORTED;
    LaunchScope ls("mx4_blocks_kernel", stream);
    mx4_blocks_kernel<T, ALIGN><<<(unsigned)ctas, 256, 0, stream>>>(X, p);
    return launch_status();
  }
  LaunchScope ls("mx4_rows_kernel", stream);
  if (p.nb > 2 * kRowThreads) {
    const long long most = 2 * kNumSMs;
    mx4_long_rows_kernel<T, ALIGN><<<(unsigned)(p.rows < most ? p.rows : most), kRowThreads, 0, stream>>>(X, p);
    return launch_status();
  }
  // few rows: a thread for every block; many: two blocks each
  const int nv = p.nb > kRowThreads || (p.rows > kNumSMs && p.nb > 32) ? 2 : 1;
  const int G = ((p.nb + nv - 1) / nv + 31) / 32 * 32, R = G <= 128 && p.rows > kNumSMs ? 256 / G : 1;
  const long long ctas = (p.rows + R - 1) / R;
  if (ctas > 0x7fffffff) return OCS_ERR_UNSUPPORTED;
  if (nv == 1) mx4_rows_kernel<T, ALIGN, 1><<<(unsigned)ctas, dim3(G, R), 0, stream>>>(X, p);
  else mx4_rows_kernel<T, ALIGN, 2><<<(unsigned)ctas, dim3(G, R), 0, stream>>>(X, p);
  return launch_status();
}

template <typename T>
ocs_status launch_quantize(const void* X_, const MxRows& p, ocs_grid grid, cudaStream_t stream) {
  const T* X = static_cast<const T*>(X_);
  const uintptr_t a = reinterpret_cast<uintptr_t>(X) | (p.rows > 1 ? (uintptr_t)(p.ldx * (int64_t)sizeof(T)) : 0);
  if (a % 32 == 0) return launch_quantize<T, 32>(X, p, grid, stream);
  if (a % 16 == 0) return launch_quantize<T, 16>(X, p, grid, stream);
  return launch_quantize<T, 0>(X, p, grid, stream);
}

// ---- codes to values
// Rows that start at 16-byte boundaries: 16 values per thread, stored 32 (WIDE) or 16 bytes at a time.
template <typename T, bool WIDE>
__global__ void __launch_bounds__(256) mx4_values_kernel(const MxRows p, int grid, T* __restrict__ Y, long long ldy) {
  const int per = (p.K + 15) / 16;
  const unsigned long long g = (unsigned long long)blockIdx.x * 256 + threadIdx.x;
  const long long r = g >> 32 ? (long long)(g / (unsigned)per) : (long long)((unsigned)g / (unsigned)per);
  if (r >= p.rows) return;
  const int u = (int)(g - (unsigned long long)r * per), c0 = u * 16, left = p.K - c0;
  const uint8_t* src = p.codes + r * p.ld_codes + u * 8;
  uint32_t w[2] = {0, 0};
  if (left >= 15 && p.code_align >= 8) {
    const uint2 v = __ldg(reinterpret_cast<const uint2*>(src));
    w[0] = v.x; w[1] = v.y;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (2 * i < left) w[i / 4] |= (uint32_t)__ldg(src + i) << (8 * (i & 3));
  }
  float unit;
  if (grid == OCS_GRID_E8M0) unit = e8m0_value(__ldg(p.scales + mx4_scale_at(r, u / 2, p.chunks)));
  else unit = __fmul_rn(e4m3_value(__ldg(p.scales + mx4_scale_at(r, u, p.chunks))), __ldg(p.row_scales + r));
  T* y = Y + r * ldy + c0;
  T out[16];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    __half2 h[4];
    e2m1_values(w[i], h);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      const float2 f = __half22float2(h[e]);
      out[8 * i + 2 * e] = from_f32<T>(__fmul_rn(f.x, unit));
      out[8 * i + 2 * e + 1] = from_f32<T>(__fmul_rn(f.y, unit));
    }
  }
  const uint32_t* o = reinterpret_cast<const uint32_t*>(out);
  if (left >= 16) {
    if constexpr (WIDE) {
#pragma unroll
      for (int i = 0; i < 4 * (int)sizeof(T); i += 8) store32(reinterpret_cast<uint32_t*>(y) + i, o + i);
    } else {
#pragma unroll
      for (int i = 0; i < (int)sizeof(T); ++i) reinterpret_cast<uint4*>(y)[i] = make_uint4(o[4 * i], o[4 * i + 1], o[4 * i + 2], o[4 * i + 3]);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i)
      if (i < left) y[i] = out[i];
  }
}

// Rows that start anywhere: a warp takes 512 values, two per lane and step, so that its stores are dense whatever their
// alignment.
template <typename T>
__global__ void __launch_bounds__(256) mx4_values_any_kernel(const MxRows p, int grid, T* __restrict__ Y, long long ldy) {
  const int per = (p.K + 511) / 512, lane = threadIdx.x & 31;
  const unsigned long long g = (unsigned long long)blockIdx.x * 8 + (threadIdx.x >> 5);
  const long long r = g >> 32 ? (long long)(g / (unsigned)per) : (long long)((unsigned)g / (unsigned)per);
  if (r >= p.rows) return;
  const int c0 = (int)(g - (unsigned long long)r * per) * 512 + 2 * lane;
  const uint8_t* src = p.codes + r * p.ld_codes + c0 / 2;
  const float row = grid == OCS_GRID_E8M0 ? 1.0f : __ldg(p.row_scales + r);
  T* y = Y + r * ldy + c0;
  const bool pairs = reinterpret_cast<uintptr_t>(y) % (2 * sizeof(T)) == 0;
  uint32_t code[8], byte[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = c0 + 64 * i;
    code[i] = c < p.K ? __ldg(src + 32 * i) : 0u;
    byte[i] = c < p.K ? __ldg(p.scales + mx4_scale_at(r, grid == OCS_GRID_E8M0 ? c / 32 : c / 16, p.chunks)) : 0u;
  }
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int c = c0 + 64 * i;
    const float unit = grid == OCS_GRID_E8M0 ? e8m0_value(byte[i]) : __fmul_rn(e4m3_value(byte[i]), row);
    const float2 f = e2m1_pair(code[i]);
    struct alignas(2 * sizeof(T)) Two { T a, b; } v{from_f32<T>(__fmul_rn(f.x, unit)), from_f32<T>(__fmul_rn(f.y, unit))};
    if (pairs && c + 1 < p.K) *reinterpret_cast<Two*>(y + 64 * i) = v;
    else {
      if (c < p.K) y[64 * i] = v.a;
      if (c + 1 < p.K) y[64 * i + 1] = v.b;
    }
  }
}

template <typename T>
ocs_status launch_values(const MxRows& p, ocs_grid grid, void* Y_, long long ldy, cudaStream_t stream) {
  T* Y = static_cast<T*>(Y_);
  const uintptr_t a = reinterpret_cast<uintptr_t>(Y) | (p.rows > 1 ? (uintptr_t)(ldy * (int64_t)sizeof(T)) : 0);
  const bool any = a % 16 != 0;
  const long long ctas = any ? (p.rows * ((p.K + 511) / 512) + 7) / 8 : (p.rows * ((p.K + 15) / 16) + 255) / 256;
  if (ctas > 0x7fffffff) return OCS_ERR_UNSUPPORTED;
  LaunchScope ls("mx4_values_kernel", stream);
  if (any) mx4_values_any_kernel<T><<<(unsigned)ctas, 256, 0, stream>>>(p, grid, Y, ldy);
  else if (a % 32 == 0) mx4_values_kernel<T, true><<<(unsigned)ctas, 256, 0, stream>>>(p, grid, Y, ldy);
  else mx4_values_kernel<T, false><<<(unsigned)ctas, 256, 0, stream>>>(p, grid, Y, ldy);
  return launch_status();
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
  if ((int64_t)C + S >= (1 << 30)) return OCS_ERR_UNSUPPORTED;
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
  if (K >= (1 << 30)) return OCS_ERR_UNSUPPORTED;
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
