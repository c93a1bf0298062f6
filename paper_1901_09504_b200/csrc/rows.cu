// ocs_quantize_rows: linear quantization with one grid per row (a token's activations, or an output
// channel's split weights), the duplicated channels of a split layer appended to the codes.
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

template <int VB> struct Word;
template <> struct Word<16> { using type = uint4; };
template <> struct Word<8> { using type = uint2; };
template <> struct Word<4> { using type = uint32_t; };
template <> struct Word<2> { using type = uint16_t; };

// VB bytes of a row in registers
template <typename T, int VB>
union Piece {
  static constexpr int VE = VB / (int)sizeof(T);
  typename Word<VB>::type w;
  T e[VE];
  __device__ __forceinline__ Piece() {}
};

template <bool SIGNED, typename T, int VB>
__device__ __forceinline__ void store_codes(const Piece<T, VB>& p, const RowGrid& g, bool scaled, int8_t* dst, int n, bool vec) {
  constexpr int VE = Piece<T, VB>::VE;
  int c[VE];
  if (!scaled) {
#pragma unroll
    for (int e = 0; e < VE; ++e) c[e] = row_code<SIGNED>(to_f32(p.e[e]), g.inv);
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e) c[e] = row_code<SIGNED>(__fmul_rn(to_f32(p.e[e]), g.up), g.inv);
  }
  if (vec && n == VE) {
    if constexpr (VE == 8) *reinterpret_cast<uint2*>(dst) = make_uint2(pack4(c[0], c[1], c[2], c[3]), pack4(c[4], c[5], c[6], c[7]));
    else if constexpr (VE == 4) *reinterpret_cast<uint32_t*>(dst) = pack4(c[0], c[1], c[2], c[3]);
    else if constexpr (VE == 2) *reinterpret_cast<uint16_t*>(dst) = (uint16_t)__byte_perm(c[0], c[1], 0x0040);
    else dst[0] = (int8_t)c[0];
  } else {
#pragma unroll
    for (int e = 0; e < VE; ++e)
      if (e < n) dst[e] = (int8_t)c[e];
  }
}

// One row per threadIdx.y, blockDim.x threads on it, NV pieces of VB bytes per thread: the row is read once and stays
// in registers between the maximum and the codes.
template <typename T, int VB, int NV>
__global__ void __launch_bounds__(1024, 1) rows_kernel(const T* __restrict__ X, const RowsParams p) {
  constexpr int VE = Piece<T, VB>::VE;
  __shared__ uint32_t s_max[32];
  grid_launch_dependents();
  const int G = blockDim.x, tx = threadIdx.x, lane = tx & 31;
  for (long long r0 = (long long)blockIdx.x * blockDim.y; r0 < p.rows; r0 += (long long)gridDim.x * blockDim.y) {
    const long long r = r0 + threadIdx.y;
    if (G == 32 && r >= p.rows) break;   // blocks of several rows have one warp on each
    const T* x = X + r * p.ldx;
    Piece<T, VB> v[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (tx + i * G) * VE;
      if (c + VE <= p.C) {
        v[i].w = __ldg(reinterpret_cast<const typename Word<VB>::type*>(x + c));
      } else {
#pragma unroll
        for (int e = 0; e < VE; ++e) v[i].e[e] = c + e < p.C ? x[c + e] : from_f32<T>(0.0f);
      }
    }
    // the first duplicated channels' values: fetched while the row is on its way
    float dup = 0.0f;
    if (tx < p.S) {
      int c = __ldg(p.idx_map + p.C + tx);
      if ((unsigned)c >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); c = 0; }
      dup = to_f32(x[c]);
    }
    // magnitudes order like their bit patterns, and so does what is not finite
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < NV; ++i)
#pragma unroll
      for (int e = 0; e < VE; ++e) m = max(m, __float_as_uint(to_f32(v[i].e[e])) & 0x7fffffffu);
    m = __reduce_max_sync(0xffffffffu, m);
    if (G > 32) {
      if (lane == 0) s_max[tx >> 5] = m;
      __syncthreads();
      m = __reduce_max_sync(0xffffffffu, lane < (G >> 5) ? s_max[lane] : 0u);
    }
    const float alpha = __uint_as_float(m);
    const RowGrid g = row_grid(alpha, p.hi);
    const bool scaled = g.up != 1.0f;
    if (tx == 0) {
      p.scales[r] = __fdiv_rn(alpha, p.hi);
      if (m >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
    }
    int8_t* dst = p.codes + r * p.ld_codes;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int c = (tx + i * G) * VE;
      if (c < p.C) {
        if (p.is_signed) store_codes<true>(v[i], g, scaled, dst + c, min(VE, p.C - c), p.code_vec);
        else store_codes<false>(v[i], g, scaled, dst + c, min(VE, p.C - c), p.code_vec);
      }
    }
    for (int s = tx; s < p.S; s += G) {
      if (s != tx) {
        int c = __ldg(p.idx_map + p.C + s);
        if ((unsigned)c >= (unsigned)p.C) { flag(p.dev_status, OCS_DEV_BAD_INDEX); c = 0; }
        dup = to_f32(x[c]);
      }
      dup = __fmul_rn(dup, g.up);
      dst[p.C + s] = (int8_t)(p.is_signed ? row_code<true>(dup, g.inv) : row_code<false>(dup, g.inv));
    }
    if (G > 32) __syncthreads();   // s_max is written again for the next row
  }
}

// Rows too long for the registers of a CTA: read twice, the second time from L2.
template <typename T, int VB>
__global__ void __launch_bounds__(1024, 1) long_rows_kernel(const T* __restrict__ X, const RowsParams p) {
  constexpr int VE = Piece<T, VB>::VE;
  __shared__ uint32_t s_max[32];
  grid_launch_dependents();
  const int tx = threadIdx.x, lane = tx & 31;
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T* x = X + r * p.ldx;
    uint32_t m = 0;
    const int full = p.C / VE;
#pragma unroll 4
    for (int i = tx; i < full; i += 1024) {
      Piece<T, VB> v;
      v.w = __ldg(reinterpret_cast<const typename Word<VB>::type*>(x + (long long)i * VE));
#pragma unroll
      for (int e = 0; e < VE; ++e) m = max(m, __float_as_uint(to_f32(v.e[e])) & 0x7fffffffu);
    }
    for (int c = full * VE + tx; c < p.C; c += 1024) m = max(m, __float_as_uint(to_f32(x[c])) & 0x7fffffffu);
    m = __reduce_max_sync(0xffffffffu, m);
    if (lane == 0) s_max[tx >> 5] = m;
    __syncthreads();
    m = __reduce_max_sync(0xffffffffu, s_max[lane]);
    const float alpha = __uint_as_float(m);
    const RowGrid g = row_grid(alpha, p.hi);
    const bool scaled = g.up != 1.0f;
    if (tx == 0) {
      p.scales[r] = __fdiv_rn(alpha, p.hi);
      if (m >= 0x7f800000u) flag(p.dev_status, OCS_DEV_NONFINITE);
    }
    int8_t* dst = p.codes + r * p.ld_codes;
#pragma unroll 4
    for (int i = tx; i < full; i += 1024) {
      Piece<T, VB> v;
      v.w = __ldg(reinterpret_cast<const typename Word<VB>::type*>(x + (long long)i * VE));
      if (p.is_signed) store_codes<true>(v, g, scaled, dst + (long long)i * VE, VE, p.code_vec);
      else store_codes<false>(v, g, scaled, dst + (long long)i * VE, VE, p.code_vec);
    }
    for (int c = full * VE + tx; c < p.C + p.S; c += 1024) {
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

template <typename T, int VB>
ocs_status launch_rows_vec(const T* X, RowsParams p, cudaStream_t stream) {
  constexpr int VE = Piece<T, VB>::VE;
  p.code_vec = aligned(p.codes, VE) && p.ld_codes % VE == 0;
  const int n_vec = (p.C + VE - 1) / VE;
  LaunchScope ls("rows_kernel", stream);
  if (n_vec > 8 * 1024) {
    const int grid = (int)(p.rows < 2 * kNumSMs ? p.rows : 2 * kNumSMs);
    long_rows_kernel<T, VB><<<grid, 1024, 0, stream>>>(X, p);
    return launch_status();
  }
  // Threads on a row: about four pieces each, at least a warp, at most 1024; rows of one warp share a CTA.
  int G = 32, nv = 1;
  while (G < 1024 && n_vec > 4 * G) G *= 2;
  while (nv * G < n_vec) nv *= 2;
  const int R = G == 32 ? 8 : 1;
  const long long want = (p.rows + R - 1) / R;
  const dim3 block(G, R);
  const unsigned grid = (unsigned)(want < 0x7fffffff ? want : 0x7fffffff);
  switch (nv) {
    case 1: rows_kernel<T, VB, 1><<<grid, block, 0, stream>>>(X, p); break;
    case 2: rows_kernel<T, VB, 2><<<grid, block, 0, stream>>>(X, p); break;
    case 4: rows_kernel<T, VB, 4><<<grid, block, 0, stream>>>(X, p); break;
    default: rows_kernel<T, VB, 8><<<grid, block, 0, stream>>>(X, p); break;
  }
  return launch_status();
}

template <typename T>
ocs_status launch_rows(const void* X_, const RowsParams& p, cudaStream_t stream) {
  const T* X = static_cast<const T*>(X_);
  // the widest accesses that the rows' alignment allows
  const uintptr_t a = reinterpret_cast<uintptr_t>(X) | (p.rows > 1 ? (uintptr_t)(p.ldx * (int64_t)sizeof(T)) : 0);
  if (a % 16 == 0) return launch_rows_vec<T, 16>(X, p, stream);
  if (a % 8 == 0) return launch_rows_vec<T, 8>(X, p, stream);
  if (sizeof(T) == 4 || a % 4 == 0) return launch_rows_vec<T, 4>(X, p, stream);
  return launch_rows_vec<T, (int)sizeof(T)>(X, p, stream);
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
