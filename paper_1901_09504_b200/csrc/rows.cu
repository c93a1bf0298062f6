// ocs_quantize_rows: linear quantization with one grid per row (a token's activations, or an output
// channel's split weights), the duplicated channels of a split layer appended to the codes.
#include "elem.cuh"

namespace ocs {
namespace {

constexpr int kRowThreads = 256;

template <typename T>
__global__ void __launch_bounds__(kRowThreads)
rows_kernel(const T* __restrict__ X, long long rows, int C, long long ldx, int S, const int32_t* __restrict__ idx_map,
            float hi, float lo, int8_t* __restrict__ codes, long long ld_codes, float* __restrict__ scales,
            int* dev_status) {
  __shared__ float s_max[kRowThreads / 32];
  for (long long r = blockIdx.x; r < rows; r += gridDim.x) {
    const T* x = X + r * ldx;
    float m = 0.0f;
    bool bad = false;
    for (int c = threadIdx.x; c < C; c += kRowThreads) {
      const float v = to_f32(x[c]);
      bad |= !is_finite(v);
      m = fmaxf(m, fabsf(v));
    }
    for (int o = 16; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    if (bad) flag(dev_status, OCS_DEV_NONFINITE);
    if ((threadIdx.x & 31) == 0) s_max[threadIdx.x >> 5] = m;
    __syncthreads();
    m = s_max[0];
    for (int w = 1; w < kRowThreads / 32; ++w) m = fmaxf(m, s_max[w]);
    __syncthreads();
    // below 2^-100 the row is scaled by 2^64 (exactly), so that hi / m stays finite
    const float up = m < 0x1p-100f ? 0x1p64f : 1.0f;
    const float inv = m > 0.0f ? __fdiv_rn(hi, __fmul_rn(m, up)) : 0.0f;
    if (threadIdx.x == 0) scales[r] = __fdiv_rn(m, hi);
    int8_t* dst = codes + r * ld_codes;
    for (int c = threadIdx.x; c < C + S; c += kRowThreads) {
      int src = c;
      if (c >= C) {
        src = __ldg(idx_map + c);
        if ((unsigned)src >= (unsigned)C) { flag(dev_status, OCS_DEV_BAD_INDEX); src = 0; }
      }
      dst[c] = (int8_t)quant_code(__fmul_rn(to_f32(x[src]), up), inv, lo, hi);
    }
  }
}

template <typename T>
ocs_status launch_rows(const void* X, long long rows, int C, long long ldx, int S, const int32_t* idx_map, int bits,
                       int is_signed, int8_t* codes, long long ld_codes, float* scales, int* dev_status,
                       cudaStream_t stream) {
  const float hi = (float)(is_signed ? (1 << (bits - 1)) - 1 : (1 << bits) - 1), lo = is_signed ? -hi : 0.0f;
  const int grid = (int)(rows < 0x7fffffff ? rows : 0x7fffffff);
  LaunchScope ls("rows_kernel", stream);
  rows_kernel<T><<<grid, kRowThreads, 0, stream>>>(static_cast<const T*>(X), rows, C, ldx, S, idx_map, hi, lo, codes,
                                                   ld_codes, scales, dev_status);
  return launch_status();
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
  switch (x_type) {
    case OCS_F16:
      return launch_rows<__half>(X, rows, C, ldx, S, idx_map, bits, is_signed, codes, ld_codes, scales, dev_status, stream);
    case OCS_BF16:
      return launch_rows<__nv_bfloat16>(X, rows, C, ldx, S, idx_map, bits, is_signed, codes, ld_codes, scales, dev_status, stream);
    default:
      return launch_rows<float>(X, rows, C, ldx, S, idx_map, bits, is_signed, codes, ld_codes, scales, dev_status, stream);
  }
}
