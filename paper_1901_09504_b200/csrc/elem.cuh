// Element types of the row-wise calls: loads to fp32, stores rounded once.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "common.cuh"

namespace ocs {

__device__ __forceinline__ float to_f32(float v) { return v; }
__device__ __forceinline__ float to_f32(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_f32(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T> __device__ __forceinline__ T from_f32(float v);
template <> __device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_f32<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

inline int elem_bytes(ocs_dtype t) { return t == OCS_F32 ? 4 : 2; }
inline bool valid_dtype(ocs_dtype t) { return t == OCS_F32 || t == OCS_F16 || t == OCS_BF16; }

// ---- the grid of one row (ocs_quantize_rows)
// A grid's constants: codes = rint(x * inv), after a multiplication by 2^64 for rows below 2^-100 (exact; it keeps
// hi / alpha finite).
struct RowGrid {
  float inv, up;
};
__device__ __forceinline__ RowGrid row_grid(float alpha, float hi) {
  RowGrid g;
  g.up = alpha < 0x1p-100f ? 0x1p64f : 1.0f;
  g.inv = alpha > 0.0f ? __fdiv_rn(hi, __fmul_rn(alpha, g.up)) : 0.0f;
  return g;
}
// |x| <= alpha, so |x * inv| <= hi * (1 + 2^-23): the rounding itself keeps the upper bound, only the unsigned grid
// has to clamp (at 0).  The rounding is the magic-number addition of quant_code; the low byte is the code.
template <bool SIGNED>
__device__ __forceinline__ int row_code(float x, float inv) {
  const float t = __fmul_rn(x, inv);
  return __float_as_int(__fadd_rn(SIGNED ? t : fmaxf(t, 0.0f), 12582912.0f));
}

}  // namespace ocs
