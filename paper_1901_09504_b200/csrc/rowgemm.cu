// ocs_qlinear_rows / ocs_linear_rows: the int8 layer with a scale per token and per output channel.
#include "elem.cuh"

namespace ocs {
namespace {

constexpr int kTile = 64;       // tokens and channels of one CTA's tile
constexpr int kStep = 64;       // contraction bytes staged at a time

struct RowGemm {
  const uint8_t* A;
  const float* a_scales;
  const int8_t* W;
  const float* w_scales;
  const float* bias;
  int M, N, K, a_signed;
  long long lda, ldw, ldy;
  int* dev_status;
};

// 64 x 64 tile, 256 threads of 4 x 4 outputs, operands staged in shared memory, four products per instruction.
template <typename T>
__global__ void __launch_bounds__(256) row_gemm_kernel(const RowGemm p, T* __restrict__ Y) {
  __shared__ uint32_t sa[kTile][kStep / 4 + 1], sw[kTile][kStep / 4 + 1];
  const int m0 = blockIdx.y * kTile, n0 = blockIdx.x * kTile;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  int acc[4][4] = {};
  for (int k0 = 0; k0 < p.K; k0 += kStep) {
    for (int i = threadIdx.x; i < kTile * kStep; i += 256) {
      const int r = i / kStep, k = i - r * kStep;
      const bool in = k0 + k < p.K;
      reinterpret_cast<uint8_t*>(&sa[r][0])[k] = in && m0 + r < p.M ? p.A[(long long)(m0 + r) * p.lda + k0 + k] : 0;
      reinterpret_cast<int8_t*>(&sw[r][0])[k] = in && n0 + r < p.N ? p.W[(long long)(n0 + r) * p.ldw + k0 + k] : 0;
    }
    __syncthreads();
    for (int k = 0; k < kStep / 4; ++k)
      for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
          const int a = (int)sa[ty + 16 * i][k], w = (int)sw[tx + 16 * j][k];
          if (p.a_signed) acc[i][j] = __dp4a(a, w, acc[i][j]);
          else asm("dp4a.u32.s32 %0, %1, %2, %0;" : "+r"(acc[i][j]) : "r"(a), "r"(w));
        }
    __syncthreads();
  }
  for (int i = 0; i < 4; ++i) {
    const int m = m0 + ty + 16 * i;
    if (m >= p.M) continue;
    for (int j = 0; j < 4; ++j) {
      const int n = n0 + tx + 16 * j;
      if (n >= p.N) continue;
      const float sc = __fmul_rn(p.a_scales[m], p.w_scales[n]);
      Y[(long long)m * p.ldy + n] = from_f32<T>(fmaf(__int2float_rn(acc[i][j]), sc, p.bias ? p.bias[n] : 0.0f));
    }
  }
}

ocs_status check_product(int a_signed, int M, int K, int64_t lda, const void* A, const int8_t* W, int N, int64_t ldw,
                         const float* bias, const void* Y, ocs_dtype y_type, int64_t ldy, const float* w_scales) {
  if (!W || !w_scales || !Y) return OCS_ERR_INVALID_ARG;
  if (lda < K || lda % 16 != 0 || !aligned(A, 16)) return OCS_ERR_SHAPE;
  if (ldw < K || ldw % 16 != 0 || !aligned(W, 16)) return OCS_ERR_SHAPE;
  if (ldy < N || !aligned(Y, elem_bytes(y_type)) || !aligned(w_scales, 4) || (bias && !aligned(bias, 4))) return OCS_ERR_SHAPE;
  if ((int64_t)K * 128 * (a_signed ? 128 : 255) > 2147483647ll || M >= (1 << 30)) return OCS_ERR_UNSUPPORTED;
  return OCS_OK;
}

template <typename T>
ocs_status launch_product(const RowGemm& p, void* Y, cudaStream_t stream) {
  const long long gy = (p.M + kTile - 1) / kTile;
  if (gy > 65535) return OCS_ERR_UNSUPPORTED;
  LaunchScope ls("row_gemm_kernel", stream);
  row_gemm_kernel<T><<<dim3((p.N + kTile - 1) / kTile, (unsigned)gy), 256, 0, stream>>>(p, static_cast<T*>(Y));
  return launch_status();
}

ocs_status run_product(const RowGemm& p, void* Y, ocs_dtype y_type, cudaStream_t stream) {
  switch (y_type) {
    case OCS_F16: return launch_product<__half>(p, Y, stream);
    case OCS_BF16: return launch_product<__nv_bfloat16>(p, Y, stream);
    default: return launch_product<float>(p, Y, stream);
  }
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
  RowGemm p{static_cast<const uint8_t*>(A_codes), a_scales, W_codes, w_scales, bias, M, N, K, a_signed ? 1 : 0,
            lda, ldw, ldy, dev_status};
  return run_product(p, Y, y_type, stream);
}

extern "C" size_t ocs_linear_rows_workspace_bytes(int M, int C, int S) {
  if (M <= 0 || C <= 0 || S < 0) return 256;
  return align_up((size_t)M * align_up((size_t)C + S, 16), 256) + align_up((size_t)M * 4, 256);
}

extern "C" ocs_status ocs_linear_rows(const void* X, ocs_dtype x_type, int M, int C, int64_t ldx, int S,
                                      const int32_t* idx_map, int bits, int is_signed, const int8_t* W_codes,
                                      const float* w_scales, int N, int64_t ldw, const float* bias, void* Y,
                                      ocs_dtype y_type, int64_t ldy, void* ws, size_t ws_bytes, int* dev_status,
                                      void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!valid_dtype(x_type) || !valid_dtype(y_type) || S < 0) return OCS_ERR_INVALID_ARG;
  if (M < 0 || C <= 0 || N <= 0) return OCS_ERR_SHAPE;
  if (M == 0) return OCS_OK;
  if ((int64_t)C + S >= (1 << 30)) return OCS_ERR_UNSUPPORTED;
  const int K = C + S;
  const int64_t lda = (int64_t)align_up((size_t)K, 16);
  if (!ws || !aligned(ws, 256) || ws_bytes < ocs_linear_rows_workspace_bytes(M, C, S)) return OCS_ERR_WORKSPACE;
  ocs_status st = check_product(is_signed, M, K, lda, ws, W_codes, N, ldw, bias, Y, y_type, ldy, w_scales);
  if (st != OCS_OK) return st;
  int8_t* codes = static_cast<int8_t*>(ws);
  float* scales = reinterpret_cast<float*>(codes + align_up((size_t)M * lda, 256));
  st = ocs_quantize_rows(X, x_type, M, C, ldx, S, idx_map, bits, is_signed, codes, lda, scales, dev_status, stream_);
  if (st != OCS_OK) return st;
  RowGemm p{reinterpret_cast<const uint8_t*>(codes), scales, W_codes, w_scales, bias, M, N, K, is_signed ? 1 : 0,
            lda, ldw, ldy, dev_status};
  return run_product(p, Y, y_type, stream);
}
