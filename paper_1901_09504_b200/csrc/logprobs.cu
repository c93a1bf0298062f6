// ocs_token_logprobs and its gradient: log probabilities of given tokens, entropy and the likeliest tokens.
#include "elem.cuh"

namespace ocs {
namespace {

constexpr int kMaxTop = 64;

// (value, index) as one whole number: larger logit first, of equal ones (-0 = 0) the lower index first
__device__ __forceinline__ unsigned long long top_key(float v, int idx) {
  return ((unsigned long long)ord_encode(v + 0.0f) << 32) | (uint32_t)(0x7fffffff - idx);
}

constexpr int kLpThreads = 256;

template <typename V, typename F>
__device__ __forceinline__ V block_reduce(V v, V* smem, F f) {
  for (int o = 16; o > 0; o >>= 1) v = f(v, __shfl_xor_sync(0xffffffffu, v, o));
  __syncthreads();
  if ((threadIdx.x & 31) == 0) smem[threadIdx.x >> 5] = v;
  __syncthreads();
  v = smem[0];
  for (int w = 1; w < kLpThreads / 32; ++w) v = f(v, smem[w]);
  return v;
}

struct LogprobParams {
  long long rows, ld;
  int V, top_k;
  const int32_t* targets;
  float beta;
  float *logprob, *entropy, *top_logprob, *stats;
  int32_t* top_ids;
  int* dev_status;
};

template <typename T>
__global__ void __launch_bounds__(kLpThreads) logprobs_kernel(const T* __restrict__ logits, const LogprobParams p) {
  __shared__ float s_f[kLpThreads / 32];
  __shared__ unsigned long long s_k[kLpThreads / 32];
  auto fmx = [](float a, float b) { return fmaxf(a, b); };
  auto add = [](float a, float b) { return a + b; };
  auto kmx = [](unsigned long long a, unsigned long long b) { return a > b ? a : b; };
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const T* x = logits + r * p.ld;
    float m = -INFINITY, bad = 0.0f;
    for (int v = threadIdx.x; v < p.V; v += kLpThreads) {
      const float l = to_f32(x[v]);
      if (!(l < INFINITY)) bad = 1.0f;
      m = fmaxf(m, l);
    }
    m = block_reduce(m, s_f, fmx);
    bad = block_reduce(bad, s_f, fmx);
    const bool empty = m == -INFINITY;
    float s = 0.0f, w = 0.0f;
    for (int v = threadIdx.x; v < p.V && !empty && bad == 0.0f; v += kLpThreads) {
      const float d = (to_f32(x[v]) - m) * p.beta;
      const float e = expf(d);
      s += e;
      if (e > 0.0f) w = fmaf(e, d, w);
    }
    s = block_reduce(s, s_f, add);
    w = block_reduce(w, s_f, add);
    const float nan = __int_as_float(0x7fffffff);
    const float ls = bad != 0.0f ? nan : (empty ? 0.0f : logf(s));
    const float H = bad != 0.0f ? nan : (empty ? 0.0f : ls - w / s);
    if (threadIdx.x == 0) {
      if (bad != 0.0f) { flag(p.dev_status, OCS_DEV_NONFINITE); m = nan; }
      if (p.entropy) p.entropy[r] = H;
      if (p.stats) {
        p.stats[4 * r] = m; p.stats[4 * r + 1] = ls; p.stats[4 * r + 2] = H; p.stats[4 * r + 3] = m * p.beta + ls;
      }
      if (p.logprob && p.targets) {
        const int y = p.targets[r];
        float lp = 0.0f;
        if (y >= p.V) flag(p.dev_status, OCS_DEV_BAD_INDEX);
        else if (y >= 0) lp = empty ? -INFINITY : (to_f32(x[y]) - m) * p.beta - ls;
        p.logprob[r] = bad != 0.0f ? nan : lp;
      }
    }
    unsigned long long last = ~0ull;
    for (int j = 0; j < p.top_k; ++j) {
      unsigned long long best = 0;
      for (int v = threadIdx.x; v < p.V; v += kLpThreads) {
        const unsigned long long k = top_key(to_f32(x[v]), v);
        if (k < last && k > best) best = k;
      }
      last = block_reduce(best, s_k, kmx);
      if (threadIdx.x == 0) {
        const int id = 0x7fffffff - (int)(uint32_t)last;
        if (p.top_ids) p.top_ids[r * p.top_k + j] = bad != 0.0f ? -1 : id;
        if (p.top_logprob)
          p.top_logprob[r * p.top_k + j] = bad != 0.0f ? nan : (empty ? -INFINITY : (to_f32(x[id]) - m) * p.beta - ls);
      }
    }
    __syncthreads();
  }
}

struct GradParams {
  long long rows, ld, ld_d;
  int V;
  const int32_t* targets;
  float beta;
  const float *stats, *g_logprob, *g_entropy;
  int* dev_status;
};

template <typename T>
__global__ void __launch_bounds__(256) logprobs_backward_kernel(const T* logits, T* d_logits, const GradParams p) {
  for (long long r = blockIdx.x; r < p.rows; r += gridDim.x) {
    const float m = p.stats[4 * r], ls = p.stats[4 * r + 1], H = p.stats[4 * r + 2];
    const bool empty = m == -INFINITY;
    const float gh = p.g_entropy ? p.g_entropy[r] : 0.0f;
    int y = p.targets ? p.targets[r] : -1;
    if (y >= p.V) { y = -1; if (threadIdx.x == 0) flag(p.dev_status, OCS_DEV_BAD_INDEX); }
    const float g = p.g_logprob && y >= 0 ? p.g_logprob[r] : 0.0f;
    for (int v = threadIdx.x; v < p.V; v += 256) {
      const float lp = (to_f32(logits[r * p.ld + v]) - m) * p.beta - ls;
      const float pr = empty ? 0.0f : expf(lp);
      float d = pr > 0.0f ? -pr * (g + gh * (lp + H)) : (pr == 0.0f ? 0.0f : pr);
      if (v == y && !empty) d += g;
      d_logits[r * p.ld_d + v] = from_f32<T>(d * p.beta);
    }
  }
}

template <typename T>
ocs_status launch_logprobs(const void* logits, const LogprobParams& p, cudaStream_t stream) {
  LaunchScope ls("logprobs_kernel", stream);
  logprobs_kernel<T><<<(int)(p.rows < 0x7fffffff ? p.rows : 0x7fffffff), kLpThreads, 0, stream>>>(static_cast<const T*>(logits), p);
  return launch_status();
}

template <typename T>
ocs_status launch_backward(const void* logits, void* d_logits, const GradParams& p, cudaStream_t stream) {
  LaunchScope ls("logprobs_backward_kernel", stream);
  logprobs_backward_kernel<T><<<(int)(p.rows < 0x7fffffff ? p.rows : 0x7fffffff), 256, 0, stream>>>(
      static_cast<const T*>(logits), static_cast<T*>(d_logits), p);
  return launch_status();
}

}  // namespace
}  // namespace ocs

using namespace ocs;

extern "C" ocs_status ocs_token_logprobs(const void* logits, ocs_dtype type, int64_t rows, int V, int64_t ld,
                                         const int32_t* targets, float inv_temperature, int top_k, float* logprob,
                                         float* entropy, int32_t* top_ids, float* top_logprob, float* stats,
                                         int* dev_status, void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!valid_dtype(type) || !(inv_temperature > 0.0f) || !is_finite_host(inv_temperature) || top_k < 0)
    return OCS_ERR_INVALID_ARG;
  if (rows < 0 || V <= 0) return OCS_ERR_SHAPE;
  if (rows == 0) return OCS_OK;
  if (!logits || (logprob && !targets)) return OCS_ERR_INVALID_ARG;
  if (ld < V || top_k > V) return OCS_ERR_SHAPE;
  if (top_k > kMaxTop || V >= (1 << 30)) return OCS_ERR_UNSUPPORTED;
  if (!aligned(logits, elem_bytes(type)) || !aligned(targets, 4) || !aligned(logprob, 4) || !aligned(entropy, 4) ||
      !aligned(top_ids, 4) || !aligned(top_logprob, 4) || !aligned(stats, 16))
    return OCS_ERR_SHAPE;
  const ocs_status st = check_device();
  if (st != OCS_OK) return st;
  if (!top_ids && !top_logprob) top_k = 0;
  LogprobParams p{rows, ld, V, top_k, targets, inv_temperature, logprob, entropy, top_logprob, stats, top_ids, dev_status};
  switch (type) {
    case OCS_F16: return launch_logprobs<__half>(logits, p, stream);
    case OCS_BF16: return launch_logprobs<__nv_bfloat16>(logits, p, stream);
    default: return launch_logprobs<float>(logits, p, stream);
  }
}

extern "C" ocs_status ocs_token_logprobs_backward(const void* logits, ocs_dtype type, int64_t rows, int V, int64_t ld,
                                                  const int32_t* targets, float inv_temperature, const float* stats,
                                                  const float* g_logprob, const float* g_entropy, void* d_logits,
                                                  int64_t ld_d, int* dev_status, void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!valid_dtype(type) || !(inv_temperature > 0.0f) || !is_finite_host(inv_temperature)) return OCS_ERR_INVALID_ARG;
  if (rows < 0 || V <= 0) return OCS_ERR_SHAPE;
  if (rows == 0) return OCS_OK;
  if (!logits || !stats || !d_logits || (g_logprob && !targets)) return OCS_ERR_INVALID_ARG;
  if (ld < V || ld_d < V || (d_logits == logits && ld_d != ld)) return OCS_ERR_SHAPE;
  if (V >= (1 << 30)) return OCS_ERR_UNSUPPORTED;
  if (!aligned(logits, elem_bytes(type)) || !aligned(d_logits, elem_bytes(type)) || !aligned(targets, 4) ||
      !aligned(stats, 16) || !aligned(g_logprob, 4) || !aligned(g_entropy, 4))
    return OCS_ERR_SHAPE;
  const ocs_status st = check_device();
  if (st != OCS_OK) return st;
  GradParams p{rows, ld, ld_d, V, targets, inv_temperature, stats, g_logprob, g_entropy, dev_status};
  switch (type) {
    case OCS_F16: return launch_backward<__half>(logits, d_logits, p, stream);
    case OCS_BF16: return launch_backward<__nv_bfloat16>(logits, d_logits, p, stream);
    default: return launch_backward<float>(logits, d_logits, p, stream);
  }
}
