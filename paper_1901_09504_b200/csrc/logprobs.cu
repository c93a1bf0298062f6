// ocs_token_logprobs and its gradient: log probabilities of given tokens, entropy and the likeliest tokens.
#include "elem.cuh"
#include "ptx.cuh"

namespace ocs {
namespace {

constexpr int kMaxTop = 64;
constexpr int kLpThreads = 256;
constexpr int kWarps = kLpThreads / 32;
constexpr int kMaxCluster = 8;        // CTAs that may share a row
constexpr int kCandidates = 2048;     // elements that can still be among the largest
constexpr float kFloor = -200.0f;     // 2^-200 is zero in fp32: exponents are clamped here, so that a masked token (d = -infinity)
                                      // contributes 0 to the sums and not 0 * infinity

typedef unsigned long long key_t;

// (logit, index) as one whole number: larger logit first, of equal ones (-0 = 0) the lower index first
__device__ __forceinline__ key_t top_key(float v, int idx) {
  return ((key_t)ord_encode(v + 0.0f) << 32) | (uint32_t)(0x7fffffff - idx);
}
__device__ __forceinline__ int key_index(key_t k) { return 0x7fffffff - (int)(uint32_t)k; }
__device__ __forceinline__ float key_value(key_t k) { return ord_decode((uint32_t)(k >> 32)); }

__device__ __forceinline__ float max_nan(float a, float b) {   // NaN if either is
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float ex2(float x) {                // 2^x, relative error about 2^-22; below 2^-126 zero
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
__device__ __forceinline__ unsigned long long add_f32x2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ unsigned long long mul_f32x2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// 16 bytes of a row
template <typename T>
struct Vec {
  static constexpr int VE = 16 / (int)sizeof(T);
  uint4 w;
  __device__ __forceinline__ uint32_t word(int i) const { return i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w; }
  // elements 2i and 2i + 1 as a packed pair of fp32
  __device__ __forceinline__ unsigned long long pair(int i) const;
  __device__ __forceinline__ float max_all() const;   // NaN if any element is
};
template <> __device__ __forceinline__ unsigned long long Vec<float>::pair(int i) const {
  return pack_f32x2(__uint_as_float(word(2 * i)), __uint_as_float(word(2 * i + 1)));
}
template <> __device__ __forceinline__ unsigned long long Vec<__nv_bfloat16>::pair(int i) const {
  const uint32_t v = word(i);
  return pack_f32x2(__uint_as_float(v << 16), __uint_as_float(v & 0xffff0000u));
}
template <> __device__ __forceinline__ unsigned long long Vec<__half>::pair(int i) const {
  const uint32_t v = word(i);
  const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&v));
  return pack_f32x2(f.x, f.y);
}
template <> __device__ __forceinline__ float Vec<float>::max_all() const {
  return max_nan(max_nan(__uint_as_float(w.x), __uint_as_float(w.y)), max_nan(__uint_as_float(w.z), __uint_as_float(w.w)));
}
template <> __device__ __forceinline__ float Vec<__nv_bfloat16>::max_all() const {
  const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&w);
  const __nv_bfloat162 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  return max_nan(__low2float(m), __high2float(m));
}
template <> __device__ __forceinline__ float Vec<__half>::max_all() const {
  const __half2* h = reinterpret_cast<const __half2*>(&w);
  const __half2 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  return max_nan(__low2float(m), __high2float(m));
}

template <typename T> __device__ __forceinline__ T minus_infinity();
template <> __device__ __forceinline__ float minus_infinity<float>() { return -INFINITY; }
template <> __device__ __forceinline__ __half minus_infinity<__half>() { return __ushort_as_half(0xfc00); }
template <> __device__ __forceinline__ __nv_bfloat16 minus_infinity<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80); }

// A row as aligned vectors of 16 bytes: vector j holds elements j * VE - a .. j * VE - a + VE - 1, where a is how many
// elements past a 16-byte boundary the row starts.  The first and the last one may hang over; what lies outside the row is
// never read and counts as -infinity.
template <typename T>
struct RowVectors {
  static constexpr int VE = Vec<T>::VE;
  const T* x;
  int V, a, count;
  __device__ __forceinline__ RowVectors(const T* row, int n) : x(row), V(n) {
    a = (int)((reinterpret_cast<uintptr_t>(row) & 15) / sizeof(T));
    count = (V + a + VE - 1) / VE;
  }
  __device__ __forceinline__ int first(int j) const { return j * VE - a; }
  __device__ __forceinline__ bool whole(int j) const { return first(j) >= 0 && first(j) + VE <= V; }
  __device__ __forceinline__ Vec<T> load(int j) const {
    Vec<T> v;
    const int e0 = first(j);
    if (whole(j)) {
      v.w = *reinterpret_cast<const uint4*>(x + e0);
    } else {
      T* e = reinterpret_cast<T*>(&v.w);
#pragma unroll
      for (int i = 0; i < VE; ++i) e[i] = (unsigned)(e0 + i) < (unsigned)V ? x[e0 + i] : minus_infinity<T>();
    }
    return v;
  }
};

// Running softmax statistics in base 2: with c = inv_temperature * log2(e) and d = (l - m) * c,
//   s = sum 2^d,  w = sum 2^d * d;   ln sum exp z = m * inv_temperature + ln s,  entropy = ln s - ln 2 * w / s.
struct Stats {
  float m, s, w;
};
__device__ __forceinline__ void move_max(Stats& t, float m, float c) {   // the same sums relative to another maximum
  const float d = fmaxf(__fmul_rn(__fsub_rn(t.m, m), c), kFloor);        // -infinity or NaN (nothing summed yet): s = w = 0
  const float r = ex2(d);
  t.w = __fmul_rn(fmaf(t.s, d, t.w), r);
  t.s = __fmul_rn(t.s, r);
  t.m = m;
}
__device__ __forceinline__ Stats warp_stats(Stats t, float c) {
  float m = t.m;
  for (int o = 16; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, o));
  move_max(t, m, c);
  for (int o = 16; o > 0; o >>= 1) {
    t.s = __fadd_rn(t.s, __shfl_xor_sync(0xffffffffu, t.s, o));
    t.w = __fadd_rn(t.w, __shfl_xor_sync(0xffffffffu, t.w, o));
  }
  return t;
}

struct LogprobParams {
  long long rows, ld;
  int V, top_k;
  const int32_t* targets;
  float beta, c;
  float *logprob, *entropy, *top_logprob, *stats;
  int32_t* top_ids;
  int* dev_status;
};

struct LogprobSmem {
  Stats warp[kWarps];
  Stats part[kMaxCluster];                       // of the CTAs that share the row
  key_t sorted[kLpThreads];                      // every thread's largest element, descending within a warp
  key_t cand[kCandidates];
  key_t top[kMaxCluster * kMaxTop];              // each CTA's largest, then the row's
  key_t best[kMaxTop];
  key_t tau;
  int hot[kLpThreads];
  int n_hot, n_cand;
  key_t round[kWarps];
};

// The k largest of n keys in list, descending, to out (all threads; n may be less than k: zeros follow).
__device__ __forceinline__ void rank_select(const key_t* list, int n, int k, key_t* out) {
  for (int i = threadIdx.x; i < k; i += kLpThreads)
    if (i >= n) out[i] = 0;
  for (int i = threadIdx.x; i < n; i += kLpThreads) {
    const key_t mine = list[i];
    int r = 0;
    for (int j = 0; j < n && r < k; ++j) r += list[j] > mine;
    if (r < k && mine != 0) out[r] = mine;
  }
}

// The k largest elements of vectors [lo, hi) of the row, as keys in out, given every thread's largest element (its value,
// and the vector that holds it first).
//   1. tau = the k-th largest of the threads' keys, each lowered to the last index of its vector: k elements at least
//      are not below it.  Only threads with a key not below tau (raised to the first index) can hold such an element:
//      the vectors are disjoint, so these are k threads at most.
//   2. A warp reads the elements of one of these threads again and collects what is not below tau.
//   3. The k largest of what was collected, by rank.
// Many equal or unluckily placed elements may overflow the list; then the keys are found one after the other.
template <typename T>
__device__ void top_of_segment(const RowVectors<T>& row, int lo, int hi, int k, float m, int pos, LogprobSmem& sm, key_t* out) {
  constexpr int VE = Vec<T>::VE;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool any = lo + tid < hi;
  const int e0 = row.first(pos);
  const key_t low = any ? top_key(m, min(e0 + VE, row.V) - 1) : 0;
  const key_t high = any ? top_key(m, max(e0, 0)) : 0;
  if (tid == 0) { sm.tau = 0; sm.n_hot = 0; sm.n_cand = 0; }
  // descending within the warp (bitonic)
  key_t v = low;
#pragma unroll
  for (int size = 2; size <= 32; size *= 2) {
#pragma unroll
    for (int o = size / 2; o > 0; o /= 2) {
      const key_t other = __shfl_xor_sync(0xffffffffu, v, o);
      const bool keep_max = ((lane & o) == 0) == ((lane & size) == 0 || size == 32);
      v = keep_max ? (v > other ? v : other) : (v < other ? v : other);
    }
  }
  sm.sorted[tid] = v;
  __syncthreads();
  // rank of v among all threads' keys: its place in its own list, and how many of each other list are larger
  if (v != 0) {
    int rank = lane;
    for (int w = 0; w < kWarps; ++w) {
      if (w == warp) continue;
      int n = 0;
#pragma unroll
      for (int step = 32; step > 0; step /= 2)
        if (n + step <= 32 && sm.sorted[w * 32 + n + step - 1] > v) n += step;
      rank += n;
    }
    if (rank == k - 1) sm.tau = v;
  }
  __syncthreads();
  const key_t tau = sm.tau;
  if (any && high >= tau) sm.hot[atomicAdd(&sm.n_hot, 1)] = tid;
  __syncthreads();
  const int n_hot = sm.n_hot;
  for (int h = warp; h < n_hot; h += kWarps) {
    for (int j = lo + sm.hot[h] + lane * kLpThreads; j < hi; j += 32 * kLpThreads) {
      const Vec<T> x = row.load(j);
      const int first = row.first(j);
#pragma unroll
      for (int i = 0; i < VE / 2; ++i) {
        float f[2];
        unpack_f32x2(x.pair(i), f[0], f[1]);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int idx = first + 2 * i + e;
          if ((unsigned)idx < (unsigned)row.V) {
            const key_t key = top_key(f[e], idx);
            if (key >= tau) {
              const int at = atomicAdd(&sm.n_cand, 1);
              if (at < kCandidates) sm.cand[at] = key;
            }
          }
        }
      }
    }
  }
  __syncthreads();
  const int n = sm.n_cand;
  if (n <= kCandidates) {
    rank_select(sm.cand, n, k, out);
  } else {
    key_t last = ~0ull;
    for (int r = 0; r < k; ++r) {
      key_t best = 0;
      for (int j = lo + tid; j < hi; j += kLpThreads) {
        const Vec<T> x = row.load(j);
        for (int i = 0; i < VE / 2; ++i) {
          float f[2];
          unpack_f32x2(x.pair(i), f[0], f[1]);
          for (int e = 0; e < 2; ++e) {
            const int idx = row.first(j) + 2 * i + e;
            const key_t key = (unsigned)idx < (unsigned)row.V ? top_key(f[e], idx) : 0;
            if (key < last && key > best) best = key;
          }
        }
      }
      for (int o = 16; o > 0; o >>= 1) { const key_t other = __shfl_xor_sync(0xffffffffu, best, o); if (other > best) best = other; }
      if (lane == 0) sm.round[warp] = best;
      __syncthreads();
      for (int w = 0; w < kWarps; ++w) if (sm.round[w] > best) best = sm.round[w];
      if (tid == 0) out[r] = best;
      last = best;
      __syncthreads();
    }
  }
  __syncthreads();
}

__device__ __forceinline__ void store_peer_u64(uint32_t addr, key_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void store_peer_f32(uint32_t addr, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(addr), "f"(v) : "memory");
}

// One row per cluster; the CTAs of a cluster take consecutive parts of it and send what they found to the first one.
template <typename T>
__global__ void __launch_bounds__(kLpThreads, 4) logprobs_kernel(const T* __restrict__ logits, const LogprobParams p) {
  constexpr int VE = Vec<T>::VE, U = 4;
  __shared__ LogprobSmem sm;
  const int CL = (int)cluster_size(), rank = CL > 1 ? (int)cluster_rank() : 0;
  if (CL > 1) asm volatile("barrier.cluster.arrive.relaxed;" ::: "memory");   // every CTA runs before its memory is written to
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long r = blockIdx.x / CL;
  const RowVectors<T> row(logits + r * p.ld, p.V);
  const int per = (row.count + CL - 1) / CL;
  const int lo = min(rank * per, row.count), hi = min(lo + per, row.count);
  int y = -1;
  float ly = 0.0f;
  if (rank == 0 && tid == 0 && p.logprob) {
    y = p.targets[r];
    if (y >= p.V) { flag(p.dev_status, OCS_DEV_BAD_INDEX); y = -1; }
    if (y >= 0) ly = to_f32(row.x[y]);
  }

  Stats t{-INFINITY, 0.0f, 0.0f};
  int pos = lo + tid;
  const float c = p.c;
  const unsigned long long c2 = pack_f32x2(c, c);
  for (int j0 = lo + tid; j0 < hi; j0 += U * kLpThreads) {
    Vec<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * kLpThreads;
      if (j < hi) v[u] = row.load(j);
    }
    float mx[U], m = t.m;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      mx[u] = j0 + u * kLpThreads < hi ? v[u].max_all() : -INFINITY;
      m = max_nan(m, mx[u]);
    }
    if (m != t.m) {   // (also NaN)
#pragma unroll
      for (int u = U - 1; u >= 0; --u)
        if (mx[u] == m) pos = j0 + u * kLpThreads;
      move_max(t, m, c);
    }
    const unsigned long long neg = pack_f32x2(-m, -m);
    unsigned long long s2 = pack_f32x2(0.0f, 0.0f), w2 = s2;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (j0 + u * kLpThreads < hi) {
#pragma unroll
        for (int i = 0; i < VE / 2; ++i) {
          float d0, d1;
          unpack_f32x2(mul_f32x2(add_f32x2(v[u].pair(i), neg), c2), d0, d1);
          d0 = fmaxf(d0, kFloor);
          d1 = fmaxf(d1, kFloor);
          const unsigned long long e = pack_f32x2(ex2(d0), ex2(d1));
          s2 = add_f32x2(s2, e);
          w2 = fma_f32x2(e, pack_f32x2(d0, d1), w2);
        }
      }
    }
    float a, b;
    unpack_f32x2(s2, a, b);
    t.s = __fadd_rn(t.s, __fadd_rn(a, b));
    unpack_f32x2(w2, a, b);
    t.w = __fadd_rn(t.w, __fadd_rn(a, b));
  }

  const float own_max = t.m;
  t = warp_stats(t, c);
  if (lane == 0) sm.warp[warp] = t;
  if (p.top_k > 0) {
    top_of_segment(row, lo, hi, p.top_k, own_max, pos, sm, sm.top + rank * p.top_k);   // begins and ends with a barrier
  } else {
    __syncthreads();
  }
  // this CTA's part of the row (every warp works it out; lane w looks at warp w)
  t = lane < kWarps ? sm.warp[lane] : Stats{-INFINITY, 0.0f, 0.0f};
  t = warp_stats(t, c);
  if (CL > 1) {
    asm volatile("barrier.cluster.wait;" ::: "memory");
    if (rank != 0) {
      if (tid == 0) {
        const uint32_t dst = peer_addr(smem_u32(&sm.part[rank]), 0);
        store_peer_f32(dst, t.m);
        store_peer_f32(dst + 4, t.s);
        store_peer_f32(dst + 8, t.w);
      }
      for (int i = tid; i < p.top_k; i += kLpThreads)
        store_peer_u64(peer_addr(smem_u32(&sm.top[rank * p.top_k + i]), 0), sm.top[rank * p.top_k + i]);
      __syncwarp();
      asm volatile("barrier.cluster.arrive.release;" ::: "memory");
      return;   // the first CTA's memory outlives the stores: it waits for this arrival
    }
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    const Stats own = t;
    t = lane == 0 ? own : (lane < CL ? sm.part[lane] : Stats{-INFINITY, 0.0f, 0.0f});
    t = warp_stats(t, c);
    if (p.top_k > 0) {
      rank_select(sm.top, CL * p.top_k, p.top_k, sm.best);
      __syncthreads();
    }
  }
  const key_t* best = CL > 1 ? sm.best : sm.top;
  const bool bad = !(t.m < INFINITY), empty = t.m == -INFINITY;
  const float nan = __int_as_float(0x7fffffff);
  const float ls = bad ? nan : (empty ? 0.0f : logf(t.s));
  if (tid == 0) {
    const float H = bad ? nan : (empty ? 0.0f : __fsub_rn(ls, __fmul_rn(__fdiv_rn(t.w, t.s), 0.693147180559945f)));
    if (bad) flag(p.dev_status, OCS_DEV_NONFINITE);
    if (p.entropy) p.entropy[r] = H;
    if (p.stats)
      reinterpret_cast<float4*>(p.stats)[r] = make_float4(bad ? nan : t.m, ls, H, fmaf(t.m, p.beta, ls));
    if (p.logprob)
      p.logprob[r] = bad ? nan : (y < 0 ? 0.0f : (empty ? -INFINITY : __fsub_rn(__fmul_rn(__fsub_rn(ly, t.m), p.beta), ls)));
  }
  for (int i = tid; i < p.top_k; i += kLpThreads) {
    const key_t k = best[i];
    if (p.top_ids) p.top_ids[r * p.top_k + i] = bad ? -1 : key_index(k);
    if (p.top_logprob)
      p.top_logprob[r * p.top_k + i] =
          bad ? nan : (empty ? -INFINITY : __fsub_rn(__fmul_rn(__fsub_rn(key_value(k), t.m), p.beta), ls));
  }
}

struct GradParams {
  long long ld, ld_d;
  int V, chunks;
  const int32_t* targets;
  float beta, c;
  const float *stats, *g_logprob, *g_entropy;
  int* dev_status;
};

template <typename T> __device__ __forceinline__ uint32_t pack_pair(float a, float b);
template <> __device__ __forceinline__ uint32_t pack_pair<__half>(float a, float b) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
template <> __device__ __forceinline__ uint32_t pack_pair<__nv_bfloat16>(float a, float b) { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }

constexpr int kGradVecs = 4;   // vectors a thread of the gradient kernel handles

// One part of a row per CTA: read, p = 2^((l - m) * c - log2 s), the gradient, write.
template <typename T>
__global__ void __launch_bounds__(kLpThreads) logprobs_backward_kernel(const T* logits, T* d_logits, const GradParams p) {
  constexpr int VE = Vec<T>::VE;
  const long long r = blockIdx.x / p.chunks;
  const int chunk = blockIdx.x - (int)(r * p.chunks);
  const RowVectors<T> row(logits + r * p.ld, p.V);
  T* dst = d_logits + r * p.ld_d;
  const int j0 = chunk * (kGradVecs * kLpThreads) + threadIdx.x;
  Vec<T> v[kGradVecs];
#pragma unroll
  for (int u = 0; u < kGradVecs; ++u) {
    const int j = j0 + u * kLpThreads;
    if (j < row.count) v[u] = row.load(j);
  }
  const float4 st = __ldg(reinterpret_cast<const float4*>(p.stats) + r);
  const float gh = p.g_entropy ? __ldg(p.g_entropy + r) : 0.0f;
  int y = p.targets ? __ldg(p.targets + r) : -1;
  if (y >= p.V) {
    if (chunk == 0 && threadIdx.x == 0) flag(p.dev_status, OCS_DEV_BAD_INDEX);
    y = -1;
  }
  const float g = p.g_logprob && y >= 0 ? __ldg(p.g_logprob + r) : 0.0f;
  const bool empty = st.x == -INFINITY;
  const float ls2 = __fmul_rn(st.y, 1.44269504088896f);
  // d = -beta * p * (g + gh * (ln p + H)) = p * (A + B * log2 p)
  const float A = -__fmul_rn(p.beta, fmaf(gh, st.z, g)), B = -__fmul_rn(__fmul_rn(gh, 0.693147180559945f), p.beta);
  const unsigned long long neg = pack_f32x2(-st.x, -st.x), c2 = pack_f32x2(p.c, p.c), l2 = pack_f32x2(-ls2, -ls2);
  const unsigned long long A2 = pack_f32x2(A, A), B2 = pack_f32x2(B, B);
  const bool same = ((reinterpret_cast<uintptr_t>(dst) ^ reinterpret_cast<uintptr_t>(row.x)) & 15) == 0;
#pragma unroll
  for (int u = 0; u < kGradVecs; ++u) {
    const int j = j0 + u * kLpThreads;
    if (j >= row.count) break;
    const int e0 = row.first(j);
    float d[VE];
#pragma unroll
    for (int i = 0; i < VE / 2; ++i) {
      float q0, q1;
      unpack_f32x2(fma_f32x2(add_f32x2(v[u].pair(i), neg), c2, l2), q0, q1);
      q0 = fmaxf(q0, kFloor);
      q1 = fmaxf(q1, kFloor);
      unpack_f32x2(mul_f32x2(pack_f32x2(ex2(q0), ex2(q1)), fma_f32x2(B2, pack_f32x2(q0, q1), A2)), d[2 * i], d[2 * i + 1]);
    }
    if ((unsigned)(y - e0) < (unsigned)VE && y >= 0 && !empty) {   // the given token is in this vector
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (e0 + e == y) d[e] = fmaf(g, p.beta, d[e]);
    }
    if (same && row.whole(j)) {
      uint4 o;
      if constexpr (sizeof(T) == 4)
        o = make_uint4(__float_as_uint(d[0]), __float_as_uint(d[1]), __float_as_uint(d[2]), __float_as_uint(d[3]));
      else
        o = make_uint4(pack_pair<T>(d[0], d[1]), pack_pair<T>(d[2], d[3]), pack_pair<T>(d[4], d[5]), pack_pair<T>(d[6], d[7]));
      *reinterpret_cast<uint4*>(dst + e0) = o;
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if ((unsigned)(e0 + e) < (unsigned)p.V) dst[e0 + e] = from_f32<T>(d[e]);
    }
  }
}

// CTAs that share a row: enough of them for every SM to have its four, each with a few vectors for every thread.
int row_ctas(long long rows, int V, int ve) {
  int cl = 1;
  while (cl < kMaxCluster && rows * cl < 8ll * kNumSMs && (long long)V > 8ll * cl * kLpThreads * ve) cl *= 2;
  return cl;
}

template <typename T>
ocs_status launch_logprobs(const void* logits_, LogprobParams p, cudaStream_t stream) {
  const T* logits = static_cast<const T*>(logits_);
  const int cl = row_ctas(p.rows, p.V, Vec<T>::VE);
  const long long rows = p.rows, step = 1ll << 27;   // rows of one launch (the grid's limit)
  for (long long r0 = 0; r0 < rows; r0 += step) {
    const long long n = rows - r0 < step ? rows - r0 : step;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n * cl), 1, 1);
    cfg.blockDim = dim3(kLpThreads, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cl; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = cl > 1 ? 1 : 0;
    LaunchScope ls("logprobs_kernel", stream);
    if (cudaLaunchKernelEx(&cfg, logprobs_kernel<T>, logits + r0 * p.ld, p) != cudaSuccess) return OCS_ERR_CUDA;
    if (p.targets) p.targets += n;
    if (p.logprob) p.logprob += n;
    if (p.entropy) p.entropy += n;
    if (p.stats) p.stats += 4 * n;
    if (p.top_ids) p.top_ids += n * p.top_k;
    if (p.top_logprob) p.top_logprob += n * p.top_k;
  }
  return launch_status();
}

template <typename T>
ocs_status launch_backward(const void* logits_, void* d_logits_, long long rows, GradParams p, cudaStream_t stream) {
  const T* logits = static_cast<const T*>(logits_);
  T* d_logits = static_cast<T*>(d_logits_);
  // vectors of a row that starts anywhere: one more than V / VE rounded up at the most
  const int vecs = p.V / Vec<T>::VE + 2, per = kGradVecs * kLpThreads;
  p.chunks = (vecs + per - 1) / per;
  const long long step = 0x7fffffffll / p.chunks;
  for (long long r0 = 0; r0 < rows; r0 += step) {
    const long long n = rows - r0 < step ? rows - r0 : step;
    LaunchScope ls("logprobs_backward_kernel", stream);
    logprobs_backward_kernel<T><<<(unsigned)(n * p.chunks), kLpThreads, 0, stream>>>(logits + r0 * p.ld, d_logits + r0 * p.ld_d, p);
    if (p.targets) p.targets += n;
    if (p.g_logprob) p.g_logprob += n;
    if (p.g_entropy) p.g_entropy += n;
    p.stats += 4 * n;
  }
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
  const float c = (float)((double)inv_temperature * 1.4426950408889634);
  LogprobParams p{rows, ld, V, top_k, targets, inv_temperature, c, logprob, entropy, top_logprob, stats, top_ids, dev_status};
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
  const float c = (float)((double)inv_temperature * 1.4426950408889634);
  GradParams p{ld, ld_d, V, 0, targets, inv_temperature, c, stats, g_logprob, g_entropy, dev_status};
  switch (type) {
    case OCS_F16: return launch_backward<__half>(logits, d_logits, rows, p, stream);
    case OCS_BF16: return launch_backward<__nv_bfloat16>(logits, d_logits, rows, p, stream);
    default: return launch_backward<float>(logits, d_logits, rows, p, stream);
  }
}
