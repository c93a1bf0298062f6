// ocs_token_logprobs and its gradient: log probabilities of given tokens, entropy and the likeliest tokens.
// With m = max l, c = inv_temperature * log2 e, d_v = (l_v - m) * c, s = sum 2^d, w = sum 2^d d:
//     ln p_v = (l_v - m) * inv_temperature - ln s,   entropy = ln s - ln 2 * w / s,
// so one pass over the logits with running sums gives everything, and the likeliest tokens come from a threshold found among
// the threads' maxima.
#include <cmath>
#include <type_traits>

#include "elem.cuh"
#include "ptx.cuh"

namespace ocs {
namespace {

constexpr int kMaxTop = 64;
constexpr int kLpThreads = 256;       // threads of a CTA; the forward kernel also has forms with fewer (NT)
constexpr int kMaxCluster = 8;        // CTAs that may share a row
constexpr float kFloor = -200.0f;     // 2^-200 is zero in fp32: exponents are clamped here, so that a masked token (d = -inf)
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
// Stand-in for masked tokens (-infinity, or a finite value below it) in the sums: so low that 2^d is zero, and near enough
// to zero that its product with c rounds by no more than one, like that of every logit that the sums can take (sums_hold()
// says which).  `two`: in both halves of a word, in the logits' type.
struct Low {
  float v;
  uint32_t two;
};
// 32 bytes of a row
template <typename T>
struct Vec {
  static constexpr int VE = 32 / (int)sizeof(T);
  uint32_t w[8];
  __device__ __forceinline__ void load(const void* p) {   // 32-byte aligned
    asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
  }
  __device__ __forceinline__ void floats(float* f) const;      // the elements as fp32
  __device__ __forceinline__ void floored(float* f, const Low& low) const;   // ... in 16 bits none below low (a packed maximum)
  __device__ __forceinline__ float max_all() const;            // the largest; NaN if any element is
};

template <> __device__ __forceinline__ void Vec<float>::floats(float* f) const {
#pragma unroll
  for (int i = 0; i < 8; ++i) f[i] = __uint_as_float(w[i]);
}
template <> __device__ __forceinline__ void Vec<float>::floored(float* f, const Low&) const { floats(f); }
template <> __device__ __forceinline__ float Vec<float>::max_all() const {
  float m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = max_nan(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
  return max_nan(max_nan(m[0], m[1]), max_nan(m[2], m[3]));
}
__device__ __forceinline__ void widen(__nv_bfloat162 h, float* f) {
  const uint32_t b = *reinterpret_cast<const uint32_t*>(&h);
  f[0] = __uint_as_float(b << 16);
  f[1] = __uint_as_float(b & 0xffff0000u);
}
__device__ __forceinline__ void widen(__half2 h, float* f) {
  const float2 x = __half22float2(h);
  f[0] = x.x;
  f[1] = x.y;
}
template <typename H2> __device__ __forceinline__ H2 as_half2(uint32_t w) { return *reinterpret_cast<const H2*>(&w); }
template <typename H2>
__device__ __forceinline__ float packed_max(const uint32_t* w) {
  H2 m[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) m[i] = __hmax2_nan(as_half2<H2>(w[2 * i]), as_half2<H2>(w[2 * i + 1]));
  float f[2];
  widen(__hmax2_nan(__hmax2_nan(m[0], m[1]), __hmax2_nan(m[2], m[3])), f);
  return max_nan(f[0], f[1]);
}
template <> __device__ __forceinline__ void Vec<__nv_bfloat16>::floats(float* f) const {
#pragma unroll
  for (int i = 0; i < 8; ++i) widen(as_half2<__nv_bfloat162>(w[i]), f + 2 * i);
}
template <> __device__ __forceinline__ void Vec<__nv_bfloat16>::floored(float* f, const Low& low) const {
#pragma unroll
  for (int i = 0; i < 8; ++i) widen(__hmax2(as_half2<__nv_bfloat162>(w[i]), as_half2<__nv_bfloat162>(low.two)), f + 2 * i);
}
template <> __device__ __forceinline__ float Vec<__nv_bfloat16>::max_all() const { return packed_max<__nv_bfloat162>(w); }
template <> __device__ __forceinline__ void Vec<__half>::floats(float* f) const {
#pragma unroll
  for (int i = 0; i < 8; ++i) widen(as_half2<__half2>(w[i]), f + 2 * i);
}
template <> __device__ __forceinline__ void Vec<__half>::floored(float* f, const Low& low) const {
#pragma unroll
  for (int i = 0; i < 8; ++i) widen(__hmax2(as_half2<__half2>(w[i]), as_half2<__half2>(low.two)), f + 2 * i);
}
template <> __device__ __forceinline__ float Vec<__half>::max_all() const { return packed_max<__half2>(w); }

template <typename T> __device__ __forceinline__ T minus_infinity();
template <> __device__ __forceinline__ float minus_infinity<float>() { return -INFINITY; }
template <> __device__ __forceinline__ __half minus_infinity<__half>() { return __ushort_as_half(0xfc00); }
template <> __device__ __forceinline__ __nv_bfloat16 minus_infinity<__nv_bfloat16>() { return __ushort_as_bfloat16(0xff80); }

// A row as aligned vectors of 32 bytes: vector j holds elements j * VE - a .. j * VE - a + VE - 1, where a is how many
// elements past a 32-byte boundary the row starts.  The first and the last one may hang over; what lies outside the row is
// never read and counts as -infinity.
template <typename T>
struct RowVectors {
  static constexpr int VE = Vec<T>::VE;
  const T* x;
  int V, a, count, n_whole;    // vectors (a > 0) .. (a > 0) + n_whole - 1 lie inside the row
  __device__ __forceinline__ RowVectors(const T* row, int n) : x(row), V(n) {
    a = (int)((reinterpret_cast<uintptr_t>(row) & 31) / sizeof(T));
    count = (V + a + VE - 1) / VE;
    n_whole = (V + a) / VE - (a > 0);
  }
  __device__ __forceinline__ int first(int j) const { return j * VE - a; }
  __device__ __forceinline__ bool whole(int j) const { return j - (a > 0) >= 0 && j - (a > 0) < n_whole; }
  __device__ __forceinline__ Vec<T> load(int j) const {
    Vec<T> v;
    const int e0 = first(j);
    if (whole(j)) {
      v.load(x + e0);
    } else {
      T* e = reinterpret_cast<T*>(v.w);
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
__device__ __forceinline__ void shift(Stats& t, float d) {   // every term's exponent moves by d
  t.w = __fmul_rn(fmaf(t.s, d, t.w), ex2(d));
  t.s = __fmul_rn(t.s, ex2(d));
}
// c * up = inv_temperature * log2 e; up is 1, or 2 where that product may not be finite
struct Scale {
  float c, up;
};
__host__ __device__ __forceinline__ float up_of(float beta) { return beta > 0x1p127f ? 2.0f : 1.0f; }
// (l - m) * c * up, l <= m.  Halves keep the difference finite where logits near both ends of fp32 meet.
__device__ __forceinline__ float scaled_distance(float l, float m, Scale k) {
  const bool far = fabsf(m) > 0x1p100f;
  const float h = far ? 0.5f : 1.0f;
  return __fmul_rn(__fmul_rn(__fsub_rn(__fmul_rn(l, h), __fmul_rn(m, h)), k.c), far ? __fadd_rn(k.up, k.up) : k.up);
}
// The exponent of a logit relative to m in base 2.  ENDS: inverse temperatures outside of [2^-64, 2^64].  Between them a
// difference that overflows has p = 0 anyway, and c is finite.
template <bool ENDS>
__device__ __forceinline__ float exponent(float l, float m, Scale k) {
  return ENDS ? scaled_distance(l, m, k) : __fmul_rn(__fsub_rn(l, m), k.c);
}
template <bool ENDS>
__device__ __forceinline__ void move_max(Stats& t, float m, Scale k) {   // the same sums relative to another maximum
  shift(t, fmaxf(exponent<ENDS>(t.m, m, k), kFloor));                    // -infinity or NaN (nothing summed yet): s = w = 0
  t.m = m;
}
// The main loop takes d = fma(l, c, -M) with M = fl(m * c) instead of (l - m) * c: one instruction, one rounding.  M's own
// rounding stays in d until the sums move to m * c at the end, so it has to be small: up to |m * c| = 2^24 it is at most
// one, while from 2^31 on it would carry 2^d out of range.  That holds for every M of a row whose maximum and whose
// stand-in for masked tokens (low) are that near to zero.  The stand-in also has to be far enough below the maximum.
// Otherwise (a row's largest logit far from zero, or nothing in it above a finite mask value) the sums are taken once more
// in the other form.
__device__ __forceinline__ bool sums_hold(float m, float c, float low) {
  return __fmul_rn(fabsf(m), c) <= 0x1p24f && __fmul_rn(-low, c) <= 0x1p24f && c < 0x1p20f &&
         __fmul_rn(__fsub_rn(low, m), c) <= -160.0f;
}
__device__ __forceinline__ float warp_max(float m) {   // NaN if any lane's is
  float r;
  asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(m));
  return r;
}
// Sums over groups of LANES lanes, whose statistics are relative to one maximum.
template <int LANES>
__device__ __forceinline__ void add_lanes(Stats& t) {
#pragma unroll
  for (int o = LANES / 2; o > 0; o >>= 1) {
    t.s = __fadd_rn(t.s, __shfl_xor_sync(0xffffffffu, t.s, o));
    t.w = __fadd_rn(t.w, __shfl_xor_sync(0xffffffffu, t.w, o));
  }
}
// The sums of vectors [lo, hi) relative to m in the other form: this warp's share, in every lane.
template <bool ENDS, int NT, typename T>
__device__ __forceinline__ Stats sums_of_differences(const RowVectors<T>& row, int lo, int hi, float m, Scale k) {
  Stats t{m, 0.0f, 0.0f};
  for (int j = lo + threadIdx.x; j < hi; j += NT) {
    float f[Vec<T>::VE];
    row.load(j).floats(f);
#pragma unroll
    for (int i = 0; i < Vec<T>::VE; ++i) {
      const float d = fmaxf(exponent<ENDS>(f[i], m, k), kFloor), e = ex2(d);
      t.s = __fadd_rn(t.s, e);
      t.w = fmaf(e, d, t.w);
    }
  }
  add_lanes<32>(t);
  return t;
}
// The eight parts that lanes 0..7 hold (and lanes 8..15, ... again) as one, in every lane.
template <bool ENDS>
__device__ __forceinline__ Stats join_eight(Stats t, Scale k) {
  move_max<ENDS>(t, warp_max(t.m), k);
  add_lanes<8>(t);
  return t;
}

// One thread's share of a row: its largest element m, the first vector that holds it, and the sums relative to M (in
// two chains each).  M is not the running maximum but follows it at a distance of up to kLag: it starts at the largest
// first element of the warp's threads, so that almost no later vector has to scale the sums.
constexpr float kLag = 8.0f;
struct Running {
  float m, M, s[2], w[2];
  int pos;
};
template <typename T>
__device__ __forceinline__ void take(Running& t, const Vec<T>& v, int j, float c, const Low& low) {
  constexpr int VE = Vec<T>::VE;
  const float mx = v.max_all();
  if (mx > t.m) t.pos = j;
  t.m = max_nan(t.m, mx);
  const float to = __fmul_rn(fmaxf(mx, low.v), c);
  if (to > __fadd_rn(t.M, kLag)) {
    const float d = fmaxf(__fsub_rn(t.M, to), kFloor), r = ex2(d);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      t.w[i] = __fmul_rn(fmaf(t.s[i], d, t.w[i]), r);
      t.s[i] = __fmul_rn(t.s[i], r);
    }
    t.M = to;
  }
  float f[VE];
  v.floored(f, low);
#pragma unroll
  for (int i = 0; i < VE; ++i) {
    float d = fmaf(f[i], c, -t.M);
    if constexpr (sizeof(T) == 4) d = fmaxf(d, kFloor);
    const float e = ex2(d);
    t.s[i & 1] = __fadd_rn(t.s[i & 1], e);
    t.w[i & 1] = fmaf(e, d, t.w[i & 1]);
  }
}

// (Every 8 bytes of a kernel's parameters cost the host about 0.3 us of a small call, so what a thread works out in an
// instruction or two stays out of them.  The stand-in is here because in a register it costs 16-bit rows 1 to 3 %.)
struct LogprobParams {
  long long ld;
  int V, top_k;
  const int32_t* targets;
  float beta, c;
  Low low;
  float *logprob, *entropy, *top_logprob, *stats;
  int32_t* top_ids;
  int* dev_status;
};

// A bisection for the k largest ends with at most this many.
__host__ __device__ constexpr int threads_left(int k) { return k + k / 2 + 8; }

// NT threads; only CTAs of kLpThreads share rows
template <int NT>
struct LogprobSmem {
  static constexpr int kWarps = NT / 32;
  static constexpr int kCandidates = 8 * NT + 16;   // elements that can still be among the largest
  static_assert(kCandidates >= 16 * (kMaxTop - 1), "fewer vectors than alternatives are collected whole");
  static constexpr int kLists = NT == kLpThreads ? kMaxCluster : 1;
  static_assert(kWarps <= 8 && kMaxCluster == 8, "join_eight");
  Stats warp[8];
  Stats part[kMaxCluster];                             // of the CTAs that share the row
  __align__(16) key_t cand[kCandidates];
  __align__(16) key_t top[kLists * kMaxTop];           // each CTA's largest, descending
  key_t best[kMaxTop];                                 // the row's
  __align__(16) key_t few[threads_left(kMaxTop)];      // what is ranked of many candidates
  int count[2][kWarps];
  uint32_t low[kWarps];                                // the smallest of a warp's threads' largest elements, as ord_encode
  key_t next[kWarps];
  int hot[NT];
  int n_hot, n_cand;
};

// How many of n keys are larger than v.
__device__ __forceinline__ int count_larger(const key_t* list, int n, key_t v) {
  const ulonglong2* two = reinterpret_cast<const ulonglong2*>(list);
  int r = 0;
#pragma unroll 4
  for (int i = 0; i < n / 2; ++i) {
    const ulonglong2 k = two[i];
    r += (k.x > v) + (k.y > v);
  }
  if (n & 1) r += list[n - 1] > v;
  return r;
}

__device__ __forceinline__ key_t warp_max_key(key_t v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const key_t other = __shfl_xor_sync(0xffffffffu, v, o);
    v = other > v ? other : v;
  }
  return v;
}

// The k largest elements of vectors [lo, hi) of the row, descending, as keys in out (zeros where there are fewer), given
// every thread's largest element (its value m, and the vector that holds it first), the segment's, and in sm every warp's
// smallest m, a count of zero and zeros in out.
//   1. tau: a key that at least k of the threads' largest elements are not below, and not many more than k, by bisection
//      (each step counts with one barrier).  The threads' keys are lowered to the last index of their vector, so at least
//      k elements are not below tau, and only threads whose key, raised to the first index, is not below tau hold one.
//   2. All threads read these threads' elements again and collect what is not below tau.
//   3. The k largest of what was collected, by rank.
// Equal elements side by side make candidates of whole vectors.  So the bisection goes on until the vectors that are left
// fit the list, and more than 2 NT candidates are bisected once more, element by element, before they are ranked (ranking
// takes n^2 / NT steps).  Rows of one value, 2000 x 8000 bf16, 64 alternatives: 40 us against 771 without both (random rows
// 32); rows with ten unmasked tokens 102 against 780.  Elements that are placed unluckily (one thread's vectors hold most of
// the largest) may still overflow the list; then the keys are found one after the other.
template <int NT, typename T>
__device__ void top_of_segment(const RowVectors<T>& row, int lo, int hi, int k, float m, int pos, float largest,
                               LogprobSmem<NT>& sm, key_t* out) {
  constexpr int VE = Vec<T>::VE, kWarps = LogprobSmem<NT>::kWarps, kCandidates = LogprobSmem<NT>::kCandidates;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool any = lo + tid < hi;
  key_t tau = 0;
  if (hi - lo >= k) {   // k threads have an element; with fewer of them nothing is left out
    const key_t low = any ? top_key(m, min(row.first(pos) + VE, row.V) - 1) : 0;
    uint32_t least = sm.low[0];
#pragma unroll
    for (int w = 1; w < kWarps; ++w) least = min(least, sm.low[w]);
    // all threads that have one are at or above tau, k - 1 at the most at or above `above`
    tau = (key_t)least << 32;
    key_t above = (key_t)ord_encode(largest + 0.0f) << 32 | 0xffffffffu;
    const int enough = max(k, min(threads_left(k), kCandidates / VE - 1));   // (and a vector that tau cuts through)
    while (above - tau > 1) {
      const key_t mid = tau + (above - tau) / 2;
      const int n = __syncthreads_count(low >= mid);
      if (n >= k) tau = mid;
      else above = mid;
      if (n >= k && n <= enough) break;
    }
  }
  if (any && top_key(m, max(row.first(pos), 0)) >= tau) sm.hot[atomicAdd(&sm.n_hot, 1)] = tid;
  __syncthreads();
  const int vecs = (hi - lo + NT - 1) / NT, total = sm.n_hot * vecs;
  for (int q = tid; q < total; q += NT) {
    const int h = q / vecs;
    const int j = lo + sm.hot[h] + (q - h * vecs) * NT;
    if (j >= hi) continue;
    const Vec<T> v = row.load(j);
    if (ord_encode(v.max_all() + 0.0f) < (uint32_t)(tau >> 32)) continue;
    float f[VE];
    v.floats(f);
    const int first = row.first(j);
#pragma unroll
    for (int i = 0; i < VE; ++i) {
      const key_t key = top_key(f[i], first + i);
      if (key >= tau && (unsigned)(first + i) < (unsigned)row.V) {
        const int at = atomicAdd(&sm.n_cand, 1);
        if (at < kCandidates) sm.cand[at] = key;
      }
    }
  }
  __syncthreads();
  const int n = sm.n_cand;
  if (n <= kCandidates && n > 2 * NT) {
    key_t cut = tau, above = (key_t)ord_encode(largest + 0.0f) << 32 | 0x80000000u;   // (no index' part is as large)
    for (int b = 0; above - cut > 1; b ^= 1) {
      const key_t mid = cut + (above - cut) / 2;
      int c = 0;
      for (int i = tid; i < n; i += NT) c += sm.cand[i] >= mid;
      c = __reduce_add_sync(0xffffffffu, c);
      if (lane == 0) sm.count[b][warp] = c;
      __syncthreads();
      c = 0;
#pragma unroll
      for (int w = 0; w < kWarps; ++w) c += sm.count[b][w];
      if (c >= k) cut = mid;
      else above = mid;
      if (c >= k && c <= threads_left(k)) break;
    }
    if (tid == 0) sm.n_hot = 0;
    __syncthreads();
    for (int i = tid; i < n; i += NT)
      if (sm.cand[i] >= cut) {
        const int at = atomicAdd(&sm.n_hot, 1);
        if (at < threads_left(k)) sm.few[at] = sm.cand[i];
      }
    __syncthreads();
    const int left = min(sm.n_hot, threads_left(k));
    for (int i = tid; i < left; i += NT) {
      const int r = count_larger(sm.few, left, sm.few[i]);
      if (r < k) out[r] = sm.few[i];
    }
  } else if (n <= kCandidates) {
    for (int i = tid; i < n; i += NT) {
      const key_t mine = sm.cand[i];
      const int r = count_larger(sm.cand, n, mine);
      if (r < k) out[r] = mine;
    }
  } else {
    key_t last = ~0ull;
    for (int r = 0; r < k; ++r) {
      key_t best = 0;
      for (int j = lo + tid; j < hi; j += NT) {
        float f[VE];
        row.load(j).floats(f);
#pragma unroll
        for (int i = 0; i < VE; ++i) {
          const int idx = row.first(j) + i;
          const key_t key = (unsigned)idx < (unsigned)row.V ? top_key(f[i], idx) : 0;
          if (key < last && key > best) best = key;
        }
      }
      best = warp_max_key(best);
      if (lane == 0) sm.next[warp] = best;
      __syncthreads();
      for (int w = 0; w < kWarps; ++w) best = max(best, sm.next[w]);
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
// A thread strides over its CTA's part in vectors of 32 bytes, one of them on its way while another is summed; five CTAs of
// 256 threads per SM, or ten of 128 (48 registers).  Deeper prefetch with fewer CTAs is slower (three and four vectors,
// four CTAs: 52 us at 2048 rows of 50257 bf16 logits; one vector, six CTAs: 53; this form 50 at the time).  What bounds it: fp32
// rows the loads (2500 x 33278: 53.3 us for 333 MB, 6.2 TB/s, without alternatives); 16-bit rows the instructions, six per
// element and one of them an exponential (2048 x 50257 bf16, 206 MB: 39.5 us, 5.2 TB/s).  Five alternatives add about 3 us per
// wave of CTAs: 47.9 us there; 20.6 instead of 17.7 us for 700 rows of 33278 fp32 logits (93 MB), which are one wave.  Few
// rows are latency: 8 x 131072 bf16 takes 4.5 us, 8.5 with twenty alternatives.
template <typename T, int NT, bool ENDS>
__global__ void __launch_bounds__(NT, 5 * 256 / NT) logprobs_kernel(const T* __restrict__ logits, const LogprobParams p) {
  constexpr int VE = Vec<T>::VE, kWarps = NT / 32;
  __shared__ LogprobSmem<NT> sm;
  const int CL = NT == kLpThreads ? (int)cluster_size() : 1, rank = CL > 1 ? (int)cluster_rank() : 0;
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

  const float c = p.c;
  const Scale scale{c, up_of(p.beta)};
  const Low low = p.low;
  Running run{-INFINITY, 0.0f, {0.0f, 0.0f}, {0.0f, 0.0f}, lo + tid};
  {
    int j = lo + tid;
    const int end = min(hi, (row.a > 0) + row.n_whole);
    const char* src = reinterpret_cast<const char*>(row.x - row.a);   // vector j starts at src + 32 j
    Vec<T> v, w;   // one is on its way while the other is summed
    const bool some = j < hi;
    if (some) v = row.load(j);
    if (j + NT < end) w.load(src + 32ll * (j + NT));
    run.M = __fmul_rn(fmaxf(warp_max(some ? v.max_all() : -INFINITY), low.v), c);
    if (some) take(run, v, j, c, low);
    if (j + 2 * NT < end) v.load(src + 32ll * (j + 2 * NT));
    for (j += NT; j < end; j += 2 * NT) {
      take(run, w, j, c, low);
      if (j + 2 * NT < end) w.load(src + 32ll * (j + 2 * NT));
      if (j + NT >= end) { j += NT; break; }
      take(run, v, j + NT, c, low);
      if (j + 3 * NT < end) v.load(src + 32ll * (j + 3 * NT));
    }
    if (j < hi) {   // the row's last vector, hanging over
      v = row.load(j);
      take(run, v, j, c, low);
    }
  }
  Stats t{warp_max(run.m), __fadd_rn(run.s[0], run.s[1]), __fadd_rn(run.w[0], run.w[1])};
  if (t.m > low.v) {         // from M to m * c
    const float d = fmaxf(fmaf(-t.m, c, run.M), kFloor), r = ex2(d), moved = fmaf(t.s, d, t.w);
    t.s = __fmul_rn(t.s, r);
    t.w = fabsf(moved) <= 0x1p-22f * fabsf(t.w) ? 0.0f : __fmul_rn(moved, r);   // of equals only rounding would be left
  } else {
    t.s = t.w = 0.0f;        // nothing but masked tokens as far as the sums can tell
  }
  add_lanes<32>(t);
  key_t* top = sm.top + rank * p.top_k;
  if (p.top_k > 0) {         // what top_of_segment() expects
    const uint32_t least = __reduce_min_sync(0xffffffffu, lo + tid < hi ? ord_encode(run.m + 0.0f) : 0xffffffffu);
    if (lane == 0) sm.low[warp] = least;
    if (tid < p.top_k) top[tid] = 0;
    if (tid == 0) sm.n_hot = sm.n_cand = 0;
  }
  if (lane == 0) sm.warp[warp] = t;
  if (kWarps < 8 && tid >= kWarps && tid < 8) sm.warp[tid] = Stats{-INFINITY, 0.0f, 0.0f};
  __syncthreads();
  float largest = sm.warp[0].m;
#pragma unroll
  for (int w = 1; w < kWarps; ++w) largest = max_nan(largest, sm.warp[w].m);
  // A part of a row with nothing above the stand-in is usually a masked stretch that weighs nothing beside the other parts:
  // it stays without sums (s = 0), and the first CTA sees whether that was right (370 x 128000 bf16, nine tenths masked with
  // -1e9: 20.6 us, 34 with the sums taken here).
  const bool left_out = !ENDS && CL > 1 && largest <= low.v;
  if (fabsf(largest) < INFINITY && !left_out && (ENDS || !sums_hold(largest, c, low.v))) {   // the same for the whole CTA
    __syncthreads();
    t = sums_of_differences<ENDS, NT>(row, lo, hi, largest, scale);
    if (lane == 0) sm.warp[warp] = t;
    __syncthreads();
  }
  if (p.top_k > 0) top_of_segment(row, lo, hi, p.top_k, run.m, run.pos, largest, sm, top);
  t = join_eight<ENDS>(sm.warp[lane & 7], scale);   // this CTA's part of the row, in every thread
  if (CL > 1) {
    asm volatile("barrier.cluster.wait;" ::: "memory");
    if (rank != 0) {
      if (tid == 0) {
        const uint32_t dst = peer_addr(smem_u32(&sm.part[rank]), 0);
        store_peer_f32(dst, t.m);
        store_peer_f32(dst + 4, t.s);
        store_peer_f32(dst + 8, t.w);
      }
      for (int i = tid; i < p.top_k; i += NT)
        store_peer_u64(peer_addr(smem_u32(&sm.top[rank * p.top_k + i]), 0), sm.top[rank * p.top_k + i]);
      __syncwarp();
      asm volatile("barrier.cluster.arrive.release;" ::: "memory");
      return;   // the first CTA's memory outlives the stores: it waits for this arrival
    }
    asm volatile("barrier.cluster.arrive.release;" ::: "memory");
    asm volatile("barrier.cluster.wait.acquire;" ::: "memory");
    const Stats own = t;
    const int part = lane & 7;
    t = part == 0 ? own : (part < CL ? sm.part[part] : Stats{-INFINITY, 0.0f, 0.0f});
    if (!ENDS && __any_sync(0xffffffffu, t.s == 0.0f && fabsf(t.m) < INFINITY)) {   // a part without sums; the same in every warp
      const float row_max = warp_max(t.m);
      if (__any_sync(0xffffffffu, t.s == 0.0f && fabsf(t.m) < INFINITY && exponent<ENDS>(t.m, row_max, scale) > -160.0f)) {
        t = sums_of_differences<ENDS, NT>(row, 0, row.count, row_max, scale);   // it counts
        if (lane == 0) sm.warp[warp] = t;
        __syncthreads();
        t = sm.warp[part];
      }
    }
    t = join_eight<ENDS>(t, scale);
    if (p.top_k > 0) {
      for (int i = tid; i < CL * p.top_k; i += NT) {
        const key_t k = sm.top[i];
        const int at = k != 0 ? count_larger(sm.top, CL * p.top_k, k) : kMaxTop;
        if (at < p.top_k) sm.best[at] = k;
      }
      __syncthreads();
    }
  }
  const key_t* best = CL > 1 ? sm.best : sm.top;
  const bool bad = !(t.m < INFINITY), empty = t.m == -INFINITY;
  const float nan = __int_as_float(0x7fffffff);
  const float ls = bad ? nan : (empty ? 0.0f : logf(t.s));
  if (tid == 0) {
    // (an entropy is not negative; rounding alone could make it so)
    const float H = bad ? nan : (empty ? 0.0f : max_nan(__fsub_rn(ls, __fmul_rn(__fdiv_rn(t.w, t.s), 0.693147180559945f)), 0.0f));
    if (bad) flag(p.dev_status, OCS_DEV_NONFINITE);
    if (p.entropy) p.entropy[r] = H;
    if (p.stats)
      reinterpret_cast<float4*>(p.stats)[r] = make_float4(bad ? nan : t.m, ls, H, fmaf(t.m, p.beta, ls));
    if (p.logprob)
      p.logprob[r] = bad ? nan : (y < 0 ? 0.0f : (empty ? -INFINITY : __fsub_rn(scaled_distance(ly, t.m, Scale{p.beta, 1.0f}), ls)));
  }
  for (int i = tid; i < p.top_k; i += NT) {
    const key_t k = best[i];
    if (p.top_ids) p.top_ids[r * p.top_k + i] = bad ? -1 : key_index(k);
    if (p.top_logprob)
      p.top_logprob[r * p.top_k + i] =
          bad ? nan : (empty ? -INFINITY : __fsub_rn(scaled_distance(key_value(k), t.m, Scale{p.beta, 1.0f}), ls));
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

constexpr int kGradVecs = 2;   // vectors a thread of the gradient kernel handles

// One part of a row per CTA: read, p = 2^((l - m) * c - log2 s), the gradient, write.  The statistics make every element
// independent, so rows are cut into parts of two vectors per thread, all loads of a thread are issued before its first
// arithmetic, and the grid is as large as the tensor.  Bound by HBM: 2048 x 50257 bf16, 412 MB, 63.5 us, 6.5 TB/s (99 % of the
// measured copy rate); 700 x 33278 fp32, 186 MB, 29.7 us, 6.3 TB/s.
template <typename T, bool ENDS>
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
  // d = -beta * p * (g + gh * (ln p + H)) = p * (A + B * log2 p).  ENDS: beta comes last, so that A is not infinite where p is zero.
  const float first = ENDS ? 1.0f : p.beta;
  const float A = -__fmul_rn(first, fmaf(gh, st.z, g)), B = -__fmul_rn(__fmul_rn(gh, 0.693147180559945f), first);
  const bool same = ((reinterpret_cast<uintptr_t>(dst) ^ reinterpret_cast<uintptr_t>(row.x)) & 31) == 0;
#pragma unroll
  for (int u = 0; u < kGradVecs; ++u) {
    const int j = j0 + u * kLpThreads;
    if (j >= row.count) break;
    const int e0 = row.first(j);
    float d[VE];
    v[u].floats(d);
#pragma unroll
    for (int i = 0; i < VE; ++i) {   // by log2 p; a masked token's p is zero
      const float q = fmaxf(ENDS ? __fsub_rn(exponent<true>(d[i], st.x, Scale{p.c, up_of(p.beta)}), ls2) : fmaf(__fsub_rn(d[i], st.x), p.c, -ls2), kFloor);
      d[i] = __fmul_rn(ex2(q), fmaf(B, q, A));
    }
    if ((unsigned)(y - e0) < (unsigned)VE && y >= 0 && !empty) {   // the given token is in this vector
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if (e0 + e == y) d[e] = fmaf(g, first, d[e]);
    }
    if (ENDS) {
#pragma unroll
      for (int e = 0; e < VE; ++e) d[e] = __fmul_rn(d[e], p.beta);
    }
    if (same && row.whole(j)) {
      uint32_t o[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) o[i] = __float_as_uint(d[i]);
        else o[i] = pack_pair<T>(d[2 * i], d[2 * i + 1]);
      }
      asm volatile("st.global.v8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
                   ::"r"(o[0]), "r"(o[1]), "r"(o[2]), "r"(o[3]), "r"(o[4]), "r"(o[5]), "r"(o[6]), "r"(o[7]), "l"(dst + e0) : "memory");
    } else {
#pragma unroll
      for (int e = 0; e < VE; ++e)
        if ((unsigned)(e0 + e) < (unsigned)p.V) dst[e0 + e] = from_f32<T>(d[e]);
    }
  }
}

// CTAs that share a row.  A row alone leaves most SMs idle, so few rows are shared, as long as every thread keeps two
// vectors; but a CTA's fixed cost (about 3 us of start, join and selection, hidden only by other CTAs of its SM) grows with
// their number: the more CTAs a row gets, the fewer there may be in all, and never more than the 740 that are resident at
// once.  Five alternatives, us with 1 / 2 / 4 / 8 CTAs on a row, 16-bit logits unless noted: 1 row of 33278 fp32: 8.1 / 7.1 /
// 6.4 / 6.1; 8 of 131072: 12.8 / 9.5 / 7.6 / 7.0; 64 of 131072: 18.8 / 13.2 / 10.8 / 11.3; 128 of 128000: 19.4 / 14.7 / 14.1 /
// 19.9; 370 of 128000: 26.7 / 24.2 / 34 / 45; 450 of 128000: 32.1 / 34.5 / 38 / 53; 2048 of 50257: 47.9 / 68 / 106 / 179.
int row_ctas(long long rows, int V, int ve) {
  int cl = 1;
  while (cl < kMaxCluster && rows * 2 * cl <= 5 * kNumSMs && rows * 4 * cl * cl <= 2048 &&
         (long long)V > 2ll * cl * kLpThreads * ve)
    cl *= 2;
  return cl;
}

// Threads of a CTA that has a row to itself.  With 128 of them ten rows are under way on an SM instead of five, which hides
// twice as much of the fixed cost; but the alternatives' threads have twice as many vectors each, which are read again, and
// where all rows are resident at once anyway (740 CTAs of 256) a long row takes its threads' time.  us with 128 / 256 threads
// (64 threads were ahead only below 2000 logits): five alternatives, bf16 4096 x 1116: 18.2 / 34.6, 4096 x 8200: 27.9 / 42.9,
// 2500 x 33278: 42.9 / 46.3, 2048 x 50257: 51.8 / 47.9, fp32 2500 x 33278: 65.4 / 67.0, 2048 x 50257: 83.3 / 75.2, 450 x 8200
// even (8.9 / 8.7), but 450 x 16228: 12.6 / 11.0 and 450 x 33278: 20.2 / 16.1; twenty alternatives: bf16 2500 x 16228: 32.2 /
// 35.8, 2500 x 33278: 53.7 / 52.0, fp32 2500 x 33278: 83 / 75 (none: 53.3 / 57.3).
int row_threads(long long rows, int V, int ve, int top_k) {
  const long long vecs = V / (128 * ve);   // a thread's, of 128
  return top_k * vecs <= 320 && (vecs <= 8 || (rows > 5 * kNumSMs && V <= 40960)) ? 128 : kLpThreads;
}

bool at_ends(float beta) { return beta < 0x1p-64f || beta > 0x1p64f; }
float base2(float beta) { return (float)((double)beta * 1.4426950408889634 / up_of(beta)); }

// Low for logits of type T: the power of two whose product with c lies in (-2^24, -2^23], where the type has it.  It bounds
// what the sums tell from a masked token, not what a logit may be: in fp16, where it is the type's lowest value up to c =
// 256, live logits may lie near it, and sums_hold() is what keeps them right.
template <typename T>
Low stand_in(float c) {
  const int k = 23 - std::ilogb(c);
  float v = -std::ldexp(1.0f, k < 100 ? k : 100);
  if constexpr (std::is_same<T, __half>::value) {
    if (v < -65504.0f) v = -65504.0f;
    const __half h = __float2half_rn(v);
    uint16_t b;
    memcpy(&b, &h, 2);
    return Low{v, b * 0x10001u};
  }
  uint32_t b;   // a power of two is its upper half as bf16
  memcpy(&b, &v, 4);
  return Low{v, (b >> 16) * 0x10001u};
}

template <typename T>
ocs_status launch_logprobs(const void* logits_, long long rows, LogprobParams p, cudaStream_t stream) {
  const T* logits = static_cast<const T*>(logits_);
  const bool ends = at_ends(p.beta);
  p.low = stand_in<T>(p.c);
  const int cl = row_ctas(rows, p.V, Vec<T>::VE), nt = cl > 1 || ends ? kLpThreads : row_threads(rows, p.V, Vec<T>::VE, p.top_k);
  const long long step = 1ll << 27;   // rows of one launch (the grid's limit)
  for (long long r0 = 0; r0 < rows; r0 += step) {
    const long long n = rows - r0 < step ? rows - r0 : step;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(n * cl), 1, 1);
    cfg.blockDim = dim3(nt, 1, 1);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = cl; attr[0].val.clusterDim.y = 1; attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr; cfg.numAttrs = cl > 1 ? 1 : 0;
    LaunchScope ls("logprobs_kernel", stream);
    const auto kernel = ends ? logprobs_kernel<T, kLpThreads, true> : nt == 128 ? logprobs_kernel<T, 128, false> : logprobs_kernel<T, kLpThreads, false>;
    if (cudaLaunchKernelEx(&cfg, kernel, logits + r0 * p.ld, p) != cudaSuccess) return OCS_ERR_CUDA;
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
    const auto kernel = at_ends(p.beta) ? logprobs_backward_kernel<T, true> : logprobs_backward_kernel<T, false>;
    kernel<<<(unsigned)(n * p.chunks), kLpThreads, 0, stream>>>(logits + r0 * p.ld, d_logits + r0 * p.ld_d, p);
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
  LogprobParams p{ld, V, top_k, targets, inv_temperature, base2(inv_temperature), Low{}, logprob, entropy, top_logprob, stats, top_ids, dev_status};
  switch (type) {
    case OCS_F16: return launch_logprobs<__half>(logits, rows, p, stream);
    case OCS_BF16: return launch_logprobs<__nv_bfloat16>(logits, rows, p, stream);
    default: return launch_logprobs<float>(logits, rows, p, stream);
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
  GradParams p{ld, ld_d, V, 0, targets, inv_temperature, base2(inv_temperature), stats, g_logprob, g_entropy, dev_status};
  switch (type) {
    case OCS_F16: return launch_backward<__half>(logits, d_logits, rows, p, stream);
    case OCS_BF16: return launch_backward<__nv_bfloat16>(logits, d_logits, rows, p, stream);
    default: return launch_backward<float>(logits, d_logits, rows, p, stream);
  }
}
