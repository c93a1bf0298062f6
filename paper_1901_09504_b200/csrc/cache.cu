// ocs_cache_write / ocs_cache_read: a paged cache of keys and values that is quantized as it is written.
// A page holds page_size tokens x heads vectors: first all their codes, then their block scales, then their row scales, so
// that every section is dense and a page moves as one run of bytes.  A thread has 32 numbers of a vector (16 where fp32 is read): a
// block of E8M0, two of E4M3.  Memory is what should bound them; what a thread does besides its numbers (finding its vector, its
// slot or page) has to stay small against them.  Read back: 350 thousand tokens, keys and values of 8 x 128, E4M3 to bf16 (1.85 GB
// in all) 282 us, 6.5 TB/s, the copy rate; int8 and E8M0 the same.  Written: 100 thousand such tokens (515 MB) 109 us, 4.7 TB/s,
// issue slots 65 % full.
#include "mx4.cuh"

namespace ocs {
namespace {

struct Page {
  int cb, sb;                       // bytes of a vector's codes and block scales
  long long at_s, at_r, bytes;      // sections: block scales, row scales; the page's bytes
};

Page page_layout(int page_size, int heads, int dim, ocs_grid grid) {
  Page g;
  const long long n = (long long)page_size * heads;
  g.cb = (int)align_up((size_t)(grid == OCS_GRID_I8 ? dim : (dim + 1) / 2), 16);
  g.sb = grid == OCS_GRID_I8 ? 0 : (int)align_up((size_t)((dim + mx4_block(grid) - 1) / mx4_block(grid)), 4);
  g.at_s = n * g.cb;
  g.at_r = (long long)align_up((size_t)(g.at_s + n * g.sb), 16);
  g.bytes = (long long)align_up((size_t)(g.at_r + (grid == OCS_GRID_E8M0 ? 0 : 4 * n)), 16);
  return g;
}

struct CacheArgs {
  Page g;
  long long n_slots, rows;
  int page_size, heads, dim, n_pages;
  uint8_t* pages[2];
  void* x[2];                       // vectors outside of the cache: rows of heads x dim elements
  long long ld_row[2], ld_head[2];
  int* dev_status;
  const int64_t* slots;             // write
  const int32_t* table;             // read
  const int32_t* starts;
  long long ld_table;
  int table_cols, B;
};

constexpr int kUnit = 32;           // elements of a vector that a thread has
constexpr int kMaxDim = 1024;

// A group of 2^gs_log2 lanes per vector.  ALIGN: what all vectors are aligned to (32, 16, or 0: their element).
template <typename T, int GRID, int ALIGN>
__global__ void __launch_bounds__(256) cache_write_kernel(const CacheArgs a, int gs_log2) {
  const unsigned long long g = (unsigned long long)blockIdx.x * 256 + threadIdx.x, vec = g >> gs_log2;
  const int lane = (int)g & ((1 << gs_log2) - 1), which = blockIdx.y;
  const long long t = vec >> 32 ? (long long)(vec / (unsigned)a.heads) : (long long)((unsigned)vec / (unsigned)a.heads);
  const int h = (int)(vec - (unsigned long long)t * a.heads);
  const int c = lane * kUnit, left = a.dim - c;      // (left <= 0: a lane of the group beyond the vector)
  long long slot = -1;
  if (t < a.rows) {
    slot = __ldg(a.slots + t);
    if (slot >= a.n_slots) { if (lane == 0) flag(a.dev_status, OCS_DEV_BAD_INDEX); slot = -1; }
  }
  Block<T, kUnit> v;
  if (slot < 0 || left <= 0) v.clear();
  else {
    const T* x = static_cast<const T*>(a.x[which]) + t * a.ld_row[which] + h * a.ld_head[which] + c;
    if (ALIGN && left >= kUnit) v.template load<ALIGN ? ALIGN : 16>(x);
    else if (ALIGN && left == kUnit / 2) {   // dim is an odd multiple of 16
      Block<T, kUnit / 2> b;
      b.template load<16>(x);
      v.clear();
#pragma unroll
      for (int j = 0; j < b.W; ++j) v.w[j] = b.w[j];
    } else v.gather(x, 0, min(left, kUnit), min(left, kUnit), nullptr, nullptr);
  }
  uint32_t m = v.max_bits();
  if (GRID != OCS_GRID_E8M0)
    for (int o = 1; o < (1 << gs_log2); o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  if (slot < 0 || left <= 0) return;
  if (m >= 0x7f800000u) flag(a.dev_status, OCS_DEV_NONFINITE);
  const long long page = (unsigned long long)slot >> 32 ? slot / a.page_size : (long long)((unsigned)slot / (unsigned)a.page_size);
  const long long at = (slot - page * a.page_size) * a.heads + h;
  uint8_t* base = a.pages[which] + page * a.g.bytes;
  float* row_scale = reinterpret_cast<float*>(base + a.g.at_r) + at;
  uint8_t* codes = base + at * a.g.cb;
  uint8_t* scales = base + a.g.at_s + at * a.g.sb;
  if constexpr (GRID == OCS_GRID_I8) {
    const float alpha = __uint_as_float(m);
    const RowGrid grid = row_grid(alpha, 127.0f);
    if (lane == 0) *row_scale = __fdiv_rn(alpha, 127.0f);
    uint32_t w[8];
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      int q[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) q[e] = row_code<true>(__fmul_rn(v[4 * j + e], grid.up), grid.inv);
      w[j] = pack4(q[0], q[1], q[2], q[3]);
    }
    *reinterpret_cast<uint4*>(codes + c) = make_uint4(w[0], w[1], w[2], w[3]);
    if (left > 16) *reinterpret_cast<uint4*>(codes + c + 16) = make_uint4(w[4], w[5], w[6], w[7]);
  } else {
    uint32_t w[4];
    if constexpr (GRID == OCS_GRID_E8M0) {
      const MxScale s = mx4_scale<GRID, T>(m, 0);
      v.template codes<GRID>(s, w);
      scales[lane] = (uint8_t)s.byte;
    } else {
      const int k = mx4_row_exponent(m);
      if (lane == 0) *row_scale = two_to(k);
      uint32_t byte[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        Block<T, 16> b;
#pragma unroll
        for (int j = 0; j < Block<T, 16>::W; ++j) b.w[j] = v.w[i * Block<T, 16>::W + j];
        const MxScale s = mx4_scale<GRID, T>(b.max_bits(), k);
        b.template codes<GRID>(s, w + 2 * i);
        byte[i] = s.byte;
      }
      if (left > 16) *reinterpret_cast<uint16_t*>(scales + 2 * lane) = (uint16_t)(byte[0] | byte[1] << 8);
      else scales[2 * lane] = (uint8_t)byte[0];
    }
    if (left > 16) *reinterpret_cast<uint4*>(codes + c / 2) = make_uint4(w[0], w[1], w[2], w[3]);
    else *reinterpret_cast<uint2*>(codes + c / 2) = make_uint2(w[0], w[1]);
  }
}

// Sequence of output row t: the b with starts[b] <= t < starts[b + 1] (-1: none).
__device__ __forceinline__ int sequence_of(const int32_t* starts, int B, long long t) {
  if (t < __ldg(starts) || t >= __ldg(starts + B)) return -1;
  int lo = 0, hi = B;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (__ldg(starts + mid) <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Most output rows of a CTA.  Vectors of few heads need many to occupy it.  Keys and values to bf16: 150 thousand tokens of 2 x 128
// 34.9 us from E4M3 (floor 30.5) and 40.4 from int8 (35.6), with at most 32 rows 37.4 and 43.7; 50 thousand of 1 x 64 from int8 7.0
// and 10.7 (3.0).
constexpr int kReadTokens = 128;

// Where a token's vectors are in its page (codes NULL: no such row; rows NULL: a bad page).
struct TokenAt {
  const uint8_t* codes;
  const uint8_t* scales;
  const float* rows;
};

template <typename T> constexpr int kReadUnit = 64 / (int)sizeof(T);

// `tokens` output rows per CTA; per = heads * units threads' worth of work each, units = ceil(dim / U), divided by as
// floor(x * inv_units / 2^32) where they are more than one (exact: x below 2^26, units at most 64).  A thread has U numbers of a
// vector: 64 bytes of output.
template <typename T, int GRID, int ALIGN>
__global__ void __launch_bounds__(256) cache_read_kernel(const CacheArgs a, int tokens, int units, uint32_t inv_units) {
  constexpr int U = kReadUnit<T>;
  __shared__ TokenAt s_at[kReadTokens];
  const long long t0 = (long long)blockIdx.x * tokens;
  const int which = blockIdx.y;
  if (threadIdx.x < tokens) {
    const long long t = t0 + threadIdx.x;
    TokenAt w{nullptr, nullptr, nullptr};
    const int b = t < a.rows ? sequence_of(a.starts, a.B, t) : -1;
    if (b >= 0) {
      const unsigned pos = (unsigned)t - (unsigned)__ldg(a.starts + b), col = pos / (unsigned)a.page_size;   // (starts may be negative)
      const int page = col < (unsigned)a.table_cols ? __ldg(a.table + b * a.ld_table + col) : -1;
      const uint8_t* base = a.pages[which];
      w.codes = base;
      if ((unsigned)page >= (unsigned)a.n_pages) flag(a.dev_status, OCS_DEV_BAD_INDEX);
      else {
        const long long at = (long long)(pos - col * (unsigned)a.page_size) * a.heads;
        base += page * a.g.bytes;
        w.codes = base + at * a.g.cb;
        w.scales = base + a.g.at_s + at * a.g.sb;
        w.rows = reinterpret_cast<const float*>(base + a.g.at_r) + at;
      }
    }
    s_at[threadIdx.x] = w;
  }
  __syncthreads();
  const int per = a.heads * units;
  const int step_tok = 256 / per, step_in = 256 - step_tok * per;
  int tok = (int)threadIdx.x / per, in = (int)threadIdx.x - tok * per;
  T* y0 = static_cast<T*>(a.x[which]) + t0 * a.ld_row[which];
#pragma unroll 2
  for (; tok < tokens; ) {
    const TokenAt w = s_at[tok];
    const int h = units == 1 ? in : (int)__umulhi((uint32_t)in, inv_units), u = in - h * units, c = u * U, left = a.dim - c;
    T* y = y0 + tok * a.ld_row[which] + h * a.ld_head[which] + c;
    tok += step_tok;
    in += step_in;
    if (in >= per) { in -= per; ++tok; }
    if (!w.codes) continue;
    T out[U];
    if (!w.rows) {
#pragma unroll
      for (int e = 0; e < U; ++e) out[e] = from_f32<T>(0.0f);
    } else if constexpr (GRID == OCS_GRID_I8) {
      const float step = __ldg(w.rows + h);
      const uint8_t* codes = w.codes + h * a.g.cb + c;
      const uint4 q0 = __ldg(reinterpret_cast<const uint4*>(codes));
      const uint4 q1 = U > 16 && left > 16 ? __ldg(reinterpret_cast<const uint4*>(codes) + 1) : make_uint4(0, 0, 0, 0);
      const uint32_t q[8] = {q0.x, q0.y, q0.z, q0.w, q1.x, q1.y, q1.z, q1.w};
#pragma unroll
      for (int e = 0; e < U; ++e) out[e] = from_f32<T>(__fmul_rn((float)(int8_t)(q[e / 4] >> (8 * (e & 3))), step));
    } else {
      const uint8_t* scales = w.scales + h * a.g.sb;
      const uint8_t* codes = w.codes + h * a.g.cb + c / 2;
      float unit[2];
      if (GRID == OCS_GRID_E8M0) unit[0] = unit[1] = e8m0_value(__ldg(scales + c / 32));
      else {
        const uint32_t s = U == 16 ? __ldg(scales + u) : __ldg(reinterpret_cast<const uint16_t*>(scales) + u);
        const float r = __ldg(w.rows + h);
        unit[0] = __fmul_rn(e4m3_value(s & 255u), r);
        unit[1] = __fmul_rn(e4m3_value(s >> 8), r);
      }
      uint32_t q[U / 8];
      if constexpr (U == 32) {
        const uint4 q4 = __ldg(reinterpret_cast<const uint4*>(codes));
        q[0] = q4.x; q[1] = q4.y; q[2] = q4.z; q[3] = q4.w;
      } else {
        const uint2 q2 = __ldg(reinterpret_cast<const uint2*>(codes));
        q[0] = q2.x; q[1] = q2.y;
      }
#pragma unroll
      for (int j = 0; j < U / 8; ++j) {
        __half2 v[4];
        e2m1_values(q[j], v);
        const unsigned long long uu = pack_f32x2(unit[j / 2], unit[j / 2]);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float2 f = __half22float2(v[e]);
          float v0, v1;
          unpack_f32x2(mul_f32x2(pack_f32x2(f.x, f.y), uu), v0, v1);
          out[8 * j + 2 * e] = from_f32<T>(v0);
          out[8 * j + 2 * e + 1] = from_f32<T>(v1);
        }
      }
    }
    const uint32_t* o = reinterpret_cast<const uint32_t*>(out);
    if (ALIGN && left >= U) {
      if constexpr (ALIGN == 32) {
#pragma unroll
        for (int j = 0; j < U * (int)sizeof(T) / 4; j += 8) store32(reinterpret_cast<uint32_t*>(y) + j, o + j);
      } else {
#pragma unroll
        for (int j = 0; j < U * (int)sizeof(T) / 16; ++j) reinterpret_cast<uint4*>(y)[j] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
      }
    } else if (ALIGN && U == 32 && left == 16) {   // half a unit: dim is an odd multiple of 16
#pragma unroll
      for (int j = 0; j < (int)sizeof(T); ++j) reinterpret_cast<uint4*>(y)[j] = make_uint4(o[4 * j], o[4 * j + 1], o[4 * j + 2], o[4 * j + 3]);
    } else {
#pragma unroll
      for (int e = 0; e < U; ++e)
        if (e < left) y[e] = out[e];
    }
  }
}

template <typename T, int GRID, int ALIGN>
ocs_status launch_write(const CacheArgs& a, int caches, cudaStream_t stream) {
  const int units = (a.dim + kUnit - 1) / kUnit;
  int gs = 0;
  while ((1 << gs) < units) ++gs;
  const long long ctas = (((a.rows * a.heads) << gs) + 255) / 256;
  if (ctas > 0x7fffffff) return OCS_ERR_UNSUPPORTED;
  LaunchScope ls("cache_write_kernel", stream);
  cache_write_kernel<T, GRID, ALIGN><<<dim3((unsigned)ctas, caches), 256, 0, stream>>>(a, gs);
  return launch_status();
}

template <typename T, int GRID, int ALIGN>
ocs_status launch_read(const CacheArgs& a, int caches, cudaStream_t stream) {
  constexpr int U = kReadUnit<T>;
  const int units = (a.dim + U - 1) / U, per = a.heads * units;
  // about four units per thread, while there are CTAs for all SMs
  int tokens = per < 1024 ? (1024 + per - 1) / per : 1;
  if (tokens > kReadTokens) tokens = kReadTokens;
  while (tokens > 1 && (a.rows + tokens - 1) / tokens * caches < 4 * kNumSMs) tokens = (tokens + 1) / 2;
  const long long ctas = (a.rows + tokens - 1) / tokens;
  if (ctas > 0x7fffffff) return OCS_ERR_UNSUPPORTED;
  LaunchScope ls("cache_read_kernel", stream);
  cache_read_kernel<T, GRID, ALIGN><<<dim3((unsigned)ctas, caches), 256, 0, stream>>>(a, tokens, units, units > 1 ? (uint32_t)((0xffffffffull + units) / units) : 0u);
  return launch_status();
}

template <bool WRITE, typename T, int GRID>
ocs_status dispatch_align(const CacheArgs& a, int align, int caches, cudaStream_t s) {
  switch (align) {
    case 32: return WRITE ? launch_write<T, GRID, 32>(a, caches, s) : launch_read<T, GRID, 32>(a, caches, s);
    case 16: return WRITE ? launch_write<T, GRID, 16>(a, caches, s) : launch_read<T, GRID, 16>(a, caches, s);
    default: return WRITE ? launch_write<T, GRID, 0>(a, caches, s) : launch_read<T, GRID, 0>(a, caches, s);
  }
}
template <bool WRITE, typename T>
ocs_status dispatch_grid(const CacheArgs& a, ocs_grid grid, int align, int caches, cudaStream_t s) {
  switch (grid) {
    case OCS_GRID_I8: return dispatch_align<WRITE, T, OCS_GRID_I8>(a, align, caches, s);
    case OCS_GRID_E8M0: return dispatch_align<WRITE, T, OCS_GRID_E8M0>(a, align, caches, s);
    default: return dispatch_align<WRITE, T, OCS_GRID_E4M3>(a, align, caches, s);
  }
}
template <bool WRITE>
ocs_status dispatch(const CacheArgs& a, ocs_grid grid, ocs_dtype type, int caches, cudaStream_t s) {
  uintptr_t al = 0;   // of every vector
  for (int i = 0; i < caches; ++i)
    al |= reinterpret_cast<uintptr_t>(a.x[i]) | (uintptr_t)(((a.rows > 1 ? a.ld_row[i] : 0) | (a.heads > 1 ? a.ld_head[i] : 0)) * elem_bytes(type));
  const int align = al % 32 == 0 ? 32 : (al % 16 == 0 ? 16 : 0);
  switch (type) {
    case OCS_F16: return dispatch_grid<WRITE, __half>(a, grid, align, caches, s);
    case OCS_BF16: return dispatch_grid<WRITE, __nv_bfloat16>(a, grid, align, caches, s);
    default: return dispatch_grid<WRITE, float>(a, grid, align, caches, s);
  }
}

bool valid_geometry(const ocs_cache* c) {
  return c->page_size > 0 && c->heads > 0 && c->dim > 0 && c->n_pages >= 0;
}

// What both calls ask of the cache and of the vectors outside of it.
ocs_status fill(CacheArgs& a, const ocs_cache* c, void* pages, void* pages2, int64_t rows, const void* x, int64_t ld_row,
                int64_t ld_head, const void* x2, int64_t ld_row2, int64_t ld_head2, ocs_dtype type) {
  if (c->dim > kMaxDim || (int64_t)c->page_size * c->heads >= (1 << 30) || (int64_t)c->heads * c->dim >= (1 << 26) || rows >= (1ll << 40))
    return OCS_ERR_UNSUPPORTED;
  if (!aligned(pages, 16) || !aligned(x, elem_bytes(type))) return OCS_ERR_SHAPE;
  if (pages2 && (!aligned(pages2, 16) || !aligned(x2, elem_bytes(type)))) return OCS_ERR_SHAPE;
  a.g = page_layout(c->page_size, c->heads, c->dim, c->grid);
  a.page_size = c->page_size; a.heads = c->heads; a.dim = c->dim; a.n_pages = c->n_pages;
  a.n_slots = (long long)c->n_pages * c->page_size;
  a.rows = rows;
  a.pages[0] = static_cast<uint8_t*>(pages); a.pages[1] = static_cast<uint8_t*>(pages2);
  a.x[0] = const_cast<void*>(x); a.x[1] = const_cast<void*>(x2);
  a.ld_row[0] = ld_row; a.ld_row[1] = pages2 ? ld_row2 : 0;
  a.ld_head[0] = ld_head; a.ld_head[1] = pages2 ? ld_head2 : 0;
  return OCS_OK;
}

// Whether no two of n0 x n1 vectors with these strides share an element: one stride goes over all vectors of the other.
bool nested(long long dim, long long n0, long long ld0, long long n1, long long ld1) {
  if ((n0 > 1 && ld0 < dim) || (n1 > 1 && ld1 < dim)) return false;
  return n0 <= 1 || n1 <= 1 || (ld0 - dim) / (n1 - 1) >= ld1 || (ld1 - dim) / (n0 - 1) >= ld0;
}

// Whether two outputs of the same strides, each of them nested and the second d elements behind the first, share an element: some
// |i| < outer count and |j| < inner count have |d - i outer stride - j inner stride| < dim.  Only the multiples of a stride on both
// sides of a distance come into question, since all inner vectors lie within one outer stride.  (Outputs of different strides
// are not looked at.)
bool on_each_other(const CacheArgs& a, long long d) {
  long long n0 = a.rows, ld0 = a.ld_row[0], n1 = a.heads, ld1 = a.ld_head[0];
  if ((n0 > 1 && ld0 != a.ld_row[1]) || (n1 > 1 && ld1 != a.ld_head[1])) return false;
  if (n0 > 1 && n1 > 1 && ld1 > ld0) {   // tokens inside of heads
    long long t = n0; n0 = n1; n1 = t;
    t = ld0; ld0 = ld1; ld1 = t;
  }
  if (d < 0) d = -d;
  if (n0 <= 1) ld0 = d + 1;              // (only i = 0 is within the bounds)
  if (n1 <= 1) ld1 = ld0;
  for (long long i = d / ld0; i <= d / ld0 + 1 && i < n0; ++i) {
    long long r = d - i * ld0;
    if (r < 0) r = -r;
    for (long long j = r / ld1; j <= r / ld1 + 1 && j < n1; ++j) {
      const long long off = r - j * ld1;
      if (off < a.dim && off > -a.dim) return true;
    }
  }
  return false;
}

}  // namespace
}  // namespace ocs

using namespace ocs;

extern "C" int64_t ocs_cache_page_bytes(const ocs_cache* c) {
  if (!c || !valid_geometry(c) || c->grid < OCS_GRID_I8 || c->grid > OCS_GRID_E4M3 || c->dim > kMaxDim ||
      (int64_t)c->page_size * c->heads >= (1 << 30))
    return 0;
  return page_layout(c->page_size, c->heads, c->dim, c->grid).bytes;
}

extern "C" ocs_status ocs_cache_write(const ocs_cache* c, void* pages, const void* X, int64_t ld_token, int64_t ld_head,
                                      void* pages2, const void* X2, int64_t ld_token2, int64_t ld_head2, ocs_dtype x_type,
                                      int64_t tokens, const int64_t* slots, int* dev_status, void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!c || !valid_dtype(x_type) || c->grid < OCS_GRID_I8 || c->grid > OCS_GRID_E4M3) return OCS_ERR_INVALID_ARG;
  if (!valid_geometry(c) || tokens < 0) return OCS_ERR_SHAPE;
  if (tokens == 0) return OCS_OK;
  if (!pages || !X || !slots || (!pages2) != (!X2)) return OCS_ERR_INVALID_ARG;
  if (pages2 == pages) return OCS_ERR_INVALID_ARG;
  CacheArgs a{};
  ocs_status st = fill(a, c, pages, pages2, tokens, X, ld_token, ld_head, X2, ld_token2, ld_head2, x_type);
  if (st != OCS_OK) return st;
  if (!aligned(slots, 8)) return OCS_ERR_SHAPE;
  if ((st = check_device()) != OCS_OK) return st;
  a.slots = slots; a.dev_status = dev_status;
  return dispatch<true>(a, c->grid, x_type, pages2 ? 2 : 1, stream);
}

extern "C" ocs_status ocs_cache_read(const ocs_cache* c, const void* pages, const void* pages2, const int32_t* table,
                                     int64_t ld_table, int table_cols, const int32_t* starts, int B, int64_t rows, void* Y,
                                     int64_t ld_token, int64_t ld_head, void* Y2, int64_t ld_token2, int64_t ld_head2,
                                     ocs_dtype y_type, int* dev_status, void* stream_) {
  cudaStream_t stream = reinterpret_cast<cudaStream_t>(stream_);
  if (!c || !valid_dtype(y_type) || c->grid < OCS_GRID_I8 || c->grid > OCS_GRID_E4M3) return OCS_ERR_INVALID_ARG;
  if (!valid_geometry(c) || rows < 0 || B < 0 || table_cols < 0) return OCS_ERR_SHAPE;
  if (rows == 0 || B == 0) return OCS_OK;
  if (!pages || (!table && table_cols) || !starts || !Y || (!pages2) != (!Y2)) return OCS_ERR_INVALID_ARG;   // (a table of no columns has no address)
  CacheArgs a{};
  ocs_status st = fill(a, c, const_cast<void*>(pages), const_cast<void*>(pages2), rows, Y, ld_token, ld_head, Y2, ld_token2, ld_head2, y_type);
  if (st != OCS_OK) return st;
  if (pages2 && Y2 == Y) return OCS_ERR_INVALID_ARG;
  for (int i = 0; i < (pages2 ? 2 : 1); ++i)
    if (!nested(c->dim, rows, a.ld_row[i], c->heads, a.ld_head[i])) return OCS_ERR_SHAPE;
  if (pages2 && on_each_other(a, (reinterpret_cast<intptr_t>(Y2) - reinterpret_cast<intptr_t>(Y)) / elem_bytes(y_type))) return OCS_ERR_SHAPE;
  if (ld_table < table_cols || !aligned(table, 4) || !aligned(starts, 4)) return OCS_ERR_SHAPE;
  if ((st = check_device()) != OCS_OK) return st;
  a.table = table; a.ld_table = ld_table; a.table_cols = table_cols; a.starts = starts; a.B = B; a.dev_status = dev_status;
  return dispatch<false>(a, c->grid, y_type, pages2 ? 2 : 1, stream);
}
