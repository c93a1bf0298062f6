// ocs_cache_write / ocs_cache_read: a paged cache of keys and values that is quantized as it is written.
// A page holds page_size tokens x heads vectors: first all their codes, then their block scales, then their row scales, so
// that every section is dense and a page moves as one run of bytes.  Four lanes' worth of arithmetic per 64 bytes: memory
// bounds both directions.
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

constexpr int kUnit = 16;           // elements of a vector that a lane has at a time
constexpr int kMaxDim = 1024;

// N = 16 elements at x, of which `left` exist (zeros behind them)
template <typename T>
__device__ __forceinline__ void load_unit(Block<T, kUnit>& v, const T* x, int left, bool wide) {
  if (wide && left >= kUnit) v.template load<16>(x);
  else v.gather(x, 0, min(left, kUnit), min(left, kUnit), nullptr, nullptr);
}

// A group of GS lanes (a power of two, at least 2) per vector, U units of 16 elements per lane, consecutive.
template <typename T, int GRID, int U>
__global__ void __launch_bounds__(256) cache_write_kernel(const CacheArgs a, int gs_log2, int wide) {
  const long long g = (long long)blockIdx.x * 256 + threadIdx.x;
  const int lane = (int)(g & ((1 << gs_log2) - 1)), which = blockIdx.y;
  const long long vec = g >> gs_log2, t = vec / a.heads;
  const int h = (int)(vec - t * a.heads);
  long long slot = -1;
  if (t < a.rows) {
    slot = __ldg(a.slots + t);
    if (slot >= a.n_slots) { if (lane == 0) flag(a.dev_status, OCS_DEV_BAD_INDEX); slot = -1; }
  }
  Block<T, kUnit> v[U];
  uint32_t mine[U], m = 0;
#pragma unroll
  for (int i = 0; i < U; ++i) {
    const int c = (lane * U + i) * kUnit;
    if (slot >= 0 && c < a.dim)
      load_unit<T>(v[i], static_cast<const T*>(a.x[which]) + t * a.ld_row[which] + h * a.ld_head[which] + c, a.dim - c, wide);
    else v[i].clear();
    mine[i] = v[i].max_bits();
    m = max(m, mine[i]);
  }
  if (GRID == OCS_GRID_E8M0) {
    // blocks of two units: a lane's own two, or a pair of lanes
    if (U == 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, 1));
  } else {
    for (int o = 1; o < (1 << gs_log2); o <<= 1) m = max(m, __shfl_xor_sync(0xffffffffu, m, o));
  }
  if (slot < 0) return;
  if (m >= 0x7f800000u) flag(a.dev_status, OCS_DEV_NONFINITE);
  const long long page = slot / a.page_size;
  const long long at = (slot - page * a.page_size) * a.heads + h;
  uint8_t* base = a.pages[which] + page * a.g.bytes;
  float* row_scale = reinterpret_cast<float*>(base + a.g.at_r) + at;
  uint8_t* codes = base + at * a.g.cb;
  uint8_t* scales = base + a.g.at_s + at * a.g.sb;
  if constexpr (GRID == OCS_GRID_I8) {
    const float alpha = __uint_as_float(m);
    const RowGrid grid = row_grid(alpha, 127.0f);
    if (lane == 0) *row_scale = __fdiv_rn(alpha, 127.0f);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int c = (lane * U + i) * kUnit;
      if (c >= a.dim) break;
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        int q[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) q[e] = row_code<true>(__fmul_rn(v[i][4 * j + e], grid.up), grid.inv);
        w[j] = pack4(q[0], q[1], q[2], q[3]);
      }
      *reinterpret_cast<uint4*>(codes + c) = make_uint4(w[0], w[1], w[2], w[3]);
    }
  } else {
    const int k = GRID == OCS_GRID_E4M3 ? mx4_row_exponent(m) : 0;
    if (GRID == OCS_GRID_E4M3 && lane == 0) *row_scale = two_to(k);
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int c = (lane * U + i) * kUnit;
      if (c >= a.dim) break;
      const uint32_t mb = GRID == OCS_GRID_E8M0 ? m : mine[i];
      const MxScale s = mx4_scale<GRID, T>(mb, k);
      uint32_t w[2];
      v[i].template codes<GRID>(s, w);
      *reinterpret_cast<uint2*>(codes + c / 2) = make_uint2(w[0], w[1]);
      if (GRID == OCS_GRID_E4M3) scales[c / 16] = (uint8_t)s.byte;
      else if (c % 32 == 0) scales[c / 32] = (uint8_t)s.byte;
    }
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

constexpr int kReadTokens = 16;     // output rows of a CTA

template <typename T, int GRID>
__global__ void __launch_bounds__(256) cache_read_kernel(const CacheArgs a, int units, int wide) {
  __shared__ long long s_page[kReadTokens], s_at[kReadTokens];   // page (-1: no such row, -2: a bad page), vector in it
  const long long t0 = (long long)blockIdx.x * kReadTokens;
  const int which = blockIdx.y;
  if (threadIdx.x < kReadTokens) {
    const long long t = t0 + threadIdx.x;
    long long page = -1, at = 0;
    const int b = t < a.rows ? sequence_of(a.starts, a.B, t) : -1;
    if (b >= 0) {
      const long long pos = t - __ldg(a.starts + b), col = pos / a.page_size;
      page = col < a.table_cols ? __ldg(a.table + b * a.ld_table + col) : -2;
      if (page < 0 || page >= a.n_pages) { flag(a.dev_status, OCS_DEV_BAD_INDEX); page = -2; }
      at = (pos - col * a.page_size) * a.heads;
    }
    s_page[threadIdx.x] = page;
    s_at[threadIdx.x] = at;
  }
  __syncthreads();
  const int per = a.heads * units, total = kReadTokens * per;
  for (int i = threadIdx.x; i < total; i += 256) {
    const int tok = i / per, in = i - tok * per, h = in / units, u = in - h * units;
    const long long page = s_page[tok];
    if (page == -1) continue;
    const int c = u * kUnit, left = a.dim - c;
    T out[kUnit];
    if (page < 0) {
#pragma unroll
      for (int e = 0; e < kUnit; ++e) out[e] = from_f32<T>(0.0f);
    } else {
      const uint8_t* base = a.pages[which] + page * a.g.bytes;
      const long long at = s_at[tok] + h;
      const uint8_t* codes = base + at * a.g.cb;
      if constexpr (GRID == OCS_GRID_I8) {
        const float step = __ldg(reinterpret_cast<const float*>(base + a.g.at_r) + at);
        const uint4 q = __ldg(reinterpret_cast<const uint4*>(codes + c));
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
        for (int e = 0; e < kUnit; ++e) out[e] = from_f32<T>(__fmul_rn((float)(int8_t)(w[e / 4] >> (8 * (e & 3))), step));
      } else {
        const uint8_t* scales = base + a.g.at_s + at * a.g.sb;
        float unit;
        if (GRID == OCS_GRID_E8M0) unit = e8m0_value(__ldg(scales + c / 32));
        else unit = __fmul_rn(e4m3_value(__ldg(scales + c / 16)), __ldg(reinterpret_cast<const float*>(base + a.g.at_r) + at));
        const uint2 q = __ldg(reinterpret_cast<const uint2*>(codes + c / 2));
        const uint32_t w[2] = {q.x, q.y};
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          __half2 v[4];
          e2m1_values(w[j], v);
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 f = __half22float2(v[e]);
            out[8 * j + 2 * e] = from_f32<T>(__fmul_rn(f.x, unit));
            out[8 * j + 2 * e + 1] = from_f32<T>(__fmul_rn(f.y, unit));
          }
        }
      }
    }
    T* y = static_cast<T*>(a.x[which]) + (t0 + tok) * a.ld_row[which] + h * a.ld_head[which] + c;
    if (wide && left >= kUnit) {
#pragma unroll
      for (int j = 0; j < (int)sizeof(T); ++j) reinterpret_cast<uint4*>(y)[j] = reinterpret_cast<uint4*>(out)[j];
    } else {
#pragma unroll
      for (int e = 0; e < kUnit; ++e)
        if (e < left) y[e] = out[e];
    }
  }
}

template <typename T, int GRID>
ocs_status launch_write(const CacheArgs& a, int caches, int wide, cudaStream_t stream) {
  const int units = (a.dim + kUnit - 1) / kUnit, U = units > 32 ? 2 : 1, lanes = (units + U - 1) / U;
  int gs = 1;
  while ((1 << gs) < lanes) ++gs;
  const long long ctas = (((a.rows * a.heads) << gs) + 255) / 256;
  if (ctas > 0x7fffffff) return OCS_ERR_UNSUPPORTED;
  LaunchScope ls("cache_write_kernel", stream);
  if (U == 1) cache_write_kernel<T, GRID, 1><<<dim3((unsigned)ctas, caches), 256, 0, stream>>>(a, gs, wide);
  else cache_write_kernel<T, GRID, 2><<<dim3((unsigned)ctas, caches), 256, 0, stream>>>(a, gs, wide);
  return launch_status();
}

template <typename T, int GRID>
ocs_status launch_read(const CacheArgs& a, int caches, int wide, cudaStream_t stream) {
  const long long ctas = (a.rows + kReadTokens - 1) / kReadTokens;
  if (ctas > 0x7fffffff) return OCS_ERR_UNSUPPORTED;
  LaunchScope ls("cache_read_kernel", stream);
  cache_read_kernel<T, GRID><<<dim3((unsigned)ctas, caches), 256, 0, stream>>>(a, (a.dim + kUnit - 1) / kUnit, wide);
  return launch_status();
}

template <bool WRITE, typename T>
ocs_status dispatch_grid(const CacheArgs& a, ocs_grid grid, int caches, int wide, cudaStream_t s) {
  switch (grid) {
    case OCS_GRID_I8: return WRITE ? launch_write<T, OCS_GRID_I8>(a, caches, wide, s) : launch_read<T, OCS_GRID_I8>(a, caches, wide, s);
    case OCS_GRID_E8M0: return WRITE ? launch_write<T, OCS_GRID_E8M0>(a, caches, wide, s) : launch_read<T, OCS_GRID_E8M0>(a, caches, wide, s);
    default: return WRITE ? launch_write<T, OCS_GRID_E4M3>(a, caches, wide, s) : launch_read<T, OCS_GRID_E4M3>(a, caches, wide, s);
  }
}
template <bool WRITE>
ocs_status dispatch(const CacheArgs& a, ocs_grid grid, ocs_dtype type, int caches, cudaStream_t s) {
  uintptr_t al = 0;   // of every vector
  for (int i = 0; i < caches; ++i)
    al |= reinterpret_cast<uintptr_t>(a.x[i]) | (uintptr_t)((a.ld_row[i] | a.ld_head[i]) * elem_bytes(type));
  const int wide = al % 16 == 0;
  switch (type) {
    case OCS_F16: return dispatch_grid<WRITE, __half>(a, grid, caches, wide, s);
    case OCS_BF16: return dispatch_grid<WRITE, __nv_bfloat16>(a, grid, caches, wide, s);
    default: return dispatch_grid<WRITE, float>(a, grid, caches, wide, s);
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
  if (!pages || !table || !starts || !Y || (!pages2) != (!Y2)) return OCS_ERR_INVALID_ARG;
  CacheArgs a{};
  ocs_status st = fill(a, c, const_cast<void*>(pages), const_cast<void*>(pages2), rows, Y, ld_token, ld_head, Y2, ld_token2, ld_head2, y_type);
  if (st != OCS_OK) return st;
  // the output's vectors must not overlap
  for (int i = 0; i < (pages2 ? 2 : 1); ++i)
    if ((c->heads > 1 && a.ld_head[i] < c->dim) || (rows > 1 && a.ld_row[i] < c->dim)) return OCS_ERR_SHAPE;
  if (ld_table < table_cols || !aligned(table, 4) || !aligned(starts, 4)) return OCS_ERR_SHAPE;
  if ((st = check_device()) != OCS_OK) return st;
  a.table = table; a.ld_table = ld_table; a.table_cols = table_cols; a.starts = starts; a.B = B; a.dev_status = dev_status;
  return dispatch<false>(a, c->grid, y_type, pages2 ? 2 : 1, stream);
}
