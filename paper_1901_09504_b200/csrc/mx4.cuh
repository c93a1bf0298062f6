// The block-scaled grids: e2m1 codes (0, .5, 1, 1.5, 2, 3, 4, 6 and their negatives) in halves of bytes, and their scales.
//   OCS_GRID_E8M0: blocks of 32, scale 2^(floor(log2 max|x|) - 2)                        (one byte: the exponent + 127)
//   OCS_GRID_E4M3: blocks of 16, scale e4m3(max|x| / r / 6) * r, r a power of two per row  (one byte, and r as fp32)
// A code is the grid point nearest to x / scale, ties to even, saturating at 6.
#pragma once

#include <type_traits>

#include "elem.cuh"
#include "ptx.cuh"

namespace ocs {

constexpr int kMxTile = 512;   // scale bytes of 128 rows x 4 blocks, the tensor cores' unit
constexpr int kMxMaxK = 1 << 27;   // channels of a row (the grids' second dimension ends at 65535)

inline bool mx4_grid(ocs_grid g) { return g == OCS_GRID_E8M0 || g == OCS_GRID_E4M3; }
__host__ __device__ constexpr int mx4_block(int grid) { return grid == OCS_GRID_E8M0 ? 32 : 16; }

// Byte of block b of row r among the scales of a matrix with `chunks` groups of four blocks: tiles of 128 rows, in them one
// 512-byte piece per group, in that [row % 32][row / 32 % 4][block % 4] -- what tcgen05.cp moves to tensor memory as it is.
__host__ __device__ __forceinline__ long long mx4_scale_at(long long r, int b, int chunks) {
  return ((r >> 7) * chunks + (b >> 2)) * kMxTile + (r & 31) * 16 + ((r >> 5) & 3) * 4 + (b & 3);
}

// Eight values as codes, the first in the lowest four bits.
__device__ __forceinline__ uint32_t e2m1_codes(const float* t) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r) : "f"(t[0]), "f"(t[1]), "f"(t[2]), "f"(t[3]), "f"(t[4]), "f"(t[5]), "f"(t[6]), "f"(t[7]));
  return r;
}
// Four bytes of codes as eight values, in four pairs of halves (exact).
__device__ __forceinline__ void e2m1_values(uint32_t codes, __half2* v) {
  uint32_t r[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(codes));
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = *reinterpret_cast<__half2*>(&r[i]);
}
__device__ __forceinline__ uint32_t e4m3_byte(float v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(v));
  return r;
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)byte));
  return __half2float(__ushort_as_half((unsigned short)r));
}
// 2^(byte - 127), and its reciprocal for bytes below 255
__device__ __forceinline__ float e8m0_value(uint32_t byte) {
  return __uint_as_float(byte == 255 ? 0x7fffffffu : (byte ? byte << 23 : 0x00400000u));
}
__device__ __forceinline__ float e8m0_inverse(uint32_t byte) { return __uint_as_float((254u - byte) << 23); }

// Exponent of a row's scale: the smallest k in [-117, 117] with alpha <= 6 * 448 * 2^k (6 * 448 = 1.3125 * 2^11).  Within
// these bounds a block's unit (2^-9 to 448 times 2^k) and its reciprocal are normal numbers.
__device__ __forceinline__ int mx4_row_exponent(uint32_t max_bits) {
  const int k = (int)(max_bits >> 23) - 127 - 11 + ((max_bits & 0x7fffffu) > 0x280000u ? 1 : 0);
  return max(-117, min(117, k));
}
__device__ __forceinline__ float two_to(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// A block's scale from the bits of its largest magnitude: the stored byte, and what takes a value to code units: the factor
// inv; E4M3 with fp32 values: the exact factor `down` to the row's units, the scale u there and its reciprocal.
// k: the row's exponent (E4M3).
struct MxScale {
  uint32_t byte;
  float inv, down, u;
};
template <int GRID, typename T>
__device__ __forceinline__ MxScale mx4_scale(uint32_t max_bits, int k) {
  MxScale s;
  if constexpr (GRID == OCS_GRID_E8M0) {
    s.byte = (uint32_t)max((int)(min(max_bits, 0x7f7fffffu) >> 23) - 2, 0);
    s.inv = e8m0_inverse(s.byte);
  } else {
    s.down = two_to(-k);
    // the quotient by 6, rounded once (by the correction that is explained below)
    const float a = __fmul_rn(__uint_as_float(max_bits), s.down), sixth = 1.0f / 6.0f, t = __fmul_rn(a, sixth);
    s.byte = e4m3_byte(fmaf(fmaf(-t, 6.0f, a), sixth, t));
    s.u = e4m3_value(s.byte);
    if constexpr (sizeof(T) == 2) {
      float y;   // (an approximation will do)
      asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(s.u));
      s.inv = s.byte ? __fmul_rn(y, s.down) : 0.0f;
    } else {
      s.inv = s.byte ? __frcp_rn(s.u) : 0.0f;
    }
  }
  return s;
}

__device__ __forceinline__ unsigned long long mul_f32x2(unsigned long long a, unsigned long long b) {
  unsigned long long r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
// Two values in units of the block's scale, as the rounding to e2m1 needs them.  E8M0: exact.
// E4M3 with 16-bit x: a value x / unit is either a border between two codes or at least 2^-13 away from each (x has at most
// 11 bits, a border times the unit at most 7), so that the product with the approximate reciprocal, rounded to multiples of
// 2^-14, falls on the right side and borders on themselves: a fused multiply-add and a subtraction instead of a division.
// E4M3 with fp32 x: the rounded quotient, by Markstein's correction.  With z = x / r (exact), u = unit / r (an e4m3 number: 4
// bits), y = rn(1 / u) and t = rn(z y), which is within two units of the quotient, z - t u has at most 6 bits and one
// fused multiply-add finds it exactly; t + (z - t u) y is then the quotient up to 2^-22 units in the last place, and rounds
// as the quotient does, since that (24 bits over 4) is never within 1/30 unit of the middle between two numbers unless it is
// one of them.  (Values z below 2^-100 may lose bits on the way; their code is 0 either way.)
// Zeros keep x's sign.
template <int GRID, typename T>
__device__ __forceinline__ void mx4_units(float x0, float x1, const MxScale& s, float* t) {
  const unsigned long long x = pack_f32x2(x0, x1), inv = pack_f32x2(s.inv, s.inv);
  if constexpr (GRID == OCS_GRID_E8M0) {
    unpack_f32x2(mul_f32x2(x, inv), t[0], t[1]);
  } else {
    if constexpr (sizeof(T) == 2) {
      const unsigned long long c = pack_f32x2(768.0f, 768.0f);
      unpack_f32x2(sub_f32x2(fma_f32x2(x, inv, c), c), t[0], t[1]);
    } else {
      const unsigned long long z = mul_f32x2(x, pack_f32x2(s.down, s.down)), q = mul_f32x2(z, inv);
      const unsigned long long rest = fma_f32x2(q, pack_f32x2(-s.u, -s.u), z);
      unpack_f32x2(fma_f32x2(rest, inv, q), t[0], t[1]);
    }
    t[0] = copysignf(t[0], x0);
    t[1] = copysignf(t[1], x1);
  }
}

__device__ __forceinline__ void store32(uint32_t* dst, const uint32_t* v) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(dst), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]) : "memory");
}

// N consecutive elements of a row in registers.
template <typename T, int N>
struct Block {
  static constexpr int W = N * (int)sizeof(T) / 4;
  uint32_t w[W];
  // x aligned to ALIGN bytes: 32, 16, or (0) its element.  The last reads the 16-byte pieces around the block and shifts it out of
  // them: up to 15 bytes before x and 16 behind the block have to be readable.  (32 bytes at an 8-byte boundary come in four
  // loads instead: 13152 x 1334 fp32 27.5 us against 30.3; 64 bytes, or eight loads of 4 bytes, are slower that way.)
  template <int ALIGN>
  __device__ __forceinline__ void load(const T* x) {
    if constexpr (ALIGN == 32) {
#pragma unroll
      for (int i = 0; i < W; i += 8)
        asm volatile("ld.global.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                     : "=r"(w[i]), "=r"(w[i + 1]), "=r"(w[i + 2]), "=r"(w[i + 3]), "=r"(w[i + 4]), "=r"(w[i + 5]), "=r"(w[i + 6]), "=r"(w[i + 7])
                     : "l"(reinterpret_cast<const uint32_t*>(x) + i));
    } else if constexpr (ALIGN == 16) {
#pragma unroll
      for (int i = 0; i < W; i += 4) {
        const uint4 v = __ldg(reinterpret_cast<const uint4*>(x) + i / 4);
        w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
      }
    } else if (W == 8 && reinterpret_cast<uintptr_t>(x) % 8 == 0) {
#pragma unroll
      for (int i = 0; i < W; i += 2) {
        const uint2 v = __ldg(reinterpret_cast<const uint2*>(x) + i / 2);
        w[i] = v.x; w[i + 1] = v.y;
      }
    } else {
      const uintptr_t at = reinterpret_cast<uintptr_t>(x);
      const uint4* c = reinterpret_cast<const uint4*>(at & ~(uintptr_t)15);
      uint32_t u[W + 4];
#pragma unroll
      for (int i = 0; i < W + 4; i += 4) {
        const uint4 v = __ldg(c + i / 4);
        u[i] = v.x; u[i + 1] = v.y; u[i + 2] = v.z; u[i + 3] = v.w;
      }
      if (at & 8) {
#pragma unroll
        for (int i = 0; i < W + 2; ++i) u[i] = u[i + 2];
      }
      if (at & 4) {
#pragma unroll
        for (int i = 0; i < W + 1; ++i) u[i] = u[i + 1];
      }
      const uint32_t sel = sizeof(T) == 2 && (at & 2) ? 0x5432u : 0x3210u;
#pragma unroll
      for (int i = 0; i < W; ++i) w[i] = sizeof(T) == 2 ? __byte_perm(u[i], u[i + 1], sel) : u[i];
    }
  }
  // Elements c, c + 1, ... of the expanded row: the row's C own, then its duplicated channels up to K, then zeros.  All
  // indices of R elements are asked for before the first value, and all values before the first is used.  (Row quantization with its
  // 40 registers a thread: 16 of 32 elements at a time spill 112 to 128 bytes, 8 of them 16 to 20: 2047 x 4096 with 82 duplicated
  // channels, bf16 E8M0, 6.1 and 5.7 us.  The cache's writing is 4 to 8 % slower on int8 with 8.)
  template <int R = (N < 16 ? N : 16)>
  __device__ __forceinline__ void gather(const T* x, int c, int C, int K, const int32_t* idx_map, int* dev_status) {
#pragma unroll
    for (int h = 0; h < N; h += R) {
      int src[R];
#pragma unroll
      for (int e = 0; e < R; ++e) {
        const int i = c + h + e;
        src[e] = i;
        if (i >= C && i < K) src[e] = __ldg(idx_map + i);
      }
      bool bad = false;
#pragma unroll
      for (int e = 0; e < R; ++e)
        if (c + h + e < K && (unsigned)src[e] >= (unsigned)C) { bad = true; src[e] = 0; }
      uint32_t v[R];
#pragma unroll
      for (int e = 0; e < R; ++e) {
        v[e] = 0;
        if (c + h + e < K) {
          if constexpr (sizeof(T) == 4) v[e] = __ldg(reinterpret_cast<const uint32_t*>(x) + src[e]);
          else v[e] = __ldg(reinterpret_cast<const uint16_t*>(x) + src[e]);
        }
      }
#pragma unroll
      for (int e = 0; e < R; ++e) {
        if constexpr (sizeof(T) == 4) w[h + e] = v[e];
        else if (e & 1) w[(h + e) / 2] = v[e - 1] | v[e] << 16;
      }
      if (bad) flag(dev_status, OCS_DEV_BAD_INDEX);
    }
  }
  // N elements from shared memory.
  __device__ __forceinline__ void from_shared(const T* s) {
#pragma unroll
    for (int i = 0; i < W; i += 4) {
      const uint4 v = *(reinterpret_cast<const uint4*>(s) + i / 4);
      w[i] = v.x; w[i + 1] = v.y; w[i + 2] = v.z; w[i + 3] = v.w;
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < W; ++i) w[i] = 0;
  }
  __device__ __forceinline__ float operator[](int e) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[e]);
    else if constexpr (std::is_same<T, __nv_bfloat16>::value) return __uint_as_float(e & 1 ? w[e / 2] & 0xffff0000u : w[e / 2] << 16);
    else return __half2float(__ushort_as_half((unsigned short)(e & 1 ? w[e / 2] >> 16 : w[e / 2] & 0xffffu)));
  }
  // Bits of the largest magnitude as fp32 (magnitudes order like their bits, and so does what is not finite).
  __device__ __forceinline__ uint32_t max_bits() const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) {
      if constexpr (sizeof(T) == 4) m = max(m, w[i] & 0x7fffffffu);
      else asm("max.u16x2 %0, %0, %1;" : "+r"(m) : "r"(w[i] & 0x7fff7fffu));
    }
    if constexpr (sizeof(T) == 4) return m;
    const uint32_t h = max(m & 0xffffu, m >> 16);
    if constexpr (std::is_same<T, __nv_bfloat16>::value) return h << 16;
    else return __float_as_uint(__half2float(__ushort_as_half((unsigned short)h)));
  }
  template <int GRID>
  __device__ __forceinline__ void codes(const MxScale& s, uint32_t* out) const {
#pragma unroll
    for (int i = 0; i < N / 8; ++i) {
      float t[8];
#pragma unroll
      for (int e = 0; e < 8; e += 2) mx4_units<GRID, T>((*this)[8 * i + e], (*this)[8 * i + e + 1], s, t + e);
      out[i] = e2m1_codes(t);
    }
  }
};

}  // namespace ocs
