// 4-bit floats with a scale per 16 columns and one per row: the byte order of packed rows.
#pragma once

#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "lowbit.cuh"

namespace ssd {

// A record is 128 rows x 256 columns.  Codes: 128 bytes a row, a column's code in the low nibble of its byte where the
// column is even, the row's eight 16-byte units in the order of the 128-byte swizzle (unit ^ row % 8), so that a copy
// of the bytes is an operand of tcgen05.mma.  Scales: e4m3, 512 bytes per 64 columns, row r's four at
// (r % 32) * 16 + r / 32 * 4: 32 lanes of four words, as tensor memory holds the scales of 128 rows.
constexpr int kF4Rows = 128, kF4Cols = 256, kF4Group = 16;
constexpr int kF4CodeBytes = kF4Rows * kF4Cols / 2, kF4Record = kF4CodeBytes + kF4Rows * kF4Cols / kF4Group;

__host__ __device__ __forceinline__ int f4_chunks(int k) { return (k + kF4Cols - 1) / kF4Cols; }
__host__ __device__ __forceinline__ int64_t f4_scales_at(int rows, int k) {  // byte of the row scales
  return static_cast<int64_t>((rows + kF4Rows - 1) / kF4Rows) * f4_chunks(k) * kF4Record;
}
// Byte of 16 columns' codes (8 bytes' aligned half of a unit) and of a group's scale in a record.
__host__ __device__ __forceinline__ int f4_code_byte(int row, int col) {
  return row * 128 + (((col >> 5) ^ (row & 7)) << 4) + (col >> 1 & 15);
}
__host__ __device__ __forceinline__ int f4_scale_byte(int row, int col) {
  return kF4CodeBytes + (col >> 6) * 512 + (row & 31) * 16 + (row >> 5) * 4 + (col >> 4 & 3);
}

// ------------------------------------------------------------------ packing

// Eight neighbouring columns as they lie in memory: fp32 numbers, or pairs of bf16.
template <typename T>
struct Raw8 {
  uint32_t w[2 * sizeof(T)];

  // From `col` on, zeros past k.  VEC: 16-byte aligned.  Else the 16-byte pieces that hold the columns are read, where
  // they lie within the row, and moved into place (a row's lanes are all off by as much); the columns at a row's ends
  // and those of short rows, which are mostly ends, are read one by one (9000 x 14335 bf16, packed and read back: 310 us with
  // all of them so, and with lanes' own stores, 242 now: 135 and 107.  fp32 311: 202 and 107).
  template <bool VEC>
  __device__ __forceinline__ void load(const T* p, int col, int k) {
    if (VEC && col + 8 <= k) {
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i)
        reinterpret_cast<uint4*>(w)[i] = reinterpret_cast<const uint4*>(p + col)[i];
      return;
    }
    constexpr int kWords = 2 * sizeof(T);
    const int off = static_cast<int>(reinterpret_cast<uintptr_t>(p + col) & 15), at = col * static_cast<int>(sizeof(T)) - off;
    if (!VEC && k >= 512 && at >= 0 && at + 4 * kWords + 16 <= k * static_cast<int>(sizeof(T))) {
      const uint4* in = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(p) + at);
      uint4 v[kWords / 4 + 1];
#pragma unroll
      for (int i = 0; i <= kWords / 4; ++i) v[i] = in[i];
      uint32_t* u = reinterpret_cast<uint32_t*>(v);
#pragma unroll
      for (int i = 0; i < kWords + 3; ++i) u[i] = off & 4 ? u[i + 1] : u[i];
#pragma unroll
      for (int i = 0; i < kWords + 1; ++i) u[i] = off & 8 ? u[i + 2] : u[i];
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = sizeof(T) == 4 ? u[i] : __funnelshift_r(u[i], u[i + 1], 8 * (off & 2));
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if constexpr (sizeof(T) == 4) {
          w[i] = col + i < k ? __float_as_uint(p[col + i]) : 0u;
        } else {
          const uint32_t v = col + i < k ? __bfloat16_as_ushort(p[col + i]) : 0u;
          w[i / 2] = i & 1 ? w[i / 2] | v << 16 : v;
        }
      }
    }
  }
  // The largest magnitude's bits as those of a float: a NaN is above infinity, infinity above the rest.
  __device__ __forceinline__ uint32_t amax() const {
    if constexpr (sizeof(T) == 4) {
      uint32_t m = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) m = max(m, w[i] & 0x7fffffffu);
      return m;
    } else {
      uint32_t m = 0;  // of the even and the odd columns
#pragma unroll
      for (int i = 0; i < 4; ++i) m = __vmaxu2(m, w[i] & 0x7fff7fffu);
      return max(m << 16, m & 0xffff0000u);
    }
  }
  __device__ __forceinline__ float2 pair(int i) const {
    if constexpr (sizeof(T) == 4) return make_float2(__uint_as_float(w[2 * i]), __uint_as_float(w[2 * i + 1]));
    return bf16x2_to_float2(w[i]);
  }
};

__device__ __forceinline__ float e4m3_value(uint32_t byte) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(byte), __NV_E4M3)));
}

// A row's scale from the bits of its largest magnitude: the exponent of the smallest 2^e with amax <= 2688 2^e
// (2688 = 1.3125 * 2^11), at least -100.
__device__ __forceinline__ int f4_row_exponent(uint32_t amax) {
  return max(static_cast<int>(amax >> 23) - 127 - 11 + ((amax & 0x7fffffu) > 0x280000u ? 1 : 0), -100);
}

// Four pairs to a word of codes, to nearest even, at most 6.
__device__ __forceinline__ uint32_t to_e2m1(const float2* q) {
  uint32_t w;
  asm("{\n .reg .b8 a, b, c, d;\n"
      " cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n mov.b32 %0, {a, b, c, d};\n}"
      : "=r"(w)
      : "f"(q[0].x), "f"(q[0].y), "f"(q[1].x), "f"(q[1].y), "f"(q[2].x), "f"(q[2].y), "f"(q[3].x), "f"(q[3].y));
  return w;
}
__device__ __forceinline__ float approx_reciprocal(float v) {
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v));
  return r;
}

// One row's 16-column group, half of it (8 columns, largest magnitude `bits`) in this lane and half in lane ^ 1, times the
// row's down = 2^-e: the scale's byte and the 8 codes.  A quotient is fma(y, h, y * l) of its divisor's reciprocal h + l,
// exact to 2^-45, and so correctly rounded: numerators have 24 bits and divisors (6, s) at most 4, so no quotient lies
// nearer than 2^-30 to the middle of two fp32 numbers.
template <typename T>
__device__ __forceinline__ void f4_encode(const Raw8<T>& x, uint32_t bits, float down, uint32_t& scale, uint32_t& codes) {
  bits = max(bits, __shfl_xor_sync(~0u, bits, 1));
  constexpr float kSixth = 1.0f / 6.0f, kSixthLow = static_cast<float>(1.0 / 6.0 - static_cast<double>(kSixth));
  const float m = __uint_as_float(bits) * down;
  scale = __nv_cvt_float_to_fp8(fmaf(m, kSixth, m * kSixthLow), __NV_SATFINITE, __NV_E4M3);
  const float s = e4m3_value(scale);
  float h = approx_reciprocal(s), l = fmaf(-s, h, 1.0f) * h;
  if (scale == 0) h = l = 0.0f;
  float2 q[4];
  // the row's power of two goes into the reciprocal, but where that would push its low part out of range
  const bool fold = down >= 0x1p-70f;
  if (fold) h *= down, l *= down;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    Float2x y(x.pair(i).x, x.pair(i).y);
    if (!fold) y = y * Float2x(down);
    q[i] = fma2(y, Float2x(h), y * Float2x(l)).get();
  }
  codes = to_e2m1(q);
}

struct F4Row {  // what a row's largest magnitude says
  bool bad;
  float down;
  __device__ __forceinline__ F4Row(uint32_t amax) {
    bad = amax >= 0x7f800000u;
    down = __uint_as_float(static_cast<uint32_t>(127 - (bad ? 0 : f4_row_exponent(amax))) << 23);
  }
  __device__ __forceinline__ float rho() const {
    return __uint_as_float(bad ? 0x7fc00000u : (254u << 23) - __float_as_uint(down));
  }
};

// Writes 8 columns' codes of a record's row r, and a group's scale as one of four in a word.
template <typename T>
__device__ __forceinline__ void f4_put(const Raw8<T>& x, uint32_t bits, const F4Row& f, uint8_t* at, uint8_t* scales, int r) {
  const int lane = threadIdx.x & 31;
  uint32_t scale, codes;
  f4_encode(x, bits, f.down, scale, codes);
  if (f.bad) scale = codes = 0;
  *reinterpret_cast<uint32_t*>(at + f4_code_byte(r, lane * 8)) = codes;
  scale <<= 8 * (lane >> 1 & 3);
  scale |= __shfl_xor_sync(~0u, scale, 2);
  scale |= __shfl_xor_sync(~0u, scale, 4);
  if ((lane & 7) == 0) *reinterpret_cast<uint32_t*>(scales + f4_scale_byte(r, lane * 8) - kF4CodeBytes) = scale;
}

// Whether a product packs its rows itself, in every CTA, instead of by a launch before it: few rows, of which a CTA's 128
// threads read 16 x 8 columns each at most.
inline bool f4_packs_inside(int rows, int k) { return rows <= 4 && static_cast<int64_t>(rows) * k <= 16384; }

ssd_status f4_check_shape(int rows, int k);
ssd_status f4_pack_rows(const char* what, const void* x, int type, int rows, int k, int64_t x_row, void* packed,
                        cudaStream_t s);

}  // namespace ssd
