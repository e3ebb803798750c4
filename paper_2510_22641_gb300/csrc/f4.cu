// 4-bit floats: packing rows and reading them back.
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "f4.cuh"

namespace ssd {
namespace {

struct F4PackParams {
  const void* x;
  int64_t x_row;
  int rows, k, chunks, warps;
  uint8_t* out;
  float* rho;
};

// Eight neighbouring columns as they lie in memory: fp32 numbers, or pairs of bf16.
template <typename T>
struct Raw8 {
  uint32_t w[2 * sizeof(T)];

  // From `col` on, zeros past k.  VEC: 16-byte aligned.
  template <bool VEC>
  __device__ __forceinline__ void load(const T* p, int col, int k) {
    if (VEC && col + 8 <= k) {
#pragma unroll
      for (int i = 0; i < static_cast<int>(sizeof(T)) / 2; ++i)
        reinterpret_cast<uint4*>(w)[i] = reinterpret_cast<const uint4*>(p + col)[i];
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
  if (down >= 0x1p-70f) {
    h *= down, l *= down;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 y = x.pair(i);
      q[i] = make_float2(fmaf(y.x, h, y.x * l), fmaf(y.y, h, y.y * l));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float2 y = make_float2(x.pair(i).x * down, x.pair(i).y * down);
      q[i] = make_float2(fmaf(y.x, h, y.x * l), fmaf(y.y, h, y.y * l));
    }
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

// Writes 8 columns' codes, and a group's scale as one of four in a word.
template <typename T>
__device__ __forceinline__ void f4_put(const Raw8<T>& x, uint32_t bits, const F4Row& f, uint8_t* at, int r) {
  const int lane = threadIdx.x & 31;
  uint32_t scale, codes;
  f4_encode(x, bits, f.down, scale, codes);
  if (f.bad) scale = codes = 0;
  *reinterpret_cast<uint32_t*>(at + f4_code_byte(r, lane * 8)) = codes;
  scale <<= 8 * (lane >> 1 & 3);
  scale |= __shfl_xor_sync(~0u, scale, 2);
  scale |= __shfl_xor_sync(~0u, scale, 4);
  if ((lane & 7) == 0) *reinterpret_cast<uint32_t*>(at + f4_scale_byte(r, lane * 8)) = scale;
}

// A row is held in registers between its maximum and its codes, by p.warps warps (1, 2, 4 or 8) of up to J chunks of
// 256 columns each, 8 columns a lane; the CTA has 8 warps.  The row is read once.
template <typename T, bool VEC, int J>
__global__ void __launch_bounds__(256) ssd_f4_pack_kernel(const F4PackParams p) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint32_t part[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, c0 = warp % p.warps;
  const int row = blockIdx.x * (8 / p.warps) + warp / p.warps;
  const bool on = row < p.rows;
  const T* src = static_cast<const T*>(p.x) + (on ? row : 0) * p.x_row;
  Raw8<T> x[J];
  uint32_t amax = 0, most[J];
#pragma unroll
  for (int j = 0; j < J; ++j)
    if (c0 + j * p.warps < p.chunks) x[j].template load<VEC>(src, (c0 + j * p.warps) * kF4Cols + lane * 8, p.k);
#pragma unroll
  for (int j = 0; j < J; ++j)
    if (c0 + j * p.warps < p.chunks) amax = max(amax, most[j] = x[j].amax());
  amax = __reduce_max_sync(~0u, amax);
  if (p.warps > 1) {
    if (lane == 0) part[warp] = amax;
    __syncthreads();
    for (int i = 0; i < p.warps; ++i) amax = max(amax, part[warp - c0 + i]);
  }
  if (!on) return;
  const F4Row f(amax);
  if (c0 == 0 && lane == 0) p.rho[row] = f.rho();
  uint8_t* rec = p.out + static_cast<int64_t>(row / kF4Rows) * p.chunks * kF4Record;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int c = c0 + j * p.warps;
    if (c < p.chunks) f4_put(x[j], most[j], f, rec + static_cast<int64_t>(c) * kF4Record, row % kF4Rows);
  }
}

// Rows of more than 16384 columns are read twice, by 8 warps.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) ssd_f4_pack_long_kernel(const F4PackParams p) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint32_t part[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x;
  const T* src = static_cast<const T*>(p.x) + row * p.x_row;
  uint32_t amax = 0;
  Raw8<T> x;
  for (int c = warp; c < p.chunks; c += 8) {
    x.template load<VEC>(src, c * kF4Cols + lane * 8, p.k);
    amax = max(amax, x.amax());
  }
  amax = __reduce_max_sync(~0u, amax);
  if (lane == 0) part[warp] = amax;
  __syncthreads();
  for (int i = 0; i < 8; ++i) amax = max(amax, part[i]);
  const F4Row f(amax);
  if (threadIdx.x == 0) p.rho[row] = f.rho();
  uint8_t* rec = p.out + static_cast<int64_t>(row / kF4Rows) * p.chunks * kF4Record;
  for (int c = warp; c < p.chunks; c += 8) {
    x.template load<VEC>(src, c * kF4Cols + lane * 8, p.k);
    f4_put(x, x.amax(), f, rec + static_cast<int64_t>(c) * kF4Record, row % kF4Rows);
  }
}

// A CTA per record: a warp takes four rows at a time, of each 4 columns a lane and the 4 that are 128 further, so that
// neighbouring lanes store neighbouring bytes.  Products of code and scale have 6 bits and are exact in fp16.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) ssd_f4_unpack_kernel(const uint8_t* packed, int rows, int k, int chunks,
                                                            const float* rho, T* out) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, chunk = blockIdx.x, tile = blockIdx.y, col = chunk * kF4Cols + lane * 4;
  const uint8_t* at = packed + (static_cast<int64_t>(tile) * chunks + chunk) * kF4Record;
  const int end = min(rows - tile * kF4Rows, kF4Rows);
  rho += static_cast<int64_t>(tile) * kF4Rows;
  out += static_cast<int64_t>(tile) * kF4Rows * k + col;
  for (int r0 = threadIdx.x >> 5; r0 < end; r0 += 32) {
    uint32_t codes[4][2], scale[4][2];
    float f[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + 8 * i;
      if (r >= end) break;
      f[i] = rho[r];
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        codes[i][h] = *reinterpret_cast<const uint16_t*>(at + f4_code_byte(r, lane * 4 + 128 * h));
        scale[i][h] = at[f4_scale_byte(r, lane * 4 + 128 * h)];
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = r0 + 8 * i;
      if (r >= end) break;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const __half2 s = __half2half2(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(scale[i][h]), __NV_E4M3)));
        float v[4];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const __half2 c(__nv_cvt_fp4x2_to_halfraw2(static_cast<__nv_fp4x2_storage_t>(codes[i][h] >> (8 * j)), __NV_E2M1));
          const float2 t = __half22float2(__hmul2(c, s));
          v[2 * j] = t.x * f[i], v[2 * j + 1] = t.y * f[i];
        }
        T* y = out + static_cast<int64_t>(r) * k + 128 * h;
        const int left = k - col - 128 * h;
        if (VEC && left >= 4) {
          if constexpr (sizeof(T) == 4) {
            *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
          } else {
            const __nv_bfloat162 b[2] = {__floats2bfloat162_rn(v[0], v[1]), __floats2bfloat162_rn(v[2], v[3])};
            *reinterpret_cast<uint2*>(y) = *reinterpret_cast<const uint2*>(b);
          }
        } else {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (j < left) y[j] = from_f32<T>(v[j]);
        }
      }
    }
  }
}

template <typename T, bool VEC>
ssd_status f4_pack_dispatch(const char* what, F4PackParams& p, cudaStream_t s) {
  // one warp a row as long as it holds the row in two chunks a lane; eight from 8 chunks on
  p.warps = p.chunks <= 2 ? 1 : p.chunks <= 4 ? 2 : p.chunks <= 8 ? 4 : 8;
  const int each = 8 / p.warps;
  const dim3 grid((p.rows + each - 1) / each);
  if (p.chunks <= 16) return op_launch(what, ssd_f4_pack_kernel<T, VEC, 2>, grid, 256, 0, s, p);
  if (p.chunks <= 32) return op_launch(what, ssd_f4_pack_kernel<T, VEC, 4>, grid, 256, 0, s, p);
  if (p.chunks <= 64) return op_launch(what, ssd_f4_pack_kernel<T, VEC, 8>, grid, 256, 0, s, p);
  return op_launch(what, ssd_f4_pack_long_kernel<T, VEC>, grid, 256, 0, s, p);
}

template <typename T>
ssd_status f4_unpack_dispatch(const uint8_t* in, int rows, int k, T* out, cudaStream_t s) {
  const int chunks = f4_chunks(k);
  const float* rho = reinterpret_cast<const float*>(in + f4_scales_at(rows, k));
  const bool vec = reinterpret_cast<uintptr_t>(out) % (4 * sizeof(T)) == 0 && k % 4 == 0;
  for (int first = 0; first < rows; first += 65535 * kF4Rows) {  // what a grid's second dimension takes
    const int n = rows - first < 65535 * kF4Rows ? rows - first : 65535 * kF4Rows;
    const dim3 grid(chunks, (n + kF4Rows - 1) / kF4Rows);
    const uint8_t* at = in + static_cast<int64_t>(first / kF4Rows) * chunks * kF4Record;
    T* y = out + static_cast<int64_t>(first) * k;
    const ssd_status e =
        vec ? op_launch("ssd_f4_unpack", ssd_f4_unpack_kernel<T, true>, grid, 256, 0, s, at, n, k, chunks, rho + first, y)
            : op_launch("ssd_f4_unpack", ssd_f4_unpack_kernel<T, false>, grid, 256, 0, s, at, n, k, chunks, rho + first, y);
    if (e) return e;
  }
  return SSD_OK;
}

}  // namespace

ssd_status f4_check_shape(int rows, int k) {
  if (rows < 1 || k < 1 || rows > 1 << 23 || k > 1 << 20)
    return op_fail(SSD_ERR_INVALID_ARG, "4-bit floats: shape [%d][%d]", rows, k);
  return SSD_OK;
}

ssd_status f4_pack_rows(const char* what, const void* x, int type, int rows, int k, int64_t x_row, void* packed,
                        cudaStream_t s) {
  F4PackParams p{x, x_row, rows, k, f4_chunks(k), 0, static_cast<uint8_t*>(packed), nullptr};
  p.rho = reinterpret_cast<float*>(p.out + f4_scales_at(rows, k));
  const int size = type == SSD_TYPE_FP32 ? 4 : 2;
  const bool vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && (rows == 1 || x_row % (16 / size) == 0);
  if (type == SSD_TYPE_FP32)
    return vec ? f4_pack_dispatch<float, true>(what, p, s) : f4_pack_dispatch<float, false>(what, p, s);
  return vec ? f4_pack_dispatch<__nv_bfloat16, true>(what, p, s) : f4_pack_dispatch<__nv_bfloat16, false>(what, p, s);
}

}  // namespace ssd

using namespace ssd;

extern "C" {

int64_t ssd_f4_bytes(int rows, int k) {
  if (f4_check_shape(rows, k)) return -1;
  return f4_scales_at(rows, k) + static_cast<int64_t>((rows + kF4Rows - 1) / kF4Rows) * kF4Rows * 4;
}

ssd_status ssd_f4_pack(const void* x, int type, int rows, int k, int64_t x_row_stride, void* packed, void* cuda_stream) {
  if (ssd_status s = f4_check_shape(rows, k)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  const int size = type == SSD_TYPE_FP32 ? 4 : 2;
  if (!x || !packed || reinterpret_cast<uintptr_t>(packed) % 16 || reinterpret_cast<uintptr_t>(x) % size)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_pack: null or unaligned buffer");
  const int64_t bytes = ssd_f4_bytes(rows, k);
  if (op_overlap({x, rows, 1, x_row_stride * size, 0, static_cast<int64_t>(k) * size}, {packed, 1, 1, 0, 0, bytes}, 1))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_pack: packed overlaps x");
  return f4_pack_rows("ssd_f4_pack", x, type, rows, k, x_row_stride, packed, static_cast<cudaStream_t>(cuda_stream));
}

ssd_status ssd_f4_unpack(const void* packed, int rows, int k, void* out, int type, void* cuda_stream) {
  if (ssd_status s = f4_check_shape(rows, k)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  const int size = type == SSD_TYPE_FP32 ? 4 : 2;
  if (!out || !packed || reinterpret_cast<uintptr_t>(packed) % 16 || reinterpret_cast<uintptr_t>(out) % size)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_unpack: null or unaligned buffer");
  const uint8_t* in = static_cast<const uint8_t*>(packed);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return type == SSD_TYPE_FP32 ? f4_unpack_dispatch(in, rows, k, static_cast<float*>(out), s)
                               : f4_unpack_dispatch(in, rows, k, static_cast<__nv_bfloat16*>(out), s);
}

}  // extern "C"
