// Products of rows and weights that are both packed to 4-bit floats.
#include "f4.cuh"

#include <cuda_fp8.h>

namespace ssd {
namespace {

struct F4MatmulParams {
  const uint8_t *w, *x;
  const float *w_rho, *x_rho;
  int n, k, rows, chunks;
  void* y;
  const void* residual;
  int64_t y_row, r_row;
};

// sum * rho_x * rho_w by two powers of two with the same sign of exponent, so that neither step leaves the range
// unless the result does.  A NaN stays one.
__device__ __forceinline__ float f4_scaled(float sum, uint32_t rho_x, uint32_t rho_w) {
  const uint32_t e = (rho_x >> 23) + (rho_w >> 23), half = e >> 1;
  if (rho_x >= 0x7f800000u || rho_w >= 0x7f800000u) return __uint_as_float(0x7fc00000u);
  return sum * __uint_as_float(half << 23) * __uint_as_float((e - half) << 23);
}

// 64 x rows by 64 weight rows a CTA, 4 x 4 a thread, 64 columns at a time from shared memory.
template <typename T>
__global__ void __launch_bounds__(256) ssd_f4_matmul_kernel(const F4MatmulParams p) {
  pdl_wait();
  pdl_trigger();
  __shared__ float xs[64][65], ws[64][65];
  const int n0 = blockIdx.x * 64, m0 = blockIdx.y * 64, tn = threadIdx.x & 15, tm = threadIdx.x >> 4;
  float acc[4][4] = {};
  for (int k0 = 0; k0 < p.chunks * kF4Cols; k0 += 64) {
    for (int i = threadIdx.x; i < 2 * 64 * 64; i += 256) {
      const bool of_w = i >= 4096;
      const int r = (i >> 6 & 63) + (of_w ? n0 : m0), c = k0 + (i & 63);
      float v = 0.0f;
      if (r < (of_w ? p.n : p.rows)) {
        const uint8_t* at = (of_w ? p.w : p.x) + (static_cast<int64_t>(r / kF4Rows) * p.chunks + c / kF4Cols) * kF4Record;
        const uint32_t code = at[f4_code_byte(r % kF4Rows, c % kF4Cols)] >> (4 * (c & 1)) & 15u;
        const float mag = (code & 7u) < 2 ? 0.5f * (code & 7u) : __uint_as_float(((code & 7u) + 252u) << 22);
        const __nv_fp8_storage_t s = at[f4_scale_byte(r % kF4Rows, c % kF4Cols)];
        v = (code & 8u ? -mag : mag) * __half2float(__half(__nv_cvt_fp8_to_halfraw(s, __NV_E4M3)));
      }
      (of_w ? ws : xs)[i >> 6 & 63][i & 63] = v;
    }
    __syncthreads();
    for (int c = 0; c < 64; ++c)
#pragma unroll
      for (int a = 0; a < 4; ++a)
#pragma unroll
        for (int b = 0; b < 4; ++b) acc[a][b] = fmaf(xs[tm + 16 * a][c], ws[tn + 16 * b][c], acc[a][b]);
    __syncthreads();
  }
#pragma unroll
  for (int a = 0; a < 4; ++a)
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      const int m = m0 + tm + 16 * a, n = n0 + tn + 16 * b;
      if (m >= p.rows || n >= p.n) continue;
      float v = f4_scaled(acc[a][b], __float_as_uint(p.x_rho[m]), __float_as_uint(p.w_rho[n]));
      if (p.residual) v += to_f32(static_cast<const T*>(p.residual)[m * p.r_row + n]);
      static_cast<T*>(p.y)[m * p.y_row + n] = from_f32<T>(v);
    }
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" {

ssd_status ssd_f4_matmul(const void* w, int n, int k, const void* x, int x_type, int rows, int64_t x_row_stride, void* y,
                         int type, int64_t y_row_stride, const void* residual, int64_t res_row_stride, void* work,
                         void* cuda_stream) {
  if (ssd_status s = f4_check_shape(n, k)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  const bool packed = x_type == SSD_TYPE_F4;
  if (!packed && x_type != SSD_TYPE_BF16 && x_type != SSD_TYPE_FP32)
    return op_fail(SSD_ERR_INVALID_ARG, "x_type %d", x_type);
  if (rows == 0) return SSD_OK;
  if (ssd_status s = f4_check_shape(rows, k)) return s;
  const void* xp = packed ? x : work;
  if (!w || !x || !y || !xp || reinterpret_cast<uintptr_t>(w) % 16 || reinterpret_cast<uintptr_t>(xp) % 16)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: null or unaligned buffer");
  const int size = type == SSD_TYPE_FP32 ? 4 : 2, xsize = x_type == SSD_TYPE_FP32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(y) | reinterpret_cast<uintptr_t>(residual)) % size ||
      (!packed && reinterpret_cast<uintptr_t>(x) % xsize))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: rows must be aligned to their elements");
  const int64_t wbytes = ssd_f4_bytes(n, k), xbytes = ssd_f4_bytes(rows, k);
  const OpRows yb{y, rows, 1, y_row_stride * size, 0, static_cast<int64_t>(n) * size}, wb{w, 1, 1, 0, 0, wbytes},
      pb{xp, 1, 1, 0, 0, xbytes}, xb{x, rows, 1, x_row_stride * xsize, 0, static_cast<int64_t>(k) * xsize},
      rb{residual, rows, 1, res_row_stride * size, 0, static_cast<int64_t>(n) * size};
  if (!op_apart(yb)) return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: rows of y overlap");
  if (op_overlap(yb, wb, 1) || op_overlap(yb, pb, 1) || (!packed && op_overlap(yb, xb, 1)))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: y overlaps x, w or work");
  if (!packed && (op_overlap(pb, xb, 1) || op_overlap(pb, wb, 1) || (residual && op_overlap(pb, rb, 1))))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: work overlaps x, w or the residual");
  const bool in_place = residual == y && (rows == 1 || res_row_stride == y_row_stride);
  if (residual && !in_place && op_overlap(rb, yb, 1))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: y overlaps the residual and is not the same rows");
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (!packed)
    if (ssd_status e = f4_pack_rows("ssd_f4_matmul", x, x_type, rows, k, x_row_stride, work, s)) return e;
  F4MatmulParams p{};
  p.w = static_cast<const uint8_t*>(w);
  p.x = static_cast<const uint8_t*>(xp);
  p.w_rho = reinterpret_cast<const float*>(p.w + f4_scales_at(n, k));
  p.x_rho = reinterpret_cast<const float*>(p.x + f4_scales_at(rows, k));
  p.n = n, p.k = k, p.rows = rows, p.chunks = f4_chunks(k);
  p.y = y, p.residual = residual, p.y_row = y_row_stride, p.r_row = res_row_stride;
  const dim3 grid((n + 63) / 64, (rows + 63) / 64);
  if (grid.y > 65535) return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: %d rows", rows);
  return type == SSD_TYPE_FP32 ? op_launch("ssd_f4_matmul", ssd_f4_matmul_kernel<float>, grid, 256, 0, s, p)
                               : op_launch("ssd_f4_matmul", ssd_f4_matmul_kernel<__nv_bfloat16>, grid, 256, 0, s, p);
}

}  // extern "C"
