// 4-bit floats: packing rows and reading them back.
#include <cuda_fp4.h>
#include <cuda_fp8.h>

#include "f4.cuh"

namespace ssd {
namespace {

struct F4PackParams {
  const void* x;
  int64_t x_row;
  int rows, k, chunks;
  uint8_t* out;
  float* rho;
};

// Eight neighbouring columns from `col` on, zeros past k.
template <bool VEC>
__device__ __forceinline__ void load8(const float* p, int col, int k, float* v) {
  if (VEC && col + 8 <= k) {
    const float4 a = *reinterpret_cast<const float4*>(p + col), b = *reinterpret_cast<const float4*>(p + col + 4);
    v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + i < k ? p[col + i] : 0.0f;
  }
}
template <bool VEC>
__device__ __forceinline__ void load8(const __nv_bfloat16* p, int col, int k, float* v) {
  if (VEC && col + 8 <= k) {
    const uint4 w = *reinterpret_cast<const uint4*>(p + col);
    const float2 a = bf16x2_to_float2(w.x), b = bf16x2_to_float2(w.y), c = bf16x2_to_float2(w.z),
                 d = bf16x2_to_float2(w.w);
    v[0] = a.x, v[1] = a.y, v[2] = b.x, v[3] = b.y, v[4] = c.x, v[5] = c.y, v[6] = d.x, v[7] = d.y;
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = col + i < k ? to_f32(p[col + i]) : 0.0f;
  }
}

__device__ __forceinline__ float e4m3_value(uint32_t byte) {
  return __half2float(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(byte), __NV_E4M3)));
}

// A row's scale from the bits of its largest magnitude: the exponent of the smallest 2^e with amax <= 2688 2^e
// (2688 = 1.3125 * 2^11), at least -100.
__device__ __forceinline__ int f4_row_exponent(uint32_t amax) {
  return max(static_cast<int>(amax >> 23) - 127 - 11 + ((amax & 0x7fffffu) > 0x280000u ? 1 : 0), -100);
}

// One row's 16-column group, half of it (8 columns) in this lane and half in lane ^ 1, scaled by the row's 2^-e:
// the scale's byte and the 8 codes.  Quotients are correctly rounded by one step of Markstein's (IBM J. R&D 34, 1990)
// from a correctly rounded reciprocal; s has four bits, so its reciprocal is never the theorem's exception.
__device__ __forceinline__ void f4_encode(float* y, uint32_t& scale, uint32_t& codes) {
  float m = 0.0f;
#pragma unroll
  for (int i = 0; i < 8; ++i) m = fmaxf(m, fabsf(y[i]));
  m = fmaxf(m, __shfl_xor_sync(~0u, m, 1));
  scale = __nv_cvt_float_to_fp8(m / 6.0f, __NV_SATFINITE, __NV_E4M3);
  const float s = e4m3_value(scale), r = s > 0.0f ? __frcp_rn(s) : 0.0f;
  codes = 0;
#pragma unroll
  for (int i = 0; i < 8; i += 2) {
    float2 q;
    q.x = y[i] * r;
    q.y = y[i + 1] * r;
    q.x = fmaf(fmaf(-q.x, s, y[i]), r, q.x);
    q.y = fmaf(fmaf(-q.y, s, y[i + 1]), r, q.y);
    codes |= static_cast<uint32_t>(__nv_cvt_float2_to_fp4x2(q, __NV_E2M1, cudaRoundNearest)) << (4 * i);
  }
}

// One CTA per row, a warp per 256 columns at a time: 8 columns a lane, two lanes a group.  Two passes over the row.
template <typename T, bool VEC>
__global__ void __launch_bounds__(256) ssd_f4_pack_kernel(const F4PackParams p) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint32_t part[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, row = blockIdx.x;
  const T* src = static_cast<const T*>(p.x) + row * p.x_row;
  uint32_t amax = 0;  // as bits: a NaN is above infinity, infinity above the rest
  float v[8];
  for (int c = warp; c < p.chunks; c += 8) {
    load8<VEC>(src, c * kF4Cols + lane * 8, p.k, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) amax = max(amax, __float_as_uint(v[i]) & 0x7fffffffu);
  }
  amax = __reduce_max_sync(~0u, amax);
  if (lane == 0) part[warp] = amax;
  __syncthreads();
  for (int i = 0; i < 8; ++i) amax = max(amax, part[i]);
  const bool bad = amax >= 0x7f800000u;
  const int e = bad ? 0 : f4_row_exponent(amax);
  const float down = __uint_as_float(static_cast<uint32_t>(127 - e) << 23);
  if (threadIdx.x == 0) p.rho[row] = __uint_as_float(bad ? 0x7fc00000u : static_cast<uint32_t>(127 + e) << 23);
  const int r = row % kF4Rows;
  uint8_t* rec = p.out + static_cast<int64_t>(row / kF4Rows) * p.chunks * kF4Record;
  for (int c = warp; c < p.chunks; c += 8) {
    load8<VEC>(src, c * kF4Cols + lane * 8, p.k, v);
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = bad ? 0.0f : v[i] * down;
    uint32_t scale, codes;
    f4_encode(v, scale, codes);
    uint8_t* at = rec + static_cast<int64_t>(c) * kF4Record;
    *reinterpret_cast<uint32_t*>(at + f4_code_byte(r, lane * 8)) = codes;
    // four groups' scales are one word
    scale <<= 8 * (lane >> 1 & 3);
    scale |= __shfl_xor_sync(~0u, scale, 2);
    scale |= __shfl_xor_sync(~0u, scale, 4);
    if ((lane & 7) == 0) *reinterpret_cast<uint32_t*>(at + f4_scale_byte(r, lane * 8)) = scale;
  }
}

template <typename T>
__global__ void __launch_bounds__(256) ssd_f4_unpack_kernel(const uint8_t* packed, int k, int chunks, const float* rho, int first,
                                                            T* out) {
  pdl_wait();
  pdl_trigger();
  const int row = first + blockIdx.y, r = row % kF4Rows;
  const float scale = rho[row];
  const uint8_t* rec = packed + static_cast<int64_t>(row / kF4Rows) * chunks * kF4Record;
  for (int col = blockIdx.x * 256 + threadIdx.x; col < k; col += gridDim.x * 256) {
    const uint8_t* at = rec + static_cast<int64_t>(col / kF4Cols) * kF4Record;
    const int c = col % kF4Cols;
    const uint32_t code = at[f4_code_byte(r, c)] >> (4 * (c & 1)) & 15u;
    const float mag = (code & 7u) < 2 ? 0.5f * (code & 7u) : __uint_as_float(((code & 7u) + 252u) << 22);
    const float v = (code & 8u ? -mag : mag) * e4m3_value(at[f4_scale_byte(r, c)]) * scale;
    out[static_cast<int64_t>(row) * k + col] = from_f32<T>(v);
  }
}

}  // namespace

ssd_status f4_check_shape(int rows, int k) {
  if (rows < 1 || k < 1 || rows > 1 << 23 || k > 1 << 20)
    return op_fail(SSD_ERR_INVALID_ARG, "4-bit floats: shape [%d][%d]", rows, k);
  return SSD_OK;
}

ssd_status f4_pack_rows(const char* what, const void* x, int type, int rows, int k, int64_t x_row, void* packed,
                        cudaStream_t s) {
  F4PackParams p{x, x_row, rows, k, f4_chunks(k), static_cast<uint8_t*>(packed), nullptr};
  p.rho = reinterpret_cast<float*>(p.out + f4_scales_at(rows, k));
  const int size = type == SSD_TYPE_FP32 ? 4 : 2;
  const bool vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && x_row % (16 / size) == 0;
  const dim3 grid(rows);
  if (type == SSD_TYPE_FP32)
    return vec ? op_launch(what, ssd_f4_pack_kernel<float, true>, grid, 256, 0, s, p)
               : op_launch(what, ssd_f4_pack_kernel<float, false>, grid, 256, 0, s, p);
  return vec ? op_launch(what, ssd_f4_pack_kernel<__nv_bfloat16, true>, grid, 256, 0, s, p)
             : op_launch(what, ssd_f4_pack_kernel<__nv_bfloat16, false>, grid, 256, 0, s, p);
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
  const int chunks = f4_chunks(k);
  const uint8_t* in = static_cast<const uint8_t*>(packed);
  const float* rho = reinterpret_cast<const float*>(in + f4_scales_at(rows, k));
  for (int first = 0; first < rows; first += 65535) {
    const dim3 grid((k + 255) / 256, rows - first < 65535 ? rows - first : 65535);
    cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
    const ssd_status e =
        type == SSD_TYPE_FP32
            ? op_launch("ssd_f4_unpack", ssd_f4_unpack_kernel<float>, grid, 256, 0, s, in, k, chunks, rho, first,
                        static_cast<float*>(out))
            : op_launch("ssd_f4_unpack", ssd_f4_unpack_kernel<__nv_bfloat16>, grid, 256, 0, s, in, k, chunks, rho, first,
                        static_cast<__nv_bfloat16*>(out));
    if (e) return e;
  }
  return SSD_OK;
}

}  // extern "C"
