// 4-bit floats: packing rows and reading them back.
#include "f4.cuh"

namespace ssd {
namespace {

struct F4PackParams {
  const void* x;
  int64_t x_row;
  int rows, k, chunks, warps_log;
  uint8_t* out;
  float* rho;
};

// Packing reads x and writes 0.56 bytes an element: 22016 x 4096 bf16 in 50 us (floor 34), fp32 in 64 (floor 61).  At bf16
// neither bytes (0.68 of the copy rate) nor instructions (16 an element, 74 % of the issue slots) bound it alone: warps
// wait for loads, 57 % of the places taken.  Read twice, eight warps a row, correctly rounded reciprocals: 77.
//
// A row is held in registers between its maximum and its codes, by `warps` warps (1, 2, 4 or 8) of up to J chunks of
// 256 columns each, 8 columns a lane; the CTA has 8 warps.  The row is read once.
template <typename T, bool VEC, int J>
__global__ void __launch_bounds__(256) ssd_f4_pack_kernel(const F4PackParams p) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint32_t part[8];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = 1 << p.warps_log, c0 = warp & (warps - 1);
  const int row = (blockIdx.x << (3 - p.warps_log)) + (warp >> p.warps_log);
  const bool on = row < p.rows;
  const T* src = static_cast<const T*>(p.x) + (on ? row : 0) * p.x_row;
  Raw8<T> x[J];
  uint32_t amax = 0, most[J];
#pragma unroll
  for (int j = 0; j < J; ++j)
    if (c0 + j * warps < p.chunks) x[j].template load<VEC>(src, (c0 + j * warps) * kF4Cols + lane * 8, p.k);
#pragma unroll
  for (int j = 0; j < J; ++j)
    if (c0 + j * warps < p.chunks) amax = max(amax, most[j] = x[j].amax());
  amax = __reduce_max_sync(~0u, amax);
  if (warps > 1) {
    if (lane == 0) part[warp] = amax;
    __syncthreads();
    amax = __reduce_max_sync(~0u, part[warp - c0 + (lane & (warps - 1))]);
  }
  if (!on) return;
  const F4Row f(amax);
  if (c0 == 0 && lane == 0) p.rho[row] = f.rho();
  uint8_t* rec = p.out + static_cast<int64_t>(row / kF4Rows) * p.chunks * kF4Record;
#pragma unroll
  for (int j = 0; j < J; ++j) {
    const int c = c0 + j * warps;
    uint8_t* at = rec + static_cast<int64_t>(c) * kF4Record;
    if (c < p.chunks) f4_put(x[j], most[j], f, at, at + kF4CodeBytes, row % kF4Rows);
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
    uint8_t* at = rec + static_cast<int64_t>(c) * kF4Record;
    f4_put(x, x.amax(), f, at, at + kF4CodeBytes, row % kF4Rows);
  }
}

// Reading back writes 4 bytes an element (to fp32) for 0.56 read: 22016 x 4096 in 66 us, 0.92 of the copy rate (to bf16 40,
// 0.86); eight
// neighbouring columns a lane, whose stores leave every second 16 bytes to the next instruction, took 81, a column a
// thread 357.
//
// A CTA per record: a warp takes four rows at a time, of each 4 columns a lane and the 4 that are 128 further, so that
// neighbouring lanes store neighbouring bytes.  Products of code and scale have 6 bits and are exact in fp16.
template <typename T>
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
        if (left <= 0) continue;  // k is a multiple of four
        if constexpr (sizeof(T) == 4) {
          *reinterpret_cast<float4*>(y) = make_float4(v[0], v[1], v[2], v[3]);
        } else {
          const __nv_bfloat162 b[2] = {__floats2bfloat162_rn(v[0], v[1]), __floats2bfloat162_rn(v[2], v[3])};
          *reinterpret_cast<uint2*>(y) = *reinterpret_cast<const uint2*>(b);
        }
      }
    }
  }
}

// Rows that are not aligned to four elements: a lane decodes 8 columns, and the warp stores 32 neighbouring ones at a time,
// by way of shared memory.
template <typename T>
__global__ void __launch_bounds__(256) ssd_f4_unpack_odd_kernel(const uint8_t* packed, int rows, int k, int chunks,
                                                                const float* rho, T* out) {
  pdl_wait();
  pdl_trigger();
  __shared__ alignas(16) float turn[8][kF4Cols];  // stored by 16 bytes
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, chunk = blockIdx.x, tile = blockIdx.y;
  const int left = k - chunk * kF4Cols, end = min(rows - tile * kF4Rows, kF4Rows);
  const uint8_t* at = packed + (static_cast<int64_t>(tile) * chunks + chunk) * kF4Record;
  rho += static_cast<int64_t>(tile) * kF4Rows;
  out += static_cast<int64_t>(tile) * kF4Rows * k + chunk * kF4Cols;
  for (int r0 = warp; r0 < end; r0 += 32) {
    uint32_t codes[4], scale[4];
    float f[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int r = min(r0 + 8 * j, end - 1);
      codes[j] = *reinterpret_cast<const uint32_t*>(at + f4_code_byte(r, lane * 8));
      scale[j] = at[f4_scale_byte(r, lane * 8)];
      f[j] = rho[r];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (r0 + 8 * j >= end) break;
      const __half2 s = __half2half2(__half(__nv_cvt_fp8_to_halfraw(static_cast<__nv_fp8_storage_t>(scale[j]), __NV_E4M3)));
      float2 v[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const __half2 c(__nv_cvt_fp4x2_to_halfraw2(static_cast<__nv_fp4x2_storage_t>(codes[j] >> (8 * i)), __NV_E2M1));
        v[i] = __half22float2(__hmul2(c, s));
      }
      __syncwarp();
#pragma unroll
      for (int i = 0; i < 2; ++i)
        reinterpret_cast<float4*>(turn[warp])[lane * 2 + i] =
            make_float4(v[2 * i].x * f[j], v[2 * i].y * f[j], v[2 * i + 1].x * f[j], v[2 * i + 1].y * f[j]);
      __syncwarp();
      T* y = out + static_cast<int64_t>(r0 + 8 * j) * k + lane;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (32 * i >= left) break;
        if (32 * i + lane < left) y[32 * i] = from_f32<T>(turn[warp][32 * i + lane]);
      }
    }
  }
}

template <typename T, bool VEC>
ssd_status f4_pack_dispatch(const char* what, F4PackParams& p, cudaStream_t s) {
  // Many rows: as few warps a row as hold it in four chunks a lane, which spreads what a warp does once; few rows: two
  // chunks, for more warps.
  const int each = p.rows >= 152 * 8 ? 4 : 2;
  p.warps_log = 0;
  while (p.warps_log < 3 && p.chunks > each << p.warps_log) ++p.warps_log;
  const int in_cta = 8 >> p.warps_log, held = (p.chunks + (1 << p.warps_log) - 1) >> p.warps_log;
  const dim3 grid((p.rows + in_cta - 1) / in_cta);
  if (held <= 2) return op_launch(what, ssd_f4_pack_kernel<T, VEC, 2>, grid, 256, 0, s, p);
  if (held <= 4) return op_launch(what, ssd_f4_pack_kernel<T, VEC, 4>, grid, 256, 0, s, p);
  if (held <= 8) return op_launch(what, ssd_f4_pack_kernel<T, VEC, 8>, grid, 256, 0, s, p);
  return op_launch(what, ssd_f4_pack_long_kernel<T, VEC>, dim3(p.rows), 256, 0, s, p);
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
        vec ? op_launch("ssd_f4_unpack", ssd_f4_unpack_kernel<T>, grid, 256, 0, s, at, n, k, chunks, rho + first, y)
            : op_launch("ssd_f4_unpack", ssd_f4_unpack_odd_kernel<T>, grid, 256, 0, s, at, n, k, chunks, rho + first, y);
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

int64_t ssd_f4_work_bytes(int rows, int k) {
  if (f4_check_shape(rows, k)) return -1;
  return f4_packs_inside(rows, k) ? 0 : ssd_f4_bytes(rows, k);
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
  if (op_overlap({out, 1, 1, 0, 0, static_cast<int64_t>(rows) * k * size}, {packed, 1, 1, 0, 0, ssd_f4_bytes(rows, k)}, 1))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_unpack: out overlaps packed");
  const uint8_t* in = static_cast<const uint8_t*>(packed);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return type == SSD_TYPE_FP32 ? f4_unpack_dispatch(in, rows, k, static_cast<float*>(out), s)
                               : f4_unpack_dispatch(in, rows, k, static_cast<__nv_bfloat16*>(out), s);
}

}  // extern "C"
