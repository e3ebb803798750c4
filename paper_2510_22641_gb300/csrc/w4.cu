// 4-bit weights with group scales: packing, and products with 1..16 activation rows.
#include "lowbit.cuh"

namespace ssd {
namespace {

// ------------------------------------------------------------------ layout
//
// [16-row tile][128-column chunk]: 1024 bytes of codes, then 16 rows x (128 / group) bf16 scales.
// A lane (g = lane / 4, t = lane % 4) of mma.m16n8k16 takes rows g and g + 8 at columns 4t .. 4t + 3 of
// each 16-column step: 8 codes, one 32-bit word.  Nibble i of the low half and nibble i of the high
// half of the word form operand register i (even column in the low half), so one mask per register
// brings both codes into place.  Words of four steps make a lane's 16 bytes, lanes lie side by side.

constexpr int kChunk = 128;
constexpr int kCodeBytes = 16 * kChunk / 2;

__host__ __device__ constexpr int w4_record(int group) { return kCodeBytes + 16 * (kChunk / group) * 2; }
// Bit position of (row, column) in a tile's codes.
__host__ __device__ constexpr int w4_bit(int row, int col) {
  const int step = col >> 4, t = (col >> 2) & 3, c = col & 3;
  const int reg = (row >> 3) + 2 * (c >> 1);  // a0: row g, a1: row g + 8, a2 / a3: columns + 2
  const int nibble = reg + 4 * (c & 1);
  const int lane = (row & 7) * 4 + t;
  return (((step >> 2) * 32 + lane) * 16 + (step & 3) * 4) * 8 + nibble * 4;
}

// ------------------------------------------------------------------ pack / unpack

struct W4PackParams {
  const void* w;
  int64_t row_stride;
  int n, k, group, chunks;
  uint8_t* out;
};

// One warp per (row, group): the rows of a tile write different nibbles, so a CTA packs a whole tile
// chunk in shared memory (8 warps, two rows each).
template <typename T>
__global__ void __launch_bounds__(256) ssd_w4_pack_kernel(const W4PackParams p) {
  __shared__ uint32_t codes[kCodeBytes / 4];
  __shared__ __nv_bfloat16 scales[16 * 4];
  const int tid = threadIdx.x, lane = tid & 31, w = tid >> 5;
  const int tile = blockIdx.y, chunk = blockIdx.x, per = kChunk / p.group;
  for (int i = tid; i < kCodeBytes / 4; i += 256) codes[i] = 0;
  __syncthreads();
  for (int job = w; job < 16 * per; job += 8) {
    const int row = job / per, grp = job % per, n = tile * 16 + row;
    float x[4], amax = 0.0f;
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = lane + 32 * i, col = chunk * kChunk + grp * p.group + c;
      x[i] = 0.0f;
      if (c < p.group && n < p.n && col < p.k)
        x[i] = to_f32(static_cast<const T*>(p.w)[static_cast<int64_t>(n) * p.row_stride + col]);
      nan |= x[i] != x[i];
      amax = fmaxf(amax, fabsf(x[i]));
    }
    amax = warp_max(amax);
    if (__any_sync(~0u, nan)) amax = __int_as_float(0x7fc00000);
    const __nv_bfloat16 sb = __float2bfloat16_rn(amax / 7.0f);
    const float s = __bfloat162float(sb), inv = s > 0.0f ? 1.0f / s : 0.0f;
    if (lane == 0) scales[row * per + grp] = sb;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = lane + 32 * i;
      if (c >= p.group) continue;
      const float q = fminf(fmaxf(rintf(x[i] * inv), -8.0f), 7.0f);
      const int bit = w4_bit(row, grp * p.group + c);
      atomicOr(&codes[bit >> 5], static_cast<uint32_t>(static_cast<int>(q) + 8) << (bit & 31));
    }
  }
  __syncthreads();
  uint8_t* rec = p.out + (static_cast<size_t>(tile) * p.chunks + chunk) * w4_record(p.group);
  for (int i = tid; i < kCodeBytes / 4; i += 256) reinterpret_cast<uint32_t*>(rec)[i] = codes[i];
  for (int i = tid; i < 16 * per; i += 256) reinterpret_cast<__nv_bfloat16*>(rec + kCodeBytes)[i] = scales[i];
}

__global__ void __launch_bounds__(256) ssd_w4_unpack_kernel(const uint8_t* packed, int n, int k, int group, int chunks,
                                                            float* out) {
  const int row = blockIdx.y;
  const int per = kChunk / group;
  for (int64_t c64 = blockIdx.x * 256 + threadIdx.x; c64 < k; c64 += static_cast<int64_t>(gridDim.x) * 256) {
    const int col = static_cast<int>(c64);
    const uint8_t* rec = packed + (static_cast<size_t>(row >> 4) * chunks + col / kChunk) * w4_record(group);
    const int bit = w4_bit(row & 15, col % kChunk);
    const int code = static_cast<int>(reinterpret_cast<const uint32_t*>(rec)[bit >> 5] >> (bit & 31) & 15u) - 8;
    const __nv_bfloat16* sc = reinterpret_cast<const __nv_bfloat16*>(rec + kCodeBytes);
    out[static_cast<size_t>(row) * k + col] = code * __bfloat162float(sc[(row & 15) * per + (col % kChunk) / group]);
  }
}

// ------------------------------------------------------------------ matmul

struct W4Params {
  const uint8_t* packed;
  int n, k, group, chunks, rows;
  const void* x;
  void* y;
  const void* residual;
  int64_t x_row, y_row, r_row;
};

// One warp per output row: lanes over the columns.
template <typename T>
__global__ void __launch_bounds__(128) ssd_w4_matmul_kernel(const W4Params p) {
  const int lane = threadIdx.x & 31, row = blockIdx.x * 4 + (threadIdx.x >> 5);
  if (row >= p.n) return;
  const int per = kChunk / p.group;
  float acc[SSD_W4_MAX_ROWS];
#pragma unroll
  for (int m = 0; m < SSD_W4_MAX_ROWS; ++m) acc[m] = 0.0f;
  for (int col = lane; col < p.k; col += 32) {
    const uint8_t* rec = p.packed + (static_cast<size_t>(row >> 4) * p.chunks + col / kChunk) * w4_record(p.group);
    const int bit = w4_bit(row & 15, col % kChunk);
    const int code = static_cast<int>(reinterpret_cast<const uint32_t*>(rec)[bit >> 5] >> (bit & 31) & 15u) - 8;
    const __nv_bfloat16* sc = reinterpret_cast<const __nv_bfloat16*>(rec + kCodeBytes);
    const float w = code * __bfloat162float(sc[(row & 15) * per + (col % kChunk) / p.group]);
#pragma unroll
    for (int m = 0; m < SSD_W4_MAX_ROWS; ++m)
      if (m < p.rows) acc[m] += w * to_f32(static_cast<const T*>(p.x)[m * p.x_row + col]);
  }
#pragma unroll
  for (int m = 0; m < SSD_W4_MAX_ROWS; ++m) {
    if (m >= p.rows) break;
    const float v = warp_sum(acc[m]);
    if (lane == 0) {
      const float r = p.residual ? to_f32(static_cast<const T*>(p.residual)[m * p.r_row + row]) : 0.0f;
      static_cast<T*>(p.y)[m * p.y_row + row] = from_f32<T>(v + r);
    }
  }
}

ssd_status check_shape(int n, int k, int group) {
  if (group != 32 && group != 64 && group != 128) return op_fail(SSD_ERR_INVALID_ARG, "group %d", group);
  if (n < 1 || k < 1 || n > 16 * 65535 || k > (1 << 24))
    return op_fail(SSD_ERR_INVALID_ARG, "weight shape [%d][%d]", n, k);
  return SSD_OK;
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" {

int64_t ssd_w4_bytes(int n, int k, int group) {
  if (check_shape(n, k, group)) return -1;
  return static_cast<int64_t>((n + 15) / 16) * ((k + kChunk - 1) / kChunk) * w4_record(group);
}

int64_t ssd_w4_work_bytes(int n, int k) {
  if (check_shape(n, k, 128)) return -1;
  return 16;
}

ssd_status ssd_w4_pack(const void* w, int type, int n, int k, int64_t row_stride, int group, void* packed,
                       void* cuda_stream) {
  if (ssd_status s = check_shape(n, k, group)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  if (!w || !packed || reinterpret_cast<uintptr_t>(packed) % 16)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_w4_pack: null or unaligned buffer");
  W4PackParams p{w, row_stride, n, k, group, (k + kChunk - 1) / kChunk, static_cast<uint8_t*>(packed)};
  const dim3 grid(p.chunks, (n + 15) / 16);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (type == SSD_TYPE_FP32) ssd_w4_pack_kernel<float><<<grid, 256, 0, s>>>(p);
  else ssd_w4_pack_kernel<__nv_bfloat16><<<grid, 256, 0, s>>>(p);
  return op_launched("ssd_w4_pack");
}

ssd_status ssd_w4_unpack(const void* packed, int n, int k, int group, float* out, void* cuda_stream) {
  if (ssd_status s = check_shape(n, k, group)) return s;
  if (!out || !packed || reinterpret_cast<uintptr_t>(packed) % 16)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_w4_unpack: null or unaligned buffer");
  for (int first = 0; first < n; first += 65520) {  // whole tiles per launch
    const int m = n - first < 65520 ? n - first : 65520;
    const int chunks = (k + kChunk - 1) / kChunk;
    const dim3 grid(k < 256 * 64 ? (k + 255) / 256 : 64, m);
    ssd_w4_unpack_kernel<<<grid, 256, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
        static_cast<const uint8_t*>(packed) + static_cast<size_t>(first / 16) * chunks * w4_record(group), m, k, group,
        chunks, out + static_cast<size_t>(first) * k);
    if (ssd_status s = op_launched("ssd_w4_unpack")) return s;
  }
  return SSD_OK;
}

ssd_status ssd_w4_matmul(const void* packed, int n, int k, int group, const void* x, int type, int rows,
                         int64_t x_row_stride, void* y, int64_t y_row_stride, const void* residual,
                         int64_t res_row_stride, void* work, void* cuda_stream) {
  if (ssd_status s = check_shape(n, k, group)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  if (rows < 0 || rows > SSD_W4_MAX_ROWS)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_w4_matmul: %d rows, at most %d", rows, SSD_W4_MAX_ROWS);
  if (rows == 0) return SSD_OK;
  if (!packed || !x || !y || !work || reinterpret_cast<uintptr_t>(packed) % 16 || reinterpret_cast<uintptr_t>(work) % 16)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_w4_matmul: null or unaligned buffer");
  const int size = type == SSD_TYPE_FP32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(x) | reinterpret_cast<uintptr_t>(y) | reinterpret_cast<uintptr_t>(residual)) % size)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_w4_matmul: rows must be aligned to their elements");
  W4Params p{static_cast<const uint8_t*>(packed), n, k, group, (k + kChunk - 1) / kChunk, rows, x, y, residual,
             x_row_stride, y_row_stride, res_row_stride};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (type == SSD_TYPE_FP32) ssd_w4_matmul_kernel<float><<<(n + 3) / 4, 128, 0, s>>>(p);
  else ssd_w4_matmul_kernel<__nv_bfloat16><<<(n + 3) / 4, 128, 0, s>>>(p);
  return op_launched("ssd_w4_matmul");
}

}  // extern "C"
