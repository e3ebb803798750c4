// 4-bit weights with group scales: packing, the activation rows' form, and the C entry points.
#include "w4.cuh"

namespace ssd {
namespace {

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
    bool bad = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = lane + 32 * i, col = chunk * kChunk + grp * p.group + c;
      x[i] = 0.0f;
      if (c < p.group && n < p.n && col < p.k)
        x[i] = to_f32(static_cast<const T*>(p.w)[static_cast<int64_t>(n) * p.row_stride + col]);
      bad |= !(fabsf(x[i]) <= 3.402823466e38f);
      amax = fmaxf(amax, fabsf(x[i]));
    }
    amax = warp_max(amax);
    if (__any_sync(~0u, bad)) amax = __int_as_float(0x7fc00000);  // shows in every product of the row
    const __nv_bfloat16 sb = __float2bfloat16_rn(amax / 7.0f);
    const float s = __bfloat162float(sb);
    float inv = s > 0.0f ? 1.0f / s : 0.0f;
    if (inv > 3.402823466e38f) inv = 0.0f;  // scales below 2^-128
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

// Activation rows in the form the products take, padded to whole chunks with zeros, one warp per row and
// chunk: fp32 rows as high and low halves of x 2^(14 - e) with 2^e beside them (2^e <= the chunk's
// largest magnitude < 2^(e + 1)); bf16 rows copied.
struct W4RowsParams {
  const void* x;
  int64_t x_row;
  int rows, k, chunks;
  uint16_t* out;
  float* scale;
};

template <typename T>
__global__ void __launch_bounds__(128) ssd_w4_rows_kernel(const W4RowsParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int64_t job = static_cast<int64_t>(blockIdx.x) * 4 + (threadIdx.x >> 5);
  if (job >= static_cast<int64_t>(p.rows) * p.chunks) return;
  const int r = static_cast<int>(job % p.rows), chunk = static_cast<int>(job / p.rows);
  const T* src = static_cast<const T*>(p.x) + r * p.x_row;
  const int64_t kp = static_cast<int64_t>(p.chunks) * kChunk;
  const int col = chunk * kChunk + 4 * lane;
  T v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = col + i < p.k ? src[col + i] : from_f32<T>(0.0f);
  uint16_t* dst = p.out + r * kp + col;
  if constexpr (sizeof(T) == 2) {
    *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(v);
  } else {
    const float amax = warp_max(fmaxf(fmaxf(fabsf(v[0]), fabsf(v[1])), fmaxf(fabsf(v[2]), fabsf(v[3]))));
    // 2^e between 2^-112 and 2^127, so that 2^(14 - e) is a normal number; an infinite row stays infinite
    const uint32_t ex = min(max(__float_as_uint(amax) & 0x7f800000u, 15u << 23), 254u << 23);
    const float up = __uint_as_float(((127u + 14u + 127u) << 23) - ex);
    __half h[4], l[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float x = v[i] * up;
      h[i] = __float2half_rn(x);
      l[i] = __float2half_rn(x - __half2float(h[i]));
    }
    *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(h);
    *reinterpret_cast<uint2*>(dst + SSD_W4_MAX_ROWS * kp) = *reinterpret_cast<const uint2*>(l);
    if (lane == 0) p.scale[chunk * 16 + r] = __uint_as_float(ex);
  }
}

ssd_status check_shape(int n, int k, int group) {
  if (group != 32 && group != 64 && group != 128) return op_fail(SSD_ERR_INVALID_ARG, "group %d", group);
  if (n < 1 || k < 1 || n > 16 * 65535 || k > (1 << 20))
    return op_fail(SSD_ERR_INVALID_ARG, "weight shape [%d][%d]", n, k);
  return SSD_OK;
}

// The workspace: activation rows in 16 bits, then their scales.
struct WorkLayout {
  int64_t scale, total;
};
WorkLayout work_layout(int k) {
  const int64_t chunks = (k + kChunk - 1) / kChunk;
  WorkLayout w;
  w.scale = 2ll * SSD_W4_MAX_ROWS * chunks * kChunk * 2;
  w.total = w.scale + chunks * 16 * 4;
  return w;
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
  return work_layout(k).total;
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
  const OpRows xr{x, rows, 1, x_row_stride, 0, k}, yr{y, rows, 1, y_row_stride, 0, n},
      rr{residual, rows, 1, res_row_stride, 0, n};
  if (op_overlap(xr, yr, size)) return op_fail(SSD_ERR_INVALID_ARG, "ssd_w4_matmul: y overlaps x");
  const bool in_place = residual == y && (rows == 1 || res_row_stride == y_row_stride);
  if (residual && !in_place && op_overlap(rr, yr, size))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_w4_matmul: y overlaps the residual and is not the same rows");
  const WorkLayout lay = work_layout(k);
  uint8_t* wk = static_cast<uint8_t*>(work);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  W4Params p = {};
  p.packed = static_cast<const uint8_t*>(packed);
  p.n = n;
  p.chunks = (k + kChunk - 1) / kChunk;
  p.rec = w4_record(group);
  p.rows = rows;
  // at least two chunks for each warp of a team
  p.log_warps = p.chunks >= 16 ? 3 : p.chunks >= 8 ? 2 : p.chunks >= 4 ? 1 : 0;
  p.y = y;
  p.residual = residual;
  p.y_row = y_row_stride;
  p.r_row = res_row_stride;
  // bf16 rows that are whole chunks of aligned 16-byte pieces are operands as they lie
  if (type == SSD_TYPE_BF16 && k % kChunk == 0 && x_row_stride % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0) {
    p.x = static_cast<const uint16_t*>(x);
    p.x_row = x_row_stride;
  } else {
    p.x_row = static_cast<int64_t>(p.chunks) * kChunk;
    p.x_part = SSD_W4_MAX_ROWS * p.x_row;
    p.x_scale = reinterpret_cast<const float*>(wk + lay.scale);
    W4RowsParams r{x, x_row_stride, rows, k, p.chunks, reinterpret_cast<uint16_t*>(wk),
                   reinterpret_cast<float*>(wk + lay.scale)};
    p.x = r.out;
    const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(rows) * p.chunks + 3) / 4);
    if (ssd_status e = type == SSD_TYPE_FP32
                           ? op_launch("ssd_w4_matmul", ssd_w4_rows_kernel<float>, dim3(grid), 128, 0, s, r)
                           : op_launch("ssd_w4_matmul", ssd_w4_rows_kernel<__nv_bfloat16>, dim3(grid), 128, 0, s, r))
      return e;
  }
  const int per = kChunk / group;
  if (type == SSD_TYPE_FP32)
    return rows <= 4 ? w4_matmul_fp32_4(per, p, s) : rows <= 8 ? w4_matmul_fp32_8(per, p, s) : w4_matmul_fp32_16(per, p, s);
  return rows <= 8 ? w4_matmul_bf16_8(per, p, s) : w4_matmul_bf16_16(per, p, s);
}

}  // extern "C"
