// Norms of query and key heads and the rotation by their positions, in one pass.
#include <math.h>

#include "lowbit.cuh"

namespace ssd {
namespace {

struct RotaryOperand {
  const void* x;
  void* y;
  const void* gain;
  int64_t x_row, x_head, y_row, y_head;
  int heads, gain_fp32;
};
struct RotaryParams {
  ssd_rotary r;
  RotaryOperand op[2];
  const int32_t* pos;
  int64_t pos_row, pos_axis;
  int rows, heads;  // heads of both operands
};

// Cosine and sine of pos * step turns.  step is a 64-bit fraction of a turn, so the product's low 64 bits are the
// angle's fraction, with no rounding to grow with the position; the nearest quarter turn is taken off as an integer.
__device__ __forceinline__ void turn_of(int pos, uint64_t step, float& c, float& s) {
  const int32_t t = static_cast<int32_t>((static_cast<uint64_t>(static_cast<int64_t>(pos)) * step) >> 32);
  const int32_t quarter = static_cast<int32_t>((static_cast<uint32_t>(t) + (1u << 29)) >> 30);
  const int32_t rest = static_cast<int32_t>(static_cast<uint32_t>(t) - (static_cast<uint32_t>(quarter) << 30));
  float a, b;
  sincospif(static_cast<float>(rest) * 0x1p-31f, &b, &a);
  c = quarter & 1 ? b : a;
  s = quarter & 1 ? a : b;
  if (quarter == 1 || quarter == 2) c = -c;
  if (quarter & 2) s = -s;
}

// Any head size, pairing and stride: a warp per (row, head), pair p = lane + 32 j of a lane, scalar accesses.
template <typename T>
__global__ void __launch_bounds__(256) ssd_rotary_kernel(const RotaryParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int64_t job = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const int64_t row = job / p.heads;
  if (row >= p.rows) return;
  int head = static_cast<int>(job % p.heads);
  const bool second = head >= p.op[0].heads;
  const RotaryOperand& o = p.op[second];
  if (second) head -= p.op[0].heads;
  const T* x = static_cast<const T*>(o.x) + row * o.x_row + head * o.x_head;
  T* y = static_cast<T*>(o.y) + row * o.y_row + head * o.y_head;
  const int half = p.r.turn / 2, pairs = p.r.head_dim / 2;
  float a[4], b[4], sum = 0.0f;
  int at[4], with[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = lane + 32 * j;
    const bool split = i < half && !p.r.interleaved;
    at[j] = split ? i : 2 * i;
    with[j] = split ? i + half : 2 * i + 1;
    a[j] = i < pairs ? to_f32(x[at[j]]) : 0.0f;
    b[j] = i < pairs ? to_f32(x[with[j]]) : 0.0f;
    sum += a[j] * a[j] + b[j] * b[j];
  }
  if (o.gain) {
#pragma unroll
    for (int d = 16; d; d >>= 1) sum += __shfl_xor_sync(~0u, sum, d);
    const float inv = 1.0f / sqrtf(sum / p.r.head_dim + p.r.eps);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (lane + 32 * j >= pairs) continue;
      const float* gf = static_cast<const float*>(o.gain);
      const __nv_bfloat16* gb = static_cast<const __nv_bfloat16*>(o.gain);
      a[j] *= inv * (o.gain_fp32 ? gf[at[j]] : to_f32(gb[at[j]]));
      b[j] *= inv * (o.gain_fp32 ? gf[with[j]] : to_f32(gb[with[j]]));
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = lane + 32 * j;
    if (i >= pairs) continue;
    if (i < half) {
      float c, s;
      turn_of(p.pos[row * p.pos_row + p.r.axis[i] * p.pos_axis], p.r.step[i], c, s);
      const float u = a[j], v = b[j];
      a[j] = u * c - v * s;
      b[j] = v * c + u * s;
    }
    y[at[j]] = from_f32<T>(a[j]);
    y[with[j]] = from_f32<T>(b[j]);
  }
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" {

ssd_status ssd_rotary_init(ssd_rotary* r, int head_dim, int turn, int interleaved, int axes, const int* section,
                           double theta, float eps) {
  if (!r) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_init: null");
  if (head_dim < 2 || head_dim > SSD_ROTARY_MAX_DIM || head_dim % 2 || turn < 0 || turn > head_dim || turn % 2)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary: heads of %d with %d that turn", head_dim, turn);
  if (axes < 1 || axes > SSD_ROTARY_MAX_AXES || (axes > 1 && !section))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary: %d axes", axes);
  if (!(theta >= 1.0) || !isfinite(theta) || !(eps >= 0.0f) || !isfinite(eps))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary: theta %g, eps %g", theta, static_cast<double>(eps));
  ssd_rotary t = {};
  t.head_dim = head_dim, t.turn = turn, t.interleaved = interleaved != 0, t.axes = axes, t.eps = eps;
  int sum = 0;
  for (int a = 0; section && a < axes; ++a) {
    if (section[a] < 0 || section[a] > turn / 2 - sum)
      return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary: sections do not add up to %d pairs", turn / 2);
    for (int i = 0; i < section[a]; ++i) t.axis[sum + i] = static_cast<uint8_t>(a);
    sum += section[a];
  }
  if (section && sum != turn / 2)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary: sections do not add up to %d pairs", turn / 2);
  for (int i = 0; i < turn / 2; ++i)  // radians a position, as a 64-bit fraction of a turn
    t.step[i] = static_cast<uint64_t>(ldexp(pow(theta, -2.0 * i / turn) / (2.0 * M_PI), 64));
  *r = t;
  return SSD_OK;
}

ssd_status ssd_rotary_apply(const ssd_rotary* r, const ssd_heads* operand, int n, int type, int rows, const int32_t* pos,
                            int64_t pos_row, int64_t pos_axis, void* cuda_stream) {
  if (!r || !operand || n < 1 || n > 2) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: %d operands", n);
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  if (r->head_dim < 2 || r->head_dim > SSD_ROTARY_MAX_DIM || r->head_dim % 2 || r->turn < 0 || r->turn > r->head_dim ||
      r->turn % 2 || r->axes < 1 || r->axes > SSD_ROTARY_MAX_AXES || !(r->eps >= 0.0f))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: not what ssd_rotary_init makes");
  for (int i = 0; i < r->turn / 2; ++i)
    if (r->axis[i] >= r->axes) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: pair %d turns by axis %d", i, r->axis[i]);
  if (rows < 0 || rows > 1 << 26) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: %d rows", rows);
  if (rows == 0) return SSD_OK;
  if (!pos || reinterpret_cast<uintptr_t>(pos) % 4) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: positions");
  const int size = type == SSD_TYPE_FP32 ? 4 : 2;
  RotaryParams p = {};
  p.r = *r, p.pos = pos, p.pos_row = pos_row, p.pos_axis = pos_axis, p.rows = rows;
  for (int i = 0; i < n; ++i) {
    const ssd_heads& h = operand[i];
    if (h.heads < 1 || h.heads > 1 << 14) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: %d heads", h.heads);
    if (!h.x || !h.y || (reinterpret_cast<uintptr_t>(h.x) | reinterpret_cast<uintptr_t>(h.y)) % size)
      return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: null or unaligned buffer");
    if (h.gain && h.gain_type != SSD_TYPE_BF16 && h.gain_type != SSD_TYPE_FP32)
      return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: gain_type %d", h.gain_type);
    if (h.gain && reinterpret_cast<uintptr_t>(h.gain) % (h.gain_type == SSD_TYPE_FP32 ? 4 : 2))
      return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: unaligned gain");
    p.op[i] = {h.x, h.y, h.gain, h.x_row, h.x_head, h.y_row, h.y_head, h.heads, h.gain_type == SSD_TYPE_FP32};
    p.heads += h.heads;
  }
  for (int i = 0; i < n; ++i) {
    const ssd_heads& a = operand[i];
    const OpRows y{a.y, rows, a.heads, a.y_row, a.y_head, r->head_dim};
    if (!op_apart(y)) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: heads of an output overlap");
    for (int j = 0; j < n; ++j) {
      const ssd_heads& b = operand[j];
      const bool same = i == j && a.y == b.x && (rows == 1 || a.y_row == b.x_row) && (a.heads == 1 || a.y_head == b.x_head);
      if ((!same && op_overlap(y, {b.x, rows, b.heads, b.x_row, b.x_head, r->head_dim}, size)) ||
          (j > i && op_overlap(y, {b.y, rows, b.heads, b.y_row, b.y_head, r->head_dim}, size)))
        return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: an output overlaps another operand");
    }
  }
  const int64_t ctas = (static_cast<int64_t>(rows) * p.heads + 7) / 8;
  if (ctas > 0x7fffffff) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: %d rows of %d heads", rows, p.heads);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const dim3 grid(static_cast<unsigned>(ctas));
  return type == SSD_TYPE_FP32 ? op_launch("ssd_rotary_apply", ssd_rotary_kernel<float>, grid, 256, 0, s, p)
                               : op_launch("ssd_rotary_apply", ssd_rotary_kernel<__nv_bfloat16>, grid, 256, 0, s, p);
}

}  // extern "C"
