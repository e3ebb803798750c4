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
  int norms;        // whether any operand has a gain
  int slots, span, spans;  // lanes per head, heads per warp, warps per row
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

// One product rounded, the other not, in every kernel alike: a call's bits do not depend on its alignment.
__device__ __forceinline__ void turn_pair(float u, float v, float c, float s, float& a, float& b) {
  a = __fmaf_rn(u, c, -__fmul_rn(v, s));
  b = __fmaf_rn(v, c, __fmul_rn(u, s));
}

// What the units below do not divide: a warp per (row, head), pair p = lane + 32 j of a lane, scalar accesses.
template <typename T>
__global__ void __launch_bounds__(256) ssd_rotary_any_kernel(const RotaryParams p) {
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
      turn_pair(u, v, c, s, a[j], b[j]);
    }
    y[at[j]] = from_f32<T>(a[j]);
    y[with[j]] = from_f32<T>(b[j]);
  }
}

// What bounds this operator is one pass over the heads' bytes, so sines and cosines are made once per row and held in
// registers while a warp goes over heads.
//
// A head is cut into units of V neighbouring elements (16 bytes or less); `slots` lanes hold a head, each a pair of
// units: the two halves of a rotated pair (pairs apart), or two neighbouring units (pairs next to each other, elements
// that do not turn).  A warp takes 32 / slots heads at a time, `span` heads in all, of one row.
template <typename T, int V>
struct alignas(sizeof(T) * V) Unit {
  T v[V];
};

template <typename T, int V, bool APART>
__global__ void __launch_bounds__(256) ssd_rotary_kernel(const RotaryParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31;
  const int64_t job = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5);
  const int64_t row = job / p.spans;
  if (row >= p.rows) return;
  const int slots = p.slots, slot = lane % slots, in_warp = 32 / slots;
  int head = static_cast<int>(job % p.spans) * p.span;
  const int end = min(head + p.span, p.heads);
  const bool idle = lane >= in_warp * slots;
  const int half = p.r.turn / 2;
  // elements of the two units, and the first pair that turns with them
  int at, with, pair;
  if (APART) {
    const bool turns = slot * V < half;
    at = turns ? slot * V : p.r.turn + 2 * (slot * V - half);
    with = turns ? at + half : at + V;
    pair = turns ? slot * V : half;
  } else {
    at = slot * 2 * V, with = at + V, pair = slot * V;
  }
  float c[V], s[V];
#pragma unroll
  for (int j = 0; j < V; ++j) {
    c[j] = 1.0f, s[j] = 0.0f;
    if (pair + j < half) turn_of(p.pos[row * p.pos_row + p.r.axis[pair + j] * p.pos_axis], p.r.step[pair + j], c[j], s[j]);
  }
  float g[2][2 * V];
#pragma unroll
  for (int o = 0; o < 2; ++o) {
    const RotaryOperand& op = p.op[o];
#pragma unroll
    for (int j = 0; j < 2 * V; ++j) {
      const int i = j < V ? at + j : with + j - V;
      g[o][j] = !op.gain ? 1.0f : op.gain_fp32 ? static_cast<const float*>(op.gain)[i]
                                               : to_f32(static_cast<const __nv_bfloat16*>(op.gain)[i]);
    }
  }
  for (head += lane / slots; head - lane / slots < end; head += in_warp) {
    const bool on = !idle && head < end, second = head >= p.op[0].heads;
    const RotaryOperand& o = p.op[second];
    const int h = second ? head - p.op[0].heads : head;
    const T* x = static_cast<const T*>(o.x) + row * o.x_row + h * o.x_head;
    T* y = static_cast<T*>(o.y) + row * o.y_row + h * o.y_head;
    Unit<T, V> ua = {}, ub = {};
    if (on) {
      ua = *reinterpret_cast<const Unit<T, V>*>(x + at);
      ub = *reinterpret_cast<const Unit<T, V>*>(x + with);
    }
    float e[2 * V];
#pragma unroll
    for (int j = 0; j < V; ++j) e[j] = to_f32(ua.v[j]), e[V + j] = to_f32(ub.v[j]);
    if (p.norms) {
      float sum = 0.0f;
#pragma unroll
      for (int j = 0; j < 2 * V; ++j) sum += e[j] * e[j];
      // the sum over a head's lanes, a number that need not be a power of two
      for (int d = 1; d < slots; d <<= 1) {
        const float t = __shfl_down_sync(~0u, sum, d);
        if (slot + d < slots) sum += t;
      }
      sum = __shfl_sync(~0u, sum, lane - slot);
      if (o.gain) {
        const float inv = 1.0f / sqrtf(sum / p.r.head_dim + p.r.eps);
#pragma unroll
        for (int j = 0; j < 2 * V; ++j) e[j] *= inv * (second ? g[1][j] : g[0][j]);
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const int a = APART ? j : 2 * j, b = APART ? V + j : 2 * j + 1;
      const float u = e[a], v = e[b];
      if (pair + j < half) {
        turn_pair(u, v, c[j], s[j], e[a], e[b]);
      }
    }
#pragma unroll
    for (int j = 0; j < V; ++j) ua.v[j] = from_f32<T>(e[j]), ub.v[j] = from_f32<T>(e[V + j]);
    if (on) {
      *reinterpret_cast<Unit<T, V>*>(y + at) = ua;
      *reinterpret_cast<Unit<T, V>*>(y + with) = ub;
    }
  }
}

template <typename T, int V>
ssd_status rotary_launch(RotaryParams& p, cudaStream_t s) {
  p.slots = (p.r.head_dim / 2 + V - 1) / V;
  // A warp takes as many heads of a row as leave every SM its 48 warps or more: the row's sines are made anew by every
  // warp that works on it.
  const int in_warp = 32 / p.slots, turns = (p.heads + in_warp - 1) / in_warp;
  const int64_t all = static_cast<int64_t>(p.rows) * turns, most = all / (152 * 48);
  const int each = most < 1 ? 1 : most < turns ? static_cast<int>(most) : turns;
  const int parts = (turns + each - 1) / each;
  p.span = (turns + parts - 1) / parts * in_warp;
  p.spans = (p.heads + p.span - 1) / p.span;
  const int64_t ctas = (static_cast<int64_t>(p.rows) * p.spans + 7) / 8;
  if (ctas > 0x7fffffff) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: %d rows of %d heads", p.rows, p.heads);
  const dim3 grid(static_cast<unsigned>(ctas));
  return p.r.interleaved ? op_launch("ssd_rotary_apply", ssd_rotary_kernel<T, V, false>, grid, 256, 0, s, p)
                         : op_launch("ssd_rotary_apply", ssd_rotary_kernel<T, V, true>, grid, 256, 0, s, p);
}

// The widest unit that divides the pairs, the turning ones and every stride, and to which every head is aligned.
template <typename T>
ssd_status rotary_dispatch(RotaryParams& p, int n, cudaStream_t s) {
  uint64_t bits = static_cast<uint64_t>(p.r.head_dim / 2) | (p.r.turn / 2);
  for (int i = 0; i < n; ++i) {
    const RotaryOperand& o = p.op[i];
    bits |= (reinterpret_cast<uintptr_t>(o.x) | reinterpret_cast<uintptr_t>(o.y)) / sizeof(T);
    if (p.rows > 1) bits |= o.x_row | o.y_row;
    if (o.heads > 1) bits |= o.x_head | o.y_head;
  }
  if (sizeof(T) == 2 && bits % 8 == 0) return rotary_launch<T, 16 / sizeof(T)>(p, s);
  if (bits % 4 == 0) return rotary_launch<T, 4>(p, s);
  if (bits % 2 == 0 && p.r.head_dim <= 128) return rotary_launch<T, 2>(p, s);
  if (p.r.head_dim <= 64) return rotary_launch<T, 1>(p, s);
  const int64_t ctas = (static_cast<int64_t>(p.rows) * p.heads + 7) / 8;
  if (ctas > 0x7fffffff) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: %d rows of %d heads", p.rows, p.heads);
  return op_launch("ssd_rotary_apply", ssd_rotary_any_kernel<T>, dim3(static_cast<unsigned>(ctas)), 256, 0, s, p);
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
    p.norms |= h.gain != nullptr;
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
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return type == SSD_TYPE_FP32 ? rotary_dispatch<float>(p, n, s) : rotary_dispatch<__nv_bfloat16>(p, n, s);
}

}  // extern "C"
