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
constexpr int kRotaryWarps = 48;  // per SM
struct RotaryParams {
  ssd_rotary r;
  RotaryOperand op[2];
  const int32_t* pos;
  int64_t pos_row, pos_axis;
  int rows, heads;  // heads of both operands
  float per_element;  // 1 / head_dim
  int norms;        // whether any operand has a gain
  int slots, turns[2], warps;  // lanes per head; of each operand a warp's turns of 32 / slots heads; warps of a row in a CTA
};

// Cosine and sine of pos * step turns.  step is a 64-bit fraction of a turn, so the product's low 64 bits are the
// angle's fraction, with no rounding but the step's own to grow with the position.  Its upper 32 bits are taken, 2^-29 of a
// radian; the nearest quarter turn goes off as an integer.
__device__ __forceinline__ void turn_of(int pos, uint64_t step, float& c, float& s) {
  const int32_t t = static_cast<int32_t>((static_cast<uint64_t>(static_cast<int64_t>(pos)) * step) >> 32);
  const int32_t quarter = static_cast<int32_t>((static_cast<uint32_t>(t) + (1u << 29)) >> 30);
  const int32_t rest = static_cast<int32_t>(static_cast<uint32_t>(t) - (static_cast<uint32_t>(quarter) << 30));
  // Taylor series at |x| <= pi / 4: what is left out is below 2^-29 and 2^-33
  const float x = static_cast<float>(rest) * 1.46291807926715968e-9f, q = x * x;  // 2 pi / 2^32
  const float b = fmaf(x * q, fmaf(q, fmaf(q, fmaf(q, 1.0f / 362880.0f, -1.0f / 5040.0f), 1.0f / 120.0f), -1.0f / 6.0f), x);
  const float a =
      fmaf(q, fmaf(q, fmaf(q, fmaf(q, fmaf(q, -1.0f / 3628800.0f, 1.0f / 40320.0f), -1.0f / 720.0f), 1.0f / 24.0f), -0.5f), 1.0f);
  c = quarter & 1 ? b : a;
  s = quarter & 1 ? a : b;
  if (quarter == 1 || quarter == 2) c = -c;
  if (quarter & 2) s = -s;
}

// One product rounded, the other not, in every kernel alike: without norms a call's bits do not depend on its alignment.
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
    const float inv = rsqrtf(fmaf(sum, p.per_element, p.r.eps));
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

// What bounds this operator is one pass over the heads' bytes, so sines and cosines are made once per row (and CTA) in
// shared memory, and a warp holds its lanes' in registers while it goes over the row's heads.
//
// 16381 rows of 32 + 8 heads of 128, bf16, norms, three axes: 66 us, 5.1 TB/s (floor 50); sines in every warp 120 to 150,
// the table of frequencies read through the constant path (one address at a time) 118.  A lane has its two units and
// the next head's under way, 24 warps an SM: more warps with fewer registers are slower (72), as are 8-byte units (77).
//
// A head is cut into units of V neighbouring elements (16 bytes or less); `slots` lanes hold a head, each a pair of
// units: the two halves of a rotated pair (pairs apart), or two neighbouring units (pairs next to each other, elements
// that do not turn).  A warp takes 32 / slots heads of an operand at a time.
template <typename T, int V>
struct alignas(sizeof(T) * V) Unit {
  T v[V];
  __device__ __forceinline__ void unpack(float* e) const {
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
      for (int j = 0; j < V; j += 2) {
        const float2 f = bf16x2_to_float2(reinterpret_cast<const uint32_t*>(v)[j / 2]);
        e[j] = f.x, e[j + 1] = f.y;
      }
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) e[j] = to_f32(v[j]);
    }
  }
  __device__ __forceinline__ void pack(const float* e) {
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
      for (int j = 0; j < V; j += 2)
        reinterpret_cast<__nv_bfloat162*>(v)[j / 2] = __floats2bfloat162_rn(e[j], e[j + 1]);
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) v[j] = from_f32<T>(e[j]);
    }
  }
};

// The CTA's 8 warps work on 8 / p.warps rows, p.warps on each; gridDim.y CTAs share a row's heads.
template <typename T, int V, bool APART, bool NORM>
__global__ void __launch_bounds__(256) ssd_rotary_kernel(const __grid_constant__ RotaryParams p) {
  __shared__ float2 turn[8 * SSD_ROTARY_MAX_DIM / 2];
  __shared__ float gain[NORM ? 2 * SSD_ROTARY_MAX_DIM : 1];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, in_row = warp % p.warps;
  const int half = p.r.turn / 2, row = blockIdx.x * (8 / p.warps) + warp / p.warps;
  const bool on = row < p.rows;
  float2* const cs = turn + warp / p.warps * half;
  // lanes read different entries: through a pointer, as the constant path takes one address at a time
  const uint64_t* step = p.r.step;
  const uint8_t* axis = p.r.axis;
  asm volatile("" : "+l"(step), "+l"(axis));
  pdl_wait();
  pdl_trigger();
  if (on)
    for (int j = in_row * 32 + lane; j < half; j += p.warps * 32) {
      float c, s;
      turn_of(p.pos[row * p.pos_row + axis[j] * p.pos_axis], step[j], c, s);
      cs[j] = make_float2(c, s);
    }
  if (NORM)
    for (int i = threadIdx.x; i < 2 * p.r.head_dim; i += 256) {
      const RotaryOperand& o = p.op[i >= p.r.head_dim];
      const int j = i >= p.r.head_dim ? i - p.r.head_dim : i;
      gain[i] = !o.gain ? 1.0f : o.gain_fp32 ? static_cast<const float*>(o.gain)[j]
                                             : to_f32(static_cast<const __nv_bfloat16*>(o.gain)[j]);
    }
  __syncthreads();
  if (!on) return;
  const int slots = p.slots, in_warp = 32 / slots, mine = lane / slots, slot = lane - mine * slots;
  // elements of the two units, and whether they turn
  const bool turns = slot * V < half;
  int at = slot * 2 * V, with = at + V;
  if (APART) {
    at = turns ? slot * V : p.r.turn + 2 * (slot * V - half);
    with = turns ? at + half : at + V;
  }
  const bool pow2 = (slots & (slots - 1)) == 0;
  int t = blockIdx.y * p.warps + in_row;
  const int stride = gridDim.y * p.warps;
#pragma unroll 1
  for (int i = 0; i < 2; ++i) {
    const RotaryOperand& o = p.op[i];
    const int turns_of = p.turns[i];  // heads of this operand, in_warp at a time
    if (t >= turns_of) {
      t -= turns_of;
      continue;
    }
    const bool normed = NORM && o.gain;
    // a pair (u, v) becomes (u c - v s, v c + u s), with the gains of its elements in the factors
    float uc[V], vs[V], vc[V], us[V];  // vs negative
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const float2 f = turns ? cs[slot * V + j] : make_float2(1.0f, 0.0f);
      const int iu = APART ? at + j : at + 2 * j, iv = APART ? with + j : iu + 1;
      const float gu = NORM ? gain[i * p.r.head_dim + iu] : 1.0f, gv = NORM ? gain[i * p.r.head_dim + iv] : 1.0f;
      uc[j] = gu * f.x, vs[j] = -(gv * f.y), vc[j] = gv * f.x, us[j] = gu * f.y;
    }
    const T* x = static_cast<const T*>(o.x) + row * o.x_row + (t * in_warp + mine) * o.x_head;
    T* y = static_cast<T*>(o.y) + row * o.y_row + (t * in_warp + mine) * o.y_head;
    const int64_t x_step = stride * in_warp * o.x_head, y_step = stride * in_warp * o.y_head;
    Unit<T, V> ua = {}, ub = {};
    auto load = [&](int t, const T* x) {
      if (mine < in_warp && t * in_warp + mine < o.heads)
        ua = *reinterpret_cast<const Unit<T, V>*>(x + at), ub = *reinterpret_cast<const Unit<T, V>*>(x + with);
    };
    load(t, x);
#pragma unroll 1
    for (; t < turns_of; t += stride) {
      const bool keep = mine < in_warp && t * in_warp + mine < o.heads;
      float e[2 * V];
      ua.unpack(e), ub.unpack(e + V);
      x += x_step;
      if (t + stride < turns_of) load(t + stride, x);
      float inv = 1.0f;
      if (normed) {
        float sum = 0.0f;
        if constexpr (V % 2 == 0) {
          Float2x a(0.0f), b(0.0f);
#pragma unroll
          for (int j = 0; j < V; j += 2) {
            const Float2x u(e[j], e[j + 1]), v(e[V + j], e[V + j + 1]);
            a = fma2(u, u, a), b = fma2(v, v, b);
          }
          const float2 s = (a + b).get();
          sum = s.x + s.y;
        } else {
#pragma unroll
          for (int j = 0; j < 2 * V; ++j) sum = fmaf(e[j], e[j], sum);
        }
        if (pow2) {
          for (int d = 1; d < slots; d <<= 1) sum += __shfl_xor_sync(~0u, sum, d);
        } else {  // sums of the lanes above within the head, then the first lane's
          for (int d = 1; d < slots; d <<= 1) {
            const float v = __shfl_down_sync(~0u, sum, d);
            if (slot + d < slots) sum += v;
          }
          sum = __shfl_sync(~0u, sum, lane - slot);
        }
        inv = rsqrtf(fmaf(sum, p.per_element, p.r.eps));
      }
      float r[2 * V];
      if constexpr (APART && V % 2 == 0) {
        const Float2x f(inv);
#pragma unroll
        for (int j = 0; j < V; j += 2) {
          const Float2x u(e[j], e[j + 1]), v(e[V + j], e[V + j + 1]), c(uc[j], uc[j + 1]), d(vc[j], vc[j + 1]);
          Float2x a = u * c, b = v * d;
          if (turns) a = fma2(u, c, v * Float2x(vs[j], vs[j + 1])), b = fma2(v, d, u * Float2x(us[j], us[j + 1]));
          if (NORM) a = a * f, b = b * f;
          const float2 x2 = a.get(), y2 = b.get();
          r[j] = x2.x, r[j + 1] = x2.y, r[V + j] = y2.x, r[V + j + 1] = y2.y;
        }
      } else {
#pragma unroll
        for (int j = 0; j < V; ++j) {
          const int k = APART ? j : 2 * j, l = APART ? V + j : 2 * j + 1;
          r[k] = e[k] * uc[j], r[l] = e[l] * vc[j];
          if (turns && (APART || slot * V + j < half)) {
            r[k] = __fmaf_rn(e[k], uc[j], __fmul_rn(e[l], vs[j]));
            r[l] = __fmaf_rn(e[l], vc[j], __fmul_rn(e[k], us[j]));
          }
          if (NORM) r[k] *= inv, r[l] *= inv;
        }
      }
      Unit<T, V> ra, rb;
      ra.pack(r), rb.pack(r + V);
      if (keep) *reinterpret_cast<Unit<T, V>*>(y + at) = ra, *reinterpret_cast<Unit<T, V>*>(y + with) = rb;
      y += y_step;
    }
    t -= turns_of;
  }
}

template <typename T, int V>
ssd_status rotary_launch(RotaryParams& p, int n, cudaStream_t s) {
  p.slots = p.r.head_dim / 2 / V;
  const int in_warp = 32 / p.slots;
  for (int i = 0; i < n; ++i) p.turns[i] = (p.op[i].heads + in_warp - 1) / in_warp;
  const int turns = p.turns[0] + p.turns[1];
  // Warps of a row: as few (the row's sines are used most often) as leave every SM kRotaryWarps of them (2048 rows of 40
  // heads: with 48 13.8 us, with 192 22.9).
  const int64_t want = 152 * kRotaryWarps;
  int split = 1;
  while (split < turns && static_cast<int64_t>(p.rows) * split < want) split *= 2;
  p.warps = split < 8 ? split : 8;
  const int each = 8 / p.warps;
  const dim3 grid((p.rows + each - 1) / each, split / p.warps);
  if (p.norms)
    return p.r.interleaved ? op_launch("ssd_rotary_apply", ssd_rotary_kernel<T, V, false, true>, grid, 256, 0, s, p)
                           : op_launch("ssd_rotary_apply", ssd_rotary_kernel<T, V, true, true>, grid, 256, 0, s, p);
  return p.r.interleaved ? op_launch("ssd_rotary_apply", ssd_rotary_kernel<T, V, false, false>, grid, 256, 0, s, p)
                         : op_launch("ssd_rotary_apply", ssd_rotary_kernel<T, V, true, false>, grid, 256, 0, s, p);
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
  if (sizeof(T) == 2 && bits % 8 == 0) return rotary_launch<T, 16 / sizeof(T)>(p, n, s);
  if (bits % 4 == 0) return rotary_launch<T, 4>(p, n, s);
  if (bits % 2 == 0 && p.r.head_dim <= 128) return rotary_launch<T, 2>(p, n, s);
  if (p.r.head_dim <= 64) return rotary_launch<T, 1>(p, n, s);
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
  p.per_element = 1.0f / r->head_dim;
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
    const OpRows bytes{a.y, rows, a.heads, a.y_row * size, a.y_head * size, static_cast<int64_t>(r->head_dim) * size};
    if (op_overlap(bytes, {pos, rows, r->axes, pos_row * 4, pos_axis * 4, 4}, 1))
      return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: an output overlaps the positions");
    if (!op_apart(y)) return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: heads of an output overlap");
    for (int j = 0; j < n; ++j) {
      const ssd_heads& b = operand[j];
      const int64_t gain = r->head_dim * (b.gain_type == SSD_TYPE_FP32 ? 4 : 2);
      if (b.gain && op_overlap(bytes, {b.gain, 1, 1, 0, 0, gain}, 1))
        return op_fail(SSD_ERR_INVALID_ARG, "ssd_rotary_apply: an output overlaps a gain");
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
