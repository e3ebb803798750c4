// Attention of a step's query rows over the paged 8-bit cache.
#include "lowbit.cuh"

namespace ssd {
namespace {

struct Kv8AttnParams {
  const void* q;
  void* o;
  int64_t q_row, q_head, o_row, o_head;
  const uint32_t* row_mask;
  int32_t* step;
  int batch, rows, group, n_kv_heads, shift, n_blocks, max_blocks;
  float scale_log2;
  const uint8_t* data;
  const float* scales;
  const int32_t* table;
};

// One CTA per (row, query head); the warps take the keys in turn and merge their running maxima.
template <typename T, int D>
__global__ void __launch_bounds__(128) ssd_kv8_attn_kernel(const Kv8AttnParams p) {
  constexpr int E = D / 32;
  __shared__ float m_s[4], l_s[4], o_s[4][D];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int row = blockIdx.x, hq = blockIdx.y, h = hq / p.group;
  const StepView st = step_view(p.step, p.batch);
  T* out = static_cast<T*>(p.o) + row * p.o_row + hq * p.o_head;
  if (row >= st.row_start[p.batch]) {
    for (int d = threadIdx.x; d < D; d += 128) out[d] = from_f32<T>(0.0f);
    return;
  }
  int lo = 0, hi = p.batch;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (st.row_start[mid] <= row) lo = mid; else hi = mid;
  }
  const int b = lo, i = row - st.row_start[b], rows_b = st.row_start[b + 1] - st.row_start[b], len = st.len[b];
  const T* q = static_cast<const T*>(p.q) + row * p.q_row + hq * p.q_head;
  float qv[E], acc[E];
#pragma unroll
  for (int e = 0; e < E; ++e) {
    qv[e] = to_f32(q[lane * E + e]) * p.scale_log2;
    acc[e] = 0.0f;
  }
  float m = -INFINITY, l = 0.0f;
  const int bs = 1 << p.shift;
  const int64_t cap = static_cast<int64_t>(p.max_blocks) << p.shift;
  const int n = static_cast<int>(min(static_cast<int64_t>(len) + rows_b, cap));
  const uint32_t mask = p.row_mask ? p.row_mask[row] : 0;
  for (int pos = w; pos < n; pos += 4) {
    const int j = pos - len;
    if (j >= 0 && (p.row_mask ? j >= 32 || !(mask >> j & 1) : j > i)) continue;
    const int blk = p.table[static_cast<size_t>(b) * p.max_blocks + (pos >> p.shift)];
    if (blk < 0 || blk >= p.n_blocks) continue;
    const size_t rec = static_cast<size_t>(blk) * p.n_kv_heads + h;
    const int token = pos & (bs - 1);
    const uint8_t* tile = p.data + rec * (static_cast<size_t>(bs) * 2 * D) + (token >> 4) * (32 * D);
    float s = 0.0f;
#pragma unroll
    for (int e = 0; e < E; ++e)
      s += qv[e] * (static_cast<int>(tile[kv8_k_byte(token & 15, lane * E + e, D)]) - 128);
    s = warp_sum(s) * p.scales[rec * 2];
    const float m_new = fmaxf(m, s), a = exp2f(m - m_new), e_s = exp2f(s - m_new);
    m = m_new;
    l = l * a + e_s;
    const float wv = e_s * p.scales[rec * 2 + 1];
#pragma unroll
    for (int e = 0; e < E; ++e)
      acc[e] = acc[e] * a + wv * (static_cast<int>(tile[16 * D + kv8_v_byte(token & 15, lane * E + e)]) - 128);
  }
  if (lane == 0) {
    m_s[w] = m;
    l_s[w] = l;
  }
#pragma unroll
  for (int e = 0; e < E; ++e) o_s[w][lane * E + e] = acc[e];
  __syncthreads();
  for (int d = threadIdx.x; d < D; d += 128) {
    float mm = -INFINITY, ll = 0.0f, oo = 0.0f;
    for (int k = 0; k < 4; ++k) mm = fmaxf(mm, m_s[k]);
    for (int k = 0; k < 4; ++k) {
      const float f = l_s[k] > 0.0f || l_s[k] != l_s[k] ? exp2f(m_s[k] - mm) : 0.0f;
      ll += l_s[k] * f;
      oo += o_s[k][d] * f;
    }
    out[d] = from_f32<T>(ll == 0.0f ? 0.0f : oo / ll);
  }
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" {

int64_t ssd_kv8_work_bytes(const ssd_kv8* c) {
  if (!kv8_shape_ok(c)) return -1;
  return kKv8WorkHead * 4;
}

ssd_status ssd_kv8_attention(const ssd_kv8* c, int layer, const ssd_kv8_step* step, const void* q, void* o, int type,
                             int64_t q_row_stride, int64_t q_head_stride, int64_t o_row_stride, int64_t o_head_stride,
                             float scale, const uint32_t* row_mask, void* cuda_stream) {
  if (ssd_status s = kv8_check(c, layer)) return s;
  if (ssd_status s = kv8_check_step(c, step)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  if (step->rows == 0) return SSD_OK;
  if (!q || !o) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_attention: null buffer");
  const int size = type == SSD_TYPE_FP32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(o)) % size)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_attention: q and o must be aligned to their elements");
  Kv8AttnParams p;
  p.q = q;
  p.o = o;
  p.q_row = q_row_stride;
  p.q_head = q_head_stride;
  p.o_row = o_row_stride;
  p.o_head = o_head_stride;
  p.row_mask = row_mask;
  p.step = step->data;
  p.batch = step->batch;
  p.rows = step->rows;
  p.group = c->n_heads / c->n_kv_heads;
  p.n_kv_heads = c->n_kv_heads;
  p.shift = 31 - __builtin_clz(c->block_tokens);
  p.n_blocks = c->n_blocks;
  p.max_blocks = c->max_blocks;
  p.scale_log2 = scale * 1.4426950408889634f;
  const size_t recs = static_cast<size_t>(layer) * c->n_blocks * c->n_kv_heads;
  p.data = static_cast<const uint8_t*>(c->data) + recs * c->block_tokens * c->head_dim * 2;
  p.scales = c->scales + recs * 2;
  p.table = c->table;
  const dim3 grid(step->rows, c->n_heads);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (type == SSD_TYPE_FP32) {
    if (c->head_dim == 128) ssd_kv8_attn_kernel<float, 128><<<grid, 128, 0, s>>>(p);
    else ssd_kv8_attn_kernel<float, 64><<<grid, 128, 0, s>>>(p);
  } else {
    if (c->head_dim == 128) ssd_kv8_attn_kernel<__nv_bfloat16, 128><<<grid, 128, 0, s>>>(p);
    else ssd_kv8_attn_kernel<__nv_bfloat16, 64><<<grid, 128, 0, s>>>(p);
  }
  return op_launched("ssd_kv8_attention");
}

}  // extern "C"
