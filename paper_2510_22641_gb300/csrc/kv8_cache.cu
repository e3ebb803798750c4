// The paged 8-bit K/V cache: block tables and slot maps (plan), quantising writes (append), reads.
#include <stdarg.h>
#include <stdio.h>

#include "lowbit.cuh"

namespace ssd {

namespace {
thread_local char g_op_error[256] = "";
}

ssd_status op_fail(ssd_status s, const char* fmt, ...) {
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(g_op_error, sizeof(g_op_error), fmt, ap);
  va_end(ap);
  return s;
}

ssd_status op_launched(const char* what) {
  const cudaError_t e = cudaGetLastError();
  return e == cudaSuccess ? SSD_OK : op_fail(SSD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}

ssd_status kv8_check(const ssd_kv8* c, int layer) {
  if (!kv8_shape_ok(c)) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8: unsupported shape");
  if (!c->data || !c->scales || !c->table || !c->pool || !c->work)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8: null buffer");
  if ((reinterpret_cast<uintptr_t>(c->data) | reinterpret_cast<uintptr_t>(c->work)) % 16 ||
      reinterpret_cast<uintptr_t>(c->scales) % 8)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8: data and work must be 16-byte, scales 8-byte aligned");
  if (layer < 0 || layer >= c->n_layers) return op_fail(SSD_ERR_INVALID_ARG, "layer %d of %d", layer, c->n_layers);
  return SSD_OK;
}

ssd_status kv8_check_step(const ssd_kv8* c, const ssd_kv8_step* s) {
  if (!s || !s->data || reinterpret_cast<uintptr_t>(s->data) % 16)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_step: null or unaligned buffer");
  if (s->batch < 1 || s->batch > c->max_batch)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_step: batch %d, cache has %d seats", s->batch, c->max_batch);
  if (s->rows < 0 || static_cast<int64_t>(s->rows) * c->n_heads > 0x7fffffff)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_step: %d rows", s->rows);
  if (s->row_tile != 0 && s->row_tile != 8 && s->row_tile != 16 && s->row_tile != 24 && s->row_tile != 32)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_step: row_tile %d", s->row_tile);
  return SSD_OK;
}

namespace {

// ------------------------------------------------------------------ plan

constexpr int kPlanThreads = 256;
constexpr int kPlanPer = SSD_KV8_MAX_BATCH / kPlanThreads;

struct PlanParams {
  int batch, rows, max_batch, max_blocks, n_blocks, shift;  // block_tokens = 1 << shift
  int n_kv_heads, group, row_tile;
  const int32_t *len, *add, *state_in;
  int32_t *state_out, *table, *pool, *step, *status, *ticket;
};

// Exclusive sums of N values per thread over the CTA; total[] gets the sums.
template <int N>
__device__ __forceinline__ void block_scan(int64_t (&v)[N], int64_t (&total)[N], int64_t (*tot)[N]) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  int64_t x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = v[i];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int64_t y = __shfl_up_sync(~0u, x[i], o);
      if (lane >= o) x[i] += y;
    }
  }
  if (lane == 31)
#pragma unroll
    for (int i = 0; i < N; ++i) tot[w][i] = x[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    int64_t before = 0, all = 0;
    for (int k = 0; k < kPlanThreads / 32; ++k) {
      if (k < w) before += tot[k][i];
      all += tot[k][i];
    }
    v[i] = before + x[i] - v[i];
    total[i] = all;
  }
  __syncthreads();
}

// Last b in [0, n) with start[b] <= x (start ascends, start[0] <= x < start[n]).
__device__ __forceinline__ int find_request(const int32_t* start, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x) lo = mid; else hi = mid;
  }
  return lo;
}

// Every CTA sums the requests' lengths itself (a few KB from L2), then fills its share of the rows,
// of the new table entries and of the returned blocks.  With p = free + returned - 1 - i the i-th
// block handed out is stack entry p; returned blocks lie on top and are looked up through their
// seat's table row, so nothing that this call writes is read by it.  The counts are written by the
// CTA that finishes reading last (state_in and state_out may be one buffer).
__global__ void __launch_bounds__(kPlanThreads) ssd_kv8_plan_kernel(const PlanParams p) {
  __shared__ int32_t row_s[SSD_KV8_MAX_BATCH + 1], new_s[SSD_KV8_MAX_BATCH + 1], back_s[SSD_KV8_MAX_BATCH + 1];
  __shared__ int32_t len_s[SSD_KV8_MAX_BATCH], held_s[SSD_KV8_MAX_BATCH], seg_s[SSD_KV8_MAX_BATCH + 1];
  __shared__ int64_t work_s[SSD_KV8_MAX_BATCH + 1];
  __shared__ int64_t tot3[kPlanThreads / 32][3], tot2[kPlanThreads / 32][2];
  __shared__ int last_s, longest_s;
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  const int bs_m1 = (1 << p.shift) - 1;
  const int cap = p.max_blocks << p.shift;
  const int per = (p.batch + kPlanThreads - 1) / kPlanThreads;
  int flags = 0;

  int n_free = p.state_in[0];
  if (n_free < 0 || n_free > p.n_blocks) {
    n_free = n_free < 0 ? 0 : p.n_blocks;
    flags |= SSD_KV8_LENGTH;
  }
  int ln[kPlanPer], ad[kPlanPer], hd[kPlanPer], nw[kPlanPer];
  int64_t sum3[3] = {0, 0, 0}, all3[3];
#pragma unroll
  for (int k = 0; k < kPlanPer; ++k) {
    const int b = tid * per + k;
    ln[k] = ad[k] = hd[k] = nw[k] = 0;
    if (k >= per || b >= p.batch) continue;
    int l = p.len[b], a = p.add[b], h = p.state_in[1 + b];
    if (h < 0 || h > p.max_blocks || l > cap || l < -1 || (l >= 0 && (a < 0 || a > cap - l))) flags |= SSD_KV8_LENGTH;
    h = min(max(h, 0), p.max_blocks);
    a = l < 0 ? 0 : min(max(a, 0), cap);
    ln[k] = l < 0 ? -1 : min(l, cap);
    ad[k] = a;
    hd[k] = h;
    if (l >= 0) nw[k] = max(((min(static_cast<int64_t>(ln[k]) + a, static_cast<int64_t>(cap)) + bs_m1) >> p.shift) - h,
                            static_cast<int64_t>(0));
    sum3[0] += a;
    sum3[1] += nw[k];
    sum3[2] += l < 0 ? h : 0;
  }
  block_scan<3>(sum3, all3, tot3);
  if (all3[0] > p.rows) flags |= SSD_KV8_LENGTH;
  const int n_new = static_cast<int>(all3[1]);
  const int n_back = static_cast<int>(min(all3[2], static_cast<int64_t>(p.n_blocks - n_free)));
  if (all3[2] > n_back) flags |= SSD_KV8_LENGTH;
  const int total = n_free + n_back;
  if (n_new > total) flags |= SSD_KV8_NO_BLOCKS;
  // rows beyond the step's capacity do not exist for it
  int64_t sum2[2] = {0, 0}, all2[2];
  int64_t r = sum3[0], segs[kPlanPer], tiles[kPlanPer];
  int longest = 0;
#pragma unroll
  for (int k = 0; k < kPlanPer; ++k) {
    const int b = tid * per + k;
    segs[k] = tiles[k] = 0;
    if (k >= per || b >= p.batch) continue;
    const int r0 = static_cast<int>(min(r, static_cast<int64_t>(p.rows)));
    r += ad[k];
    const int r1 = static_cast<int>(min(r, static_cast<int64_t>(p.rows)));
    row_s[b] = r0;
    new_s[b] = static_cast<int>(sum3[1]);
    back_s[b] = static_cast<int>(min(sum3[2], static_cast<int64_t>(n_back)));
    sum3[1] += nw[k];
    sum3[2] += ln[k] < 0 ? hd[k] : 0;
    len_s[b] = max(ln[k], 0);
    held_s[b] = ln[k] < 0 ? 0 : hd[k];
    if (b == p.batch - 1) {
      row_s[p.batch] = r1;
      new_s[p.batch] = n_new;
      back_s[p.batch] = n_back;
    }
    const int rows_b = r1 - r0;
    int n = 0;
    if (rows_b > 0) {
      n = static_cast<int>((min(static_cast<int64_t>(max(ln[k], 0)) + rows_b, static_cast<int64_t>(cap)) + 15) >> 4);
      segs[k] = static_cast<int64_t>(p.n_kv_heads) *
                ((static_cast<int64_t>(rows_b) * p.group + p.row_tile - 1) / p.row_tile);
      tiles[k] = segs[k] * n;
    }
    longest = max(longest, n);
    sum2[0] += segs[k];
    sum2[1] += tiles[k];
  }
  if (tid == 0) longest_s = 0;
  block_scan<2>(sum2, all2, tot2);
  if (longest) atomicMax(&longest_s, longest);
  const StepView s = step_view(p.step, p.batch);
#pragma unroll
  for (int k = 0; k < kPlanPer; ++k) {
    const int b = tid * per + k;
    if (k >= per || b >= p.batch) continue;
    seg_s[b] = static_cast<int>(sum2[0]);
    work_s[b] = sum2[1];
    sum2[0] += segs[k];
    sum2[1] += tiles[k];
  }
  if (tid == 0) {
    seg_s[p.batch] = static_cast<int>(all2[0]);
    work_s[p.batch] = all2[1];
  }
  __syncthreads();
  if (blockIdx.x == 0) {
    for (int b = tid; b <= p.batch; b += kPlanThreads) {
      s.seg_start[b] = seg_s[b];
      s.row_start[b] = row_s[b];
      if (b < p.batch) s.len[b] = len_s[b];
    }
    if (flags) atomicOr(p.status, flags);
  }
  if (tid == 0) last_s = atomicAdd(p.ticket, 1) == static_cast<int>(gridDim.x) - 1;
  __syncthreads();

  // the block handed out i-th, or -1
  auto handed = [&](int i) -> int {
    const int q = total - 1 - i;
    if (q < 0) return -1;
    int id;
    if (q >= n_free) {
      const int b = find_request(back_s, p.batch, q - n_free);
      id = p.table[static_cast<size_t>(b) * p.max_blocks + (q - n_free - back_s[b])];
    } else {
      id = p.pool[q];
    }
    if (id < 0 || id >= p.n_blocks) {
      atomicOr(p.status, SSD_KV8_SLOT);
      id = -1;
    }
    return id;
  };
  const int first = blockIdx.x * kPlanThreads + tid, stride = gridDim.x * kPlanThreads;
  int32_t* slot = s.slot;
  const int n_rows = row_s[p.batch];
  for (int64_t r64 = first; r64 < p.rows; r64 += stride) {
    const int row = static_cast<int>(r64);
    int out = -1;
    if (row < n_rows) {
      const int b = find_request(row_s, p.batch, row);
      const int64_t pos = static_cast<int64_t>(len_s[b]) + (row - row_s[b]);
      if (pos < cap) {
        const int j = static_cast<int>(pos >> p.shift);
        int id;
        if (j < held_s[b]) {
          id = p.table[static_cast<size_t>(b) * p.max_blocks + j];
          if (id >= p.n_blocks) {
            atomicOr(p.status, SSD_KV8_SLOT);
            id = -1;
          }
        } else {
          id = handed(new_s[b] + j - held_s[b]);
        }
        if (id >= 0) out = (id << p.shift) + static_cast<int>(pos & bs_m1);
      }
    }
    slot[row] = out;
  }
  for (int64_t i = first; i < n_new; i += stride) {
    const int b = find_request(new_s, p.batch, static_cast<int>(i));
    p.table[static_cast<size_t>(b) * p.max_blocks + held_s[b] + (i - new_s[b])] = handed(static_cast<int>(i));
  }
  // returned blocks that are not handed out again stay on the stack
  for (int64_t i = first; i < min(n_back, total - n_new); i += stride) {
    const int b = find_request(back_s, p.batch, static_cast<int>(i));
    p.pool[n_free + i] = p.table[static_cast<size_t>(b) * p.max_blocks + (i - back_s[b])];
  }
  // ---- the attention's partition
  {
    const int n_segs = seg_s[p.batch];
    const int64_t all = work_s[p.batch];
    const AttnShape sh = attn_shape(p.row_tile);
    const int ctas = kAttnSms * sh.ctas;
    // Short contexts, a CTA for each: one segment per team, whatever its length, so that nothing is
    // merged through global memory (64 tiles take one SM about as long as that merge).
    const bool each = n_segs <= ctas && longest_s <= 64;
    // Else CTAs, unless there are segments for all teams of a smaller size.  Then single warps where
    // segments are short (they share nothing but the states of cut segments), and quarter or half CTAs
    // where they are long, which cut fewer (measured, 8 rows: 640 segments of 42 tiles 34 us with single
    // warps and 38 with four, 512 of 320 tiles 119 and 113 us).
    int W = sh.warps;
    if (!each && n_segs >= ctas) {
      const int small = sh.warps / sh.teams, mid = sh.warps == 12 ? 3 : 4;
      W = all < static_cast<int64_t>(128) * n_segs ? small : mid;
    }
    const int per_cta = sh.warps / W, teams = ctas * per_cta;
    const int64_t span = max((all + teams - 1) / teams, static_cast<int64_t>(4 * W));
    const int64_t snap = span / 4;
    auto request_at = [&](int64_t u) -> int {  // 0 <= u < all
      int lo = 0, hi = p.batch;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (work_s[mid] <= u) lo = mid; else hi = mid;
      }
      return lo;
    };
    auto tiles_of = [&](int b) -> int { return static_cast<int>((work_s[b + 1] - work_s[b]) / (seg_s[b + 1] - seg_s[b])); };
    // Equal spans; a cut inside a segment that is short against the span moves to its nearer end.
    auto cut = [&](int c) -> int64_t {
      const int64_t x = c * span;
      if (x >= all) return all;
      const int b = request_at(x), n = tiles_of(b);
      if (n > snap) return x;
      const int tile = static_cast<int>((x - work_s[b]) % n);
      return tile < n - tile ? x - tile : x - tile + n;
    };
    if (first == 0) *s.head = StepHead{span, W, n_rows, {}};
    for (int i = first; i < ctas * sh.teams; i += stride) {
      const int sub = i % sh.teams, team = i / sh.teams * per_cta + sub;
      TeamSpan t = {};
      if (sub < per_cta) {
        if (each) {
          if (team < n_segs) {
            const int b = find_request(seg_s, p.batch, team), n = tiles_of(b);
            t.u0 = work_s[b] + static_cast<int64_t>(team - seg_s[b]) * n;
            t.u1 = t.u0 + n;
          }
        } else {
          t.u0 = cut(team);
          t.u1 = cut(team + 1);
        }
        if (t.u0 < t.u1) {
          t.b = request_at(t.u0);
          t.n = tiles_of(t.b);
          t.groups = (seg_s[t.b + 1] - seg_s[t.b]) / p.n_kv_heads;
          const int64_t d = t.u0 - work_s[t.b];
          const int seg = static_cast<int>(d / t.n);
          t.tile = static_cast<int>(d - static_cast<int64_t>(seg) * t.n);
          t.head = seg / t.groups;
          t.rg = seg - t.head * t.groups;
          t.row0 = row_s[t.b];
          t.rows = row_s[t.b + 1] - t.row0;
          t.len = len_s[t.b];
        }
      }
      s.teams[i] = t;
    }
  }
  if (last_s) {  // every CTA has read the counts
    if (tid == 0) {
      *p.ticket = 0;
      p.state_out[0] = max(total - n_new, 0);
    }
#pragma unroll
    for (int k = 0; k < kPlanPer; ++k) {
      const int b = tid * per + k;
      if (k >= per || b >= p.batch) continue;
      // as many of its blocks as the stack had
      p.state_out[1 + b] = held_s[b] + min(max(total - new_s[b], 0), new_s[b + 1] - new_s[b]);
    }
    if (p.state_out != p.state_in)
      for (int b = p.batch + tid; b < p.max_batch; b += kPlanThreads) p.state_out[1 + b] = p.state_in[1 + b];
  }
}

// ------------------------------------------------------------------ append

struct AppendParams {
  const void *k, *v;
  int64_t k_row, k_head, v_row, v_head;
  const int32_t* slot;
  int rows, window, shift, n_blocks, n_kv_heads;
  uint8_t* data;   // this layer's
  float* scales;
  int32_t* status;
};

__device__ __forceinline__ int quantise8(float x, float inv) {
  const float q = rintf(x * inv);
  return x != x ? 0 : static_cast<int>(fminf(fmaxf(q, -127.0f), 127.0f));
}

// One warp per (block that the call touches, kv head, K or V): the rows of a block are neighbours, the
// first of them (its predecessor's slot is not one less, or it opens the block) stands for all.
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(128) ssd_kv8_append_kernel(const AppendParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int h = blockIdx.y * 2 + (w >> 1), kv = w & 1;
  if (h >= p.n_kv_heads) return;
  const int bs = 1 << p.shift;
  const T* src = static_cast<const T*>(kv ? p.v : p.k);
  const int64_t row_stride = kv ? p.v_row : p.k_row;
  src += h * (kv ? p.v_head : p.k_head);
  const int64_t r_begin = static_cast<int64_t>(blockIdx.x) * p.window;
  const int r_end = static_cast<int>(min(r_begin + p.window, static_cast<int64_t>(p.rows)));
  int flags = 0;
  for (int r = static_cast<int>(r_begin); r < r_end; ++r) {
    const int s0 = p.slot[r];
    if (s0 < 0) continue;
    if (s0 >= (p.n_blocks << p.shift)) {
      flags |= SSD_KV8_SLOT;
      continue;
    }
    const int off = s0 & (bs - 1);
    if (off != 0 && r > 0 && p.slot[r - 1] == s0 - 1) continue;
    int n = 1;  // rows of this block
    for (int base = 1; base < bs - off; base += 32) {
      const int i = base + lane;
      const bool mine = i < bs - off && r + i < p.rows && p.slot[r + i] == s0 + i;
      const unsigned m = __ballot_sync(~0u, mine);
      const int run = m == ~0u ? 32 : __ffs(~m) - 1;
      n += run;
      if (run < 32) break;
    }
    const size_t rec = static_cast<size_t>(s0 >> p.shift) * p.n_kv_heads + h;
    uint8_t* blk = p.data + rec * (static_cast<size_t>(bs) * 2 * D) + kv * (16 * D);
    float* sc = p.scales + rec * 2 + kv;
    const float s_old = off ? *sc : 0.0f;

    constexpr int D4 = D / 4;
    float amax = 0.0f;
    bool bad = false;
#pragma unroll 4
    for (int c = lane; c < n * D4; c += 32) {
      const float4 x = load4<VEC>(src + (r + c / D4) * row_stride + (c % D4) * 4);
      const float e[4] = {fabsf(x.x), fabsf(x.y), fabsf(x.z), fabsf(x.w)};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool fin = e[i] <= 3.402823466e38f;
        bad |= !fin;
        amax = fmaxf(amax, fin ? e[i] : 0.0f);
      }
    }
    if (bad) flags |= SSD_KV8_NON_FINITE;
    amax = warp_max(amax);
    const float s_new = fmaxf(s_old, fmaxf(amax / 127.0f, 0x1p-100f));
    const float inv = 1.0f / s_new;
    if (off && s_new > s_old) {
      // older tokens of the block; a word may hold later ones too, which are rewritten or stale
      const float ratio = s_old / s_new;
      const int tiles = (off + 15) >> 4;
      for (int i = lane; i < tiles * (4 * D); i += 32) {
        uint32_t* word = reinterpret_cast<uint32_t*>(blk + (i / (4 * D)) * (32 * D) + (i % (4 * D)) * 4);
        const uint32_t old = *word;
        uint32_t now = 0;
#pragma unroll
        for (int b = 0; b < 4; ++b) {
          const int q = static_cast<int>((old >> (8 * b)) & 255u) - 128;
          now |= static_cast<uint32_t>(static_cast<int>(rintf(q * ratio)) + 128) << (8 * b);
        }
        *word = now;
      }
    }
    __syncwarp();
    if (lane == 0) *sc = s_new;
#pragma unroll 4
    for (int c = lane; c < n * D4; c += 32) {
      const float4 x = load4<VEC>(src + (r + c / D4) * row_stride + (c % D4) * 4);
      const int token = off + c / D4, d = (c % D4) * 4;
      const int q[4] = {quantise8(x.x, inv) + 128, quantise8(x.y, inv) + 128, quantise8(x.z, inv) + 128,
                        quantise8(x.w, inv) + 128};
      uint8_t* tile = blk + (token >> 4) * (32 * D);
      if (kv == 0) {
        *reinterpret_cast<uint32_t*>(tile + kv8_k_byte(token & 15, d, D)) = q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) tile[kv8_v_byte(token & 15, d + i)] = static_cast<uint8_t>(q[i]);
      }
    }
    __syncwarp();
  }
  if (flags) atomicOr(p.status, flags);
}

// ------------------------------------------------------------------ read

struct ReadParams {
  const int32_t* slot;
  int n, shift, n_blocks, n_kv_heads;
  const uint8_t* data;
  const float* scales;
  void *k, *v;
  int32_t* status;
};

// One warp per (slot, kv head, K or V).
template <typename T, int D>
__global__ void __launch_bounds__(128) ssd_kv8_read_kernel(const ReadParams p) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int h = blockIdx.y * 2 + (w >> 1), kv = w & 1;
  if (h >= p.n_kv_heads) return;
  const int i = blockIdx.x;
  int s = p.slot[i];
  if (s >= (p.n_blocks << p.shift)) {
    if (lane == 0) atomicOr(p.status, SSD_KV8_SLOT);
    s = -1;
  }
  T* out = static_cast<T*>(kv ? p.v : p.k) + (static_cast<size_t>(i) * p.n_kv_heads + h) * D;
  const int bs = 1 << p.shift, token = s & (bs - 1);
  const size_t rec = static_cast<size_t>(s < 0 ? 0 : s >> p.shift) * p.n_kv_heads + h;
  const uint8_t* tile = p.data + rec * (static_cast<size_t>(bs) * 2 * D) + (token >> 4) * (32 * D) + kv * (16 * D);
  const float sc = s < 0 ? 0.0f : p.scales[rec * 2 + kv];
  for (int d = lane; d < D; d += 32) {
    const int byte = kv ? kv8_v_byte(token & 15, d) : kv8_k_byte(token & 15, d, D);
    out[d] = from_f32<T>(s < 0 ? 0.0f : (static_cast<int>(tile[byte]) - 128) * sc);
  }
}

int log2_of(int bs) { return bs == 16 ? 4 : bs == 32 ? 5 : bs == 64 ? 6 : 7; }

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" {

const char* ssd_op_last_error(void) { return g_op_error; }

int64_t ssd_kv8_data_bytes(const ssd_kv8* c) {
  if (!kv8_shape_ok(c)) return -1;
  return static_cast<int64_t>(c->n_layers) * c->n_blocks * c->n_kv_heads * c->block_tokens * c->head_dim * 2;
}

int64_t ssd_kv8_step_ints(int batch, int rows) {
  if (batch < 1 || batch > SSD_KV8_MAX_BATCH || rows < 0) return -1;
  return SSD_KV8_STEP_HEAD + 3ll * batch + 2 + rows;
}

ssd_status ssd_kv8_plan(const ssd_kv8* c, const ssd_kv8_step* step, const int32_t* len, const int32_t* add,
                        const int32_t* state_in, int32_t* state_out, void* cuda_stream) {
  if (ssd_status s = kv8_check(c, 0)) return s;
  if (ssd_status s = kv8_check_step(c, step)) return s;
  if (!len || !add || !state_in || !state_out) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_plan: null buffer");
  PlanParams p;
  p.batch = step->batch;
  p.rows = step->rows;
  p.max_batch = c->max_batch;
  p.max_blocks = c->max_blocks;
  p.n_blocks = c->n_blocks;
  p.shift = log2_of(c->block_tokens);
  p.n_kv_heads = c->n_kv_heads;
  p.group = c->n_heads / c->n_kv_heads;
  p.row_tile = step_row_tile(c, step);
  p.len = len;
  p.add = add;
  p.state_in = state_in;
  p.state_out = state_out;
  p.table = c->table;
  p.pool = c->pool;
  p.step = step->data;
  p.status = static_cast<int32_t*>(c->work);
  p.ticket = p.status + 1;
  // a thread per team of the attention's partition, or per four rows
  const AttnShape sh = attn_shape(p.row_tile);
  const int teams = (kAttnSms * sh.ctas * sh.teams + kPlanThreads - 1) / kPlanThreads;
  int grid = (step->rows + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
  grid = grid < teams ? teams : grid > kAttnSms ? kAttnSms : grid;
  return op_launch("ssd_kv8_plan", ssd_kv8_plan_kernel, dim3(grid), kPlanThreads, 0,
                   static_cast<cudaStream_t>(cuda_stream), p);
}

ssd_status ssd_kv8_append(const ssd_kv8* c, int layer, const void* k, const void* v, int type, int rows,
                          int64_t k_row_stride, int64_t k_head_stride, int64_t v_row_stride, int64_t v_head_stride,
                          const int32_t* slot, void* cuda_stream) {
  if (ssd_status s = kv8_check(c, layer)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  if (rows < 0) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_append: %d rows", rows);
  if (rows == 0) return SSD_OK;
  if (!k || !v || !slot) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_append: null buffer");
  const int size = type == SSD_TYPE_FP32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) % size)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_append: k and v must be aligned to their elements");
  AppendParams p;
  p.k = k;
  p.v = v;
  p.k_row = k_row_stride;
  p.k_head = k_head_stride;
  p.v_row = v_row_stride;
  p.v_head = v_head_stride;
  p.slot = slot;
  p.rows = rows;
  p.window = rows <= 4096 ? 1 : c->block_tokens;
  p.shift = log2_of(c->block_tokens);
  p.n_blocks = c->n_blocks;
  p.n_kv_heads = c->n_kv_heads;
  const size_t recs = static_cast<size_t>(layer) * c->n_blocks * c->n_kv_heads;
  p.data = static_cast<uint8_t*>(c->data) + recs * c->block_tokens * c->head_dim * 2;
  p.scales = c->scales + recs * 2;
  p.status = static_cast<int32_t*>(c->work);
  const bool vec = aligned4(k, size, k_row_stride, k_head_stride) && aligned4(v, size, v_row_stride, v_head_stride);
  const dim3 grid((rows + p.window - 1) / p.window, (c->n_kv_heads + 1) / 2);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
#define SSD_APPEND(T, D, V) op_launch("ssd_kv8_append", ssd_kv8_append_kernel<T, D, V>, grid, 128, 0, s, p)
#define SSD_APPEND_D(T, V) (c->head_dim == 128 ? SSD_APPEND(T, 128, V) : SSD_APPEND(T, 64, V))
  const ssd_status out = type == SSD_TYPE_FP32 ? (vec ? SSD_APPEND_D(float, true) : SSD_APPEND_D(float, false))
                                               : (vec ? SSD_APPEND_D(__nv_bfloat16, true) : SSD_APPEND_D(__nv_bfloat16, false));
#undef SSD_APPEND_D
#undef SSD_APPEND
  return out;
}

ssd_status ssd_kv8_read(const ssd_kv8* c, int layer, const int32_t* slot, int n, void* k, void* v, int type,
                        void* cuda_stream) {
  if (ssd_status s = kv8_check(c, layer)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  if (n < 0) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_read: %d slots", n);
  if (n == 0) return SSD_OK;
  if (!k || !v || !slot) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_read: null buffer");
  ReadParams p;
  p.slot = slot;
  p.n = n;
  p.shift = log2_of(c->block_tokens);
  p.n_blocks = c->n_blocks;
  p.n_kv_heads = c->n_kv_heads;
  const size_t recs = static_cast<size_t>(layer) * c->n_blocks * c->n_kv_heads;
  p.data = static_cast<const uint8_t*>(c->data) + recs * c->block_tokens * c->head_dim * 2;
  p.scales = c->scales + recs * 2;
  p.k = k;
  p.v = v;
  p.status = static_cast<int32_t*>(c->work);
  const dim3 grid(n, (c->n_kv_heads + 1) / 2);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const char* what = "ssd_kv8_read";
  if (type == SSD_TYPE_FP32)
    return c->head_dim == 128 ? op_launch(what, ssd_kv8_read_kernel<float, 128>, grid, 128, 0, s, p)
                              : op_launch(what, ssd_kv8_read_kernel<float, 64>, grid, 128, 0, s, p);
  return c->head_dim == 128 ? op_launch(what, ssd_kv8_read_kernel<__nv_bfloat16, 128>, grid, 128, 0, s, p)
                            : op_launch(what, ssd_kv8_read_kernel<__nv_bfloat16, 64>, grid, 128, 0, s, p);
}

ssd_status ssd_kv8_status(const ssd_kv8* c, int* bits, void* cuda_stream) {
  if (ssd_status s = kv8_check(c, 0)) return s;
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  int got = 0;
  cudaError_t e = cudaMemcpyAsync(&got, c->work, sizeof(int), cudaMemcpyDeviceToHost, s);
  if (e == cudaSuccess) e = cudaMemsetAsync(c->work, 0, sizeof(int), s);
  if (e == cudaSuccess) e = cudaStreamSynchronize(s);
  if (e != cudaSuccess) return op_fail(SSD_ERR_CUDA, "ssd_kv8_status: %s", cudaGetErrorString(e));
  if (bits) *bits = got;
  if (!got) return SSD_OK;
  return op_fail(SSD_ERR_DEVICE, "8-bit cache:%s%s%s%s", got & SSD_KV8_NO_BLOCKS ? " out of blocks;" : "",
                 got & SSD_KV8_LENGTH ? " a length, row count or block count out of range;" : "",
                 got & SSD_KV8_SLOT ? " a slot or block id outside the cache;" : "",
                 got & SSD_KV8_NON_FINITE ? " a non-finite value appended;" : "");
}

}  // extern "C"
