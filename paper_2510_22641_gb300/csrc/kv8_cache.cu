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
  int n_kv_heads, group, row_tile, dim;
  const int32_t *len, *add, *state_in;
  int32_t *state_out, *table, *pool, *step, *status, *ticket;
};

// Exclusive sums of N values per thread over the CTA; total[] gets the sums.
template <int N, typename I>
__device__ __forceinline__ void block_scan(I (&v)[N], I (&total)[N], I (*tot)[N]) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  I x[N];
#pragma unroll
  for (int i = 0; i < N; ++i) x[i] = v[i];
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const I y = __shfl_up_sync(~0u, x[i], o);
      if (lane >= o) x[i] += y;
    }
  }
  if (lane == 31)
#pragma unroll
    for (int i = 0; i < N; ++i) tot[w][i] = x[i];
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    I before = 0, all = 0;
#pragma unroll
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
// CTA that finishes reading last (state_in and state_out may be one buffer).  Latency bound: a step of 16
// requests 6.1 us, 64 prompts with a slot map of 2 MB 10.8 us.
__global__ void __launch_bounds__(kPlanThreads) ssd_kv8_plan_kernel(const PlanParams p) {
  __shared__ int32_t row_s[SSD_KV8_MAX_BATCH + 1], new_s[SSD_KV8_MAX_BATCH + 1], back_s[SSD_KV8_MAX_BATCH + 1];
  __shared__ int32_t len_s[SSD_KV8_MAX_BATCH], held_s[SSD_KV8_MAX_BATCH], seg_s[SSD_KV8_MAX_BATCH + 1],
      n_s[SSD_KV8_MAX_BATCH];
  __shared__ int64_t work_s[SSD_KV8_MAX_BATCH + 1];
  __shared__ int32_t tot3[kPlanThreads / 32][3];
  __shared__ int64_t tot2[kPlanThreads / 32][2];
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
  int32_t sum3[3] = {0, 0, 0}, all3[3];  // at most max_blocks * block_tokens * max_batch < 2^31
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
  block_scan(sum3, all3, tot3);
  if (all3[0] > p.rows) flags |= SSD_KV8_LENGTH;
  const int n_new = all3[1];
  const int n_back = min(all3[2], p.n_blocks - n_free);
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
    new_s[b] = sum3[1];
    back_s[b] = min(sum3[2], n_back);
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
    n_s[b] = n;
    longest = max(longest, n);
    sum2[0] += segs[k];
    sum2[1] += tiles[k];
  }
  if (tid == 0) longest_s = 0;
  block_scan(sum2, all2, tot2);
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
  // the ticket that says whether all CTAs have read the counts; its answer is awaited at the end
  int ticket = 0;
  if (tid == 0) ticket = atomicAdd(p.ticket, 1);

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
  // Four lists are filled (rows, new table entries, returned blocks, team spans), each from another CTA on,
  // so that for a small step their loads' latencies do not add up.
  const int stride = gridDim.x * kPlanThreads;
  auto begin = [&](int cta) -> int { return (blockIdx.x + gridDim.x - cta) % gridDim.x * kPlanThreads + tid; };
  const int first = begin(0);
  int32_t* slot = s.slot;
  const int n_rows = row_s[p.batch];
  // four rows per thread: usually of one request and one block
  auto block_of = [&](int b, int j) -> int {  // id of the seat's j-th block after this call, or -1
    if (j >= held_s[b]) return handed(new_s[b] + j - held_s[b]);
    const int id = p.table[static_cast<size_t>(b) * p.max_blocks + j];
    if (id < p.n_blocks) return id;
    atomicOr(p.status, SSD_KV8_SLOT);
    return -1;
  };
  const bool quads = (reinterpret_cast<uintptr_t>(slot) & 15) == 0;
  for (int64_t r64 = 4ll * first; r64 < p.rows; r64 += 4ll * stride) {
    const int row = static_cast<int>(r64);
    int out[4] = {-1, -1, -1, -1};
    if (row < n_rows) {
      int b = find_request(row_s, p.batch, row), j = -1, id = -1;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (row + k >= n_rows) break;
        while (row + k >= row_s[b + 1]) ++b, j = -1;
        const int64_t pos = static_cast<int64_t>(len_s[b]) + (row + k - row_s[b]);
        if (pos >= cap) continue;
        const int block = static_cast<int>(pos >> p.shift);
        if (block != j) j = block, id = block_of(b, j);
        if (id >= 0) out[k] = (id << p.shift) + static_cast<int>(pos & bs_m1);
      }
    }
    if (quads && row + 4 <= p.rows) {
      *reinterpret_cast<int4*>(slot + row) = make_int4(out[0], out[1], out[2], out[3]);
    } else {
      for (int k = 0; k < 4 && row + k < p.rows; ++k) slot[row + k] = out[k];
    }
  }
  for (int64_t i = begin(1); i < n_new; i += stride) {
    const int b = find_request(new_s, p.batch, static_cast<int>(i));
    p.table[static_cast<size_t>(b) * p.max_blocks + held_s[b] + (i - new_s[b])] = handed(static_cast<int>(i));
  }
  // returned blocks that are not handed out again stay on the stack
  for (int64_t i = begin(2); i < min(n_back, total - n_new); i += stride) {
    const int b = find_request(back_s, p.batch, static_cast<int>(i));
    p.pool[n_free + i] = p.table[static_cast<size_t>(b) * p.max_blocks + (i - back_s[b])];
  }
  // ---- the attention's partition
  {
    const int n_segs = seg_s[p.batch];
    const int64_t all = work_s[p.batch];
    const AttnShape sh = attn_shape(p.row_tile, p.dim);
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
    // quotient and remainder, in 32 bits where they fit (64-bit division is many times slower)
    auto divide = [](int64_t x, int64_t y, int64_t& rest) -> int64_t {
      if (((x | y) >> 32) == 0) {
        const uint32_t q = static_cast<uint32_t>(x) / static_cast<uint32_t>(y);
        rest = static_cast<uint32_t>(x) - q * static_cast<uint32_t>(y);
        return q;
      }
      rest = x % y;
      return x / y;
    };
    int64_t rest;
    // Segments of up to four tiles a warp are not cut, and spans are no shorter, but where every segment is.
    const int64_t few = min(4 * W, longest_s);
    const int64_t span = max(divide(all + teams - 1, teams, rest), few);
    const int64_t snap = max(span / 4, few);
    auto request_at = [&](int64_t u) -> int {  // 0 <= u < all
      int lo = 0, hi = p.batch;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (work_s[mid] <= u) lo = mid; else hi = mid;
      }
      return lo;
    };
    // Equal spans; a cut inside a segment that is short against the span moves to its nearer end.
    auto cut = [&](int c) -> int64_t {
      const int64_t x = c * span;
      if (x >= all) return all;
      const int b = request_at(x), n = n_s[b];
      if (n > snap) return x;
      int64_t tile;
      divide(x - work_s[b], n, tile);
      return tile < n - tile ? x - tile : x - tile + n;
    };
    if (first == 0) *s.head = StepHead{span, W, n_rows, {}};
    for (int i = begin(3); i < ctas * sh.teams; i += stride) {
      const int sub = i % sh.teams, team = i / sh.teams * per_cta + sub;
      TeamSpan t = {};
      if (sub < per_cta) {
        if (each) {
          if (team < n_segs) {
            const int b = find_request(seg_s, p.batch, team), n = n_s[b];
            t.u0 = work_s[b] + static_cast<int64_t>(team - seg_s[b]) * n;
            t.u1 = t.u0 + n;
          }
        } else {
          t.u0 = cut(team);
          t.u1 = cut(team + 1);
        }
        if (t.u0 < t.u1) {
          t.b = request_at(t.u0);
          t.n = n_s[t.b];
          t.groups = (seg_s[t.b + 1] - seg_s[t.b]) / p.n_kv_heads;
          int64_t tile;
          const int seg = static_cast<int>(divide(t.u0 - work_s[t.b], t.n, tile));
          t.tile = static_cast<int>(tile);
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
  if (tid == 0) last_s = ticket == static_cast<int>(gridDim.x) - 1;
  __syncthreads();
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
  int rows, takers, shift, n_blocks, n_kv_heads;  // takers: CTAs that share a window of rows
  uint8_t* data;   // this layer's
  float* scales;
  int32_t* status;
};

// Codes plus 128 of four values as bytes.  The product is rounded to fp32, then the addition of
// 1.5 2^23 + 128 rounds it to an integer (ties to even) whose low byte is the code: |x inv| <= 127.5 here.
__device__ __forceinline__ uint32_t code8(float x, float inv) { return __float_as_uint(__fadd_rn(__fmul_rn(x, inv), 12583040.0f)); }
__device__ __forceinline__ uint32_t pack4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
// The same for values that may be NaN (code 0) or infinite (the largest code).  The product is clamped, not the
// value: 127 times the scale of the largest fp32 values rounds to infinity.
__device__ __forceinline__ uint32_t code8_any(float x, float inv) {
  return code8(x != x ? 0.0f : fminf(fmaxf(__fmul_rn(x, inv), -127.0f), 127.0f), 1.0f);
}
// The four codes of a word at a scale `ratio` times as large.
__device__ __forceinline__ uint32_t rescale8(uint32_t word, float ratio) {
  uint32_t q[4];
#pragma unroll
  for (int b = 0; b < 4; ++b) q[b] = code8(static_cast<float>(static_cast<int>(word >> (8 * b) & 255u) - 128), ratio);
  return pack4(q[0], q[1], q[2], q[3]);
}
// Maximum that keeps a NaN.
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}

// E consecutive elements of a row, as they lie in memory.
template <typename T, int E>
struct Piece {
  uint32_t w[E * sizeof(T) / 4];
  template <bool VEC>
  __device__ __forceinline__ void load(const T* p) {
    if constexpr (!VEC) {
      T e[E];
#pragma unroll
      for (int i = 0; i < E; ++i) e[i] = p[i];
#pragma unroll
      for (int i = 0; i < E * static_cast<int>(sizeof(T)) / 4; ++i) w[i] = reinterpret_cast<const uint32_t*>(e)[i];
    } else if constexpr (sizeof(w) == 16) {
      const uint4 v = *reinterpret_cast<const uint4*>(p);
      w[0] = v.x, w[1] = v.y, w[2] = v.z, w[3] = v.w;
    } else if constexpr (sizeof(w) == 8) {
      const uint2 v = *reinterpret_cast<const uint2*>(p);
      w[0] = v.x, w[1] = v.y;
    } else {
      w[0] = *reinterpret_cast<const uint32_t*>(p);
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (uint32_t& x : w) x = 0;
  }
  __device__ __forceinline__ float operator[](int i) const {
    if constexpr (sizeof(T) == 4) return __uint_as_float(w[i]);
    else return i & 1 ? __uint_as_float(w[i / 2] & 0xffff0000u) : __uint_as_float(w[i / 2] << 16);
  }
};

// Decode steps: few rows per block.  One warp per (row that stands for a block, kv head, K or V), which
// takes the rows of the block that follow it; the lanes go over (row, 4 dimensions).  Latency bound: the
// rows are read twice (the second time from L1) so that a warp needs few registers and all are resident.
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(128) ssd_kv8_append_rows_kernel(const AppendParams p) {
  constexpr int D4 = D / 4;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int h = blockIdx.y * 2 + (w >> 1), kv = w & 1, r = blockIdx.x;
  if (h >= p.n_kv_heads) return;
  const int bs = 1 << p.shift;
  // the slots from the row before on: one load shows whether this row stands for its block, and which follow
  const int at = r - 1 + lane;
  int s = at >= 0 && at < p.rows ? p.slot[at] : -1;
  const int before = __shfl_sync(~0u, s, 0), s0 = __shfl_sync(~0u, s, 1);
  if (s0 < 0) return;
  if (s0 >= p.n_blocks << p.shift) {
    if (lane == 0) atomicOr(p.status, SSD_KV8_SLOT);
    return;
  }
  const int off = s0 & (bs - 1);
  if (off != 0 && r > 0 && before == s0 - 1) return;
  unsigned m = __ballot_sync(~0u, lane > 0 && s == s0 + lane - 1 && off + lane - 1 < bs) >> 1;
  int n = m == 0x7fffffffu ? 31 : __ffs(~m) - 1;  // rows of this block
  for (int base = 31; n == base && base < bs - off; base += 32) {
    const int i = base + lane;
    m = __ballot_sync(~0u, i < bs - off && r + i < p.rows && p.slot[r + i] == s0 + i);
    n += m == ~0u ? 32 : __ffs(~m) - 1;
  }
  const T* src = static_cast<const T*>(kv ? p.v : p.k) + h * (kv ? p.v_head : p.k_head) + r * (kv ? p.v_row : p.k_row);
  const int64_t row_stride = kv ? p.v_row : p.k_row;
  const size_t rec = static_cast<size_t>(s0 >> p.shift) * p.n_kv_heads + h;
  uint8_t* blk = p.data + rec * (static_cast<size_t>(bs) * 2 * D) + kv * (16 * D);
  float* sc = p.scales + rec * 2 + kv;
  const float s_old = off ? *sc : 0.0f;

  float amax = 0.0f;
  bool bad = false;
#pragma unroll 4
  for (int c = lane; c < n * D4; c += 32) {
    const float4 x = load4<VEC>(src + c / D4 * row_stride + c % D4 * 4);
    const float e[4] = {fabsf(x.x), fabsf(x.y), fabsf(x.z), fabsf(x.w)};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool fin = e[i] <= 3.402823466e38f;
      bad |= !fin;
      amax = fmaxf(amax, fin ? e[i] : 0.0f);
    }
  }
  if (bad) atomicOr(p.status, SSD_KV8_NON_FINITE);
  amax = warp_max(amax);
  const float s_new = fmaxf(s_old, fmaxf(amax / 127.0f, 0x1p-100f));
  const float inv = 1.0f / s_new;
  if (off && s_new > s_old) {
    // older tokens of the block; a word may hold later ones too, which are rewritten or stale
    const float ratio = s_old / s_new;
    const int tiles = (off + 15) >> 4;
#pragma unroll 4
    for (int i = lane; i < tiles * (4 * D); i += 32) {
      uint32_t* word = reinterpret_cast<uint32_t*>(blk + i / (4 * D) * (32 * D) + i % (4 * D) * 4);
      *word = rescale8(*word, ratio);
    }
  }
  __syncwarp();
  if (lane == 0) *sc = s_new;
#pragma unroll 4
  for (int c = lane; c < n * D4; c += 32) {
    const float4 x = load4<VEC>(src + c / D4 * row_stride + c % D4 * 4);
    const int token = off + c / D4, d = c % D4 * 4;
    const uint32_t q[4] = {code8_any(x.x, inv), code8_any(x.y, inv), code8_any(x.z, inv), code8_any(x.w, inv)};
    uint8_t* tile = blk + (token >> 4) * (32 * D);
    if (kv == 0) {
      *reinterpret_cast<uint32_t*>(tile + kv8_k_byte(token & 15, d, D)) = pack4(q[0], q[1], q[2], q[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) tile[kv8_v_byte(token & 15, d + i)] = static_cast<uint8_t>(q[i]);
    }
  }
}

// The entries of a window of a slot list that begin a run (consecutive slots, cut where a slot is a
// multiple of `cut`), listed by the whole CTA of 8 warps (a ballot per 32 entries).  A run that began in
// the window before is that window's, and negative entries or ones past the cache are none; with `all`
// the window's first entry begins a run, and each such entry is one.  Returns how many; flags bad slots.
constexpr int kWindow = 512;

struct Runs {
  uint16_t first[kWindow];  // index in the window
  int32_t slot[kWindow];    // its slot
  int count[kWindow / 32];
};

__device__ __forceinline__ int list_runs(Runs& runs, const int32_t* slot, int begin, int end, int most, int cut, bool all,
                                         int& flags) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  unsigned mine[2];
  int own[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = begin + (w + 8 * i) * 32 + lane;
    const int s = r < end ? slot[r] : -1;
    own[i] = s;
    if (s >= most) flags |= SSD_KV8_SLOT;
    const bool in = s >= 0 && s < most;
    const bool starts = in ? (s & (cut - 1)) == 0 || r == 0 || (all && r == begin) || slot[r - 1] != s - 1 : all;
    mine[i] = __ballot_sync(~0u, r < end && starts);
    if (lane == 0) runs.count[w + 8 * i] = __popc(mine[i]);
  }
  __syncthreads();
  int total = 0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    int before = 0;
    total = 0;
#pragma unroll
    for (int k = 0; k < kWindow / 32; ++k) {
      before += k < w + 8 * i ? runs.count[k] : 0;
      total += runs.count[k];
    }
    if (mine[i] >> lane & 1u) {
      const int o = before + __popc(mine[i] & ((1u << lane) - 1));
      runs.first[o] = static_cast<uint16_t>((w + 8 * i) * 32 + lane);
      runs.slot[o] = own[i];
    }
  }
  __syncthreads();
  return total;
}

// A job is the rows that the call puts into one block, for one kv head and K or V: the rows of a block
// are neighbours, and the first of them (its predecessor's slot is not one less, or it opens the block)
// stands for all.  Each 16-token tile of the block has a warp, which holds the tile's new values in
// registers between the maximum and the rounding (a lane D / 32 dimensions of all 16 tokens), so rows
// are read once.  A word of V holds four tokens of one dimension: where old tokens share it with new
// ones, or the scale has grown, it is read first.
//
// Prompts; bound: bytes.  A CTA of 8 warps takes 8 / (block / 16) jobs at a time and every `takers`-th of
// its window's blocks, so that rows that stand for none cost nothing.  43,565 rows of 8 prompts, 8 heads,
// bf16: 74 us, 41 % of the DRAM rate (16 warps an SM: a tile's values take 64 registers).
template <typename T, int D, bool VEC>
__global__ void __launch_bounds__(256, 2) ssd_kv8_append_kernel(const AppendParams p) {
  constexpr int E = D / 32;
  __shared__ Runs runs;
  __shared__ float amax_s[8];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int bs = 1 << p.shift, log_tiles = p.shift - 4, tiles = 1 << log_tiles;
  const int job = (blockIdx.y * 8 + w) >> log_tiles, tile = w & (tiles - 1);
  const int h = job >> 1, kv = job & 1;
  const bool live = h < p.n_kv_heads;  // a warp without a job still takes part in the barriers
  const T* src = static_cast<const T*>(kv ? p.v : p.k) + lane * E;
  const int64_t row_stride = kv ? p.v_row : p.k_row;
  if (live) src += h * (kv ? p.v_head : p.k_head);
  const int window = blockIdx.x / p.takers, taker = blockIdx.x - window * p.takers;
  const int r_begin = window * kWindow, r_end = min(r_begin + kWindow, p.rows);
  int flags = 0;
  const int total = list_runs(runs, p.slot, r_begin, r_end, p.n_blocks << p.shift, bs, false, flags);

  for (int o = taker; o < total; o += p.takers) {  // the same for all warps of the CTA
    const int r = r_begin + runs.first[o];
    const int s0 = runs.slot[o], off = s0 & (bs - 1);
    const size_t rec = static_cast<size_t>(s0 >> p.shift) * p.n_kv_heads + (live ? h : 0);
    float* sc = p.scales + rec * 2 + kv;
    const float s_old = off ? *sc : 0.0f;
    int n = 0;  // rows that go on in this block
    for (int base = 0; base < bs - off; base += 32) {
      const int i = base + lane;
      const unsigned m = __ballot_sync(~0u, i < bs - off && r + i < p.rows && p.slot[r + i] == s0 + i);
      n += m == ~0u ? 32 : __ffs(~m) - 1;
      if (m != ~0u) break;
    }
    // tokens first .. last - 1 of the tile are new, those before them older (16: all of the tile)
    const int first = min(max(off - 16 * tile, 0), 16), last = live ? min(off + n - 16 * tile, 16) : 0;
    const T* rows = src + (r + 16 * tile - off) * row_stride;  // token i at rows + i * row_stride
    Piece<T, E> x[16];
    float amax = 0.0f;
    bool full = first == 0 && last == 16;
    if (full) {
#pragma unroll
      for (int i = 0; i < 16; ++i) x[i].template load<VEC>(rows + i * row_stride);
#pragma unroll
      for (int i = 0; i < 16; ++i)
#pragma unroll
        for (int e = 0; e < E; ++e) amax = max_nan(amax, fabsf(x[i][e]));
      full = !__any_sync(~0u, !(amax <= 3.402823466e38f));
    }
    if (!full) {  // part of a tile, or one with NaN or infinities
      amax = 0.0f;
      bool bad = false;
#pragma unroll 4
      for (int i = first; i < last; ++i) {
        Piece<T, E> y;
        y.template load<VEC>(rows + i * row_stride);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float a = fabsf(y[e]);
          const bool fin = a <= 3.402823466e38f;
          bad |= !fin;
          amax = fmaxf(amax, fin ? a : 0.0f);
        }
      }
      if (bad) flags |= SSD_KV8_NON_FINITE;
    }
    amax = warp_max(amax);
    if (tiles > 1) {
      if (lane == 0) amax_s[w] = amax;
      __syncthreads();
      for (int i = 0; i < tiles; ++i) amax = fmaxf(amax, amax_s[(w & ~(tiles - 1)) + i]);
      __syncthreads();  // before the next block's maxima
    }
    if (!live) continue;
    const float s_new = fmaxf(s_old, fmaxf(amax / 127.0f, 0x1p-100f));
    const float inv = 1.0f / s_new;
    // (every warp of the job has read the old scale before the barrier; a block of one tile is one warp's)
    __syncwarp();
    if (tile == 0 && lane == 0) *sc = s_new;
    uint8_t* dst = p.data + rec * (static_cast<size_t>(bs) * 2 * D) + tile * (32 * D) + kv * (16 * D);
    if (full) {
      auto code = [&](int i, int e) -> uint32_t { return code8(x[i][e], inv); };
      if (kv == 0) {
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          uint8_t* at = dst + kv8_k_byte(i, lane * E, D);
          if constexpr (E == 4) *reinterpret_cast<uint32_t*>(at) = pack4(code(i, 0), code(i, 1), code(i, 2), code(i, 3));
          else *reinterpret_cast<uint16_t*>(at) = static_cast<uint16_t>(__byte_perm(code(i, 0), code(i, 1), 0x0040));
        }
      } else {
#pragma unroll
        for (int t = 0; t < 4; ++t)
#pragma unroll
          for (int e = 0; e < E; ++e)
            *reinterpret_cast<uint32_t*>(dst + kv8_v_byte(4 * t, lane * E + e)) =
                pack4(code(4 * t, e), code(4 * t + 1, e), code(4 * t + 2, e), code(4 * t + 3, e));
      }
      continue;
    }
    const bool grown = off && s_new > s_old;
    const float ratio = s_old / s_new;
    if (kv == 0) {
#pragma unroll 4
      for (int i = grown ? 0 : first; i < max(first, last); ++i) {
        uint8_t* at = dst + kv8_k_byte(i, lane * E, D);
        uint32_t word;
        if (i < first) {
          if constexpr (E == 4) word = *reinterpret_cast<const uint32_t*>(at);
          else word = *reinterpret_cast<const uint16_t*>(at);
          word = rescale8(word, ratio);
        } else {
          Piece<T, E> y;
          y.template load<VEC>(rows + i * row_stride);
          word = 0;
#pragma unroll
          for (int e = 0; e < E; ++e) word |= (code8_any(y[e], inv) & 255u) << (8 * e);
        }
        if constexpr (E == 4) *reinterpret_cast<uint32_t*>(at) = word;
        else *reinterpret_cast<uint16_t*>(at) = static_cast<uint16_t>(word);
      }
    } else {
#pragma unroll 1
      for (int t = 0; t < 4; ++t) {
        const bool has_new = 4 * t + 3 >= first && 4 * t < last;
        if (!has_new && !(grown && 4 * t < first)) continue;
        uint32_t word[E], put = 0;  // the bytes of new tokens
#pragma unroll
        for (int e = 0; e < E; ++e) word[e] = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (4 * t + i >= first && 4 * t + i < last) {
            Piece<T, E> y;
            y.template load<VEC>(rows + (4 * t + i) * row_stride);
            put |= 255u << (8 * i);
#pragma unroll
            for (int e = 0; e < E; ++e) word[e] |= (code8_any(y[e], inv) & 255u) << (8 * i);
          }
#pragma unroll
        for (int e = 0; e < E; ++e) {
          uint32_t* at = reinterpret_cast<uint32_t*>(dst + kv8_v_byte(4 * t, lane * E + e));
          uint32_t old = *at;
          if (grown) old = rescale8(old, ratio);
          *at = (old & ~put) | word[e];
        }
      }
    }
  }
  if (flags) atomicOr(p.status, flags);
}

// ------------------------------------------------------------------ read

struct ReadParams {
  const int32_t* slot;
  int n, takers, shift, n_blocks, n_kv_heads;
  const uint8_t* data;
  const float* scales;
  void *k, *v;
  int32_t* status;
};

template <typename T, int E>
__device__ __forceinline__ void store_row(T* p, const float (&x)[E]) {
  if constexpr (sizeof(T) == 4) {
    if constexpr (E == 4) *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
    else *reinterpret_cast<float2*>(p) = make_float2(x[0], x[1]);
  } else {
    __nv_bfloat162 h[E / 2];
#pragma unroll
    for (int i = 0; i < E / 2; ++i) h[i] = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    if constexpr (E == 4) *reinterpret_cast<uint2*>(p) = *reinterpret_cast<const uint2*>(h);
    else *reinterpret_cast<uint32_t*>(p) = *reinterpret_cast<const uint32_t*>(h);
  }
}

// The value of byte `b` of a word: the byte goes into the mantissa of 2^23.
__device__ __forceinline__ float value8(uint32_t word, int b, float scale) {
  return (__uint_as_float(__byte_perm(word, 0x4b000000u, 0x7440 + b)) - 8388736.0f) * scale;
}

// A warp per run of slots inside a 16-token tile (list_runs), kv head and K or V.  Bound: bytes, mostly
// those written: the same rows 44 us, 62 % of the DRAM rate.
template <typename T, int D>
__global__ void __launch_bounds__(256, 3) ssd_kv8_read_kernel(const ReadParams p) {
  constexpr int E = D / 32;
  __shared__ Runs runs;
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int bs = 1 << p.shift, most = p.n_blocks << p.shift;
  const int window = blockIdx.x / p.takers, taker = blockIdx.x - window * p.takers;
  const int i_begin = window * kWindow, i_end = min(i_begin + kWindow, p.n);
  int flags = 0;
  const int total = list_runs(runs, p.slot, i_begin, i_end, most, 16, true, flags);
  if (flags) atomicOr(p.status, flags);
  const int h = blockIdx.y * 4 + (w >> 1), kv = w & 1;
  if (h >= p.n_kv_heads) return;
  const size_t row = static_cast<size_t>(p.n_kv_heads) * D;
  T* out0 = static_cast<T*>(kv ? p.v : p.k) + static_cast<size_t>(h) * D + lane * E;
#pragma unroll 1
  for (int o = taker; o < total; o += p.takers) {
    const int i0 = i_begin + runs.first[o], n = (o + 1 < total ? i_begin + runs.first[o + 1] : i_end) - i0;
    T* out = out0 + i0 * row;
    const int s0 = runs.slot[o];
    float x[E];
    if (s0 < 0 || s0 >= most) {
#pragma unroll
      for (int e = 0; e < E; ++e) x[e] = 0.0f;
      store_row<T, E>(out, x);  // an entry of its own
      continue;
    }
    const size_t rec = static_cast<size_t>(s0 >> p.shift) * p.n_kv_heads + h;
    const uint8_t* tile = p.data + rec * (static_cast<size_t>(bs) * 2 * D) + ((s0 & (bs - 1)) >> 4) * (32 * D) + kv * (16 * D);
    const float scale = p.scales[rec * 2 + kv];
    // the whole tile's words, whatever part of it is asked for: all loads are in flight at once
    const int t0 = s0 & 15;
    T* base = out - t0 * static_cast<int64_t>(row);
    uint32_t word[4 * E];  // K: token by token (E == 2: two tokens a word); V: four tokens of a dimension
    if (kv) {
#pragma unroll
      for (int j = 0; j < 4 * E; ++j) word[j] = *reinterpret_cast<const uint32_t*>(tile + kv8_v_byte(4 * (j / E), lane * E + j % E));
#pragma unroll
      for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = value8(word[i / 4 * E + e], i & 3, scale);
        if (i >= t0 && i < t0 + n) store_row<T, E>(base + i * row, x);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const uint8_t* at = tile + kv8_k_byte(i, lane * E, D);
        if constexpr (E == 4) word[i] = *reinterpret_cast<const uint32_t*>(at);
        else if (i % 2 == 0) word[i / 2] = *reinterpret_cast<const uint16_t*>(at);
        else word[i / 2] |= static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(at)) << 16;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
#pragma unroll
        for (int e = 0; e < E; ++e) x[e] = E == 4 ? value8(word[i], e, scale) : value8(word[i / 2], i % 2 * 2 + e, scale);
        if (i >= t0 && i < t0 + n) store_row<T, E>(base + i * row, x);
      }
    }
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
  p.dim = c->head_dim;
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
  const AttnShape sh = attn_shape(p.row_tile, p.dim);
  const int teams = (kAttnSms * sh.ctas * sh.teams + kPlanThreads - 1) / kPlanThreads;
  int grid = (step->rows + 4 * kPlanThreads - 1) / (4 * kPlanThreads);
  grid = grid < teams + 3 ? teams + 3 : grid > kAttnSms ? kAttnSms : grid;
  return op_launch("ssd_kv8_plan", ssd_kv8_plan_kernel, dim3(grid), kPlanThreads, 0,
                   static_cast<cudaStream_t>(cuda_stream), p);
}

ssd_status ssd_kv8_append(const ssd_kv8* c, int layer, const void* k, const void* v, int type, int rows,
                          int64_t k_row_stride, int64_t k_head_stride, int64_t v_row_stride, int64_t v_head_stride,
                          const int32_t* slot, void* cuda_stream) {
  if (ssd_status s = kv8_check(c, layer)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  if (rows < 0 || rows > 1 << 30) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_append: %d rows", rows);
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
  // as many CTAs per window as blocks may begin in it: every block_tokens rows, and with each request (the call
  // does not know how many there are: at most one a seat)
  const int in_window = rows < kWindow ? rows : kWindow;
  p.takers = static_cast<int>(in_window / c->block_tokens + static_cast<int64_t>(c->max_batch) * in_window / rows + 1);
  p.shift = log2_of(c->block_tokens);
  p.n_blocks = c->n_blocks;
  p.n_kv_heads = c->n_kv_heads;
  const size_t recs = static_cast<size_t>(layer) * c->n_blocks * c->n_kv_heads;
  p.data = static_cast<uint8_t*>(c->data) + recs * c->block_tokens * c->head_dim * 2;
  p.scales = c->scales + recs * 2;
  p.status = static_cast<int32_t*>(c->work);
  const bool vec = aligned4(k, size, k_row_stride, k_head_stride) && aligned4(v, size, v_row_stride, v_head_stride);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  // A warp per row and head where rows of a block are few; a warp per 16 tokens of a block else.  The call knows
  // its rows but not its requests, so the rule takes the seats for them: at most the 16 rows of a decode step
  // for each.  Where every seat takes part that is right: 62 rows of 16 requests, 40 heads, blocks of 32 take 4.9
  // and 22 us, a prompt of 640 rows in a cache of one seat, 32 heads, blocks of 64, 42 and 7.1 us.  A prompt of
  // up to 16 rows a seat in a cache of many gets the slow one: those 640 rows take 9.1 us with 16 seats, 42 us
  // with 64 or more.
  const bool few = rows <= SSD_MAX_ROWS * c->max_batch;
  const int per_cta = 128 / c->block_tokens;  // jobs
  const dim3 grid = few ? dim3(rows, (c->n_kv_heads + 1) / 2)
                        : dim3((rows + kWindow - 1) / kWindow * p.takers, (2 * c->n_kv_heads + per_cta - 1) / per_cta);
#define SSD_APPEND(T, D, V) (few ? op_launch("ssd_kv8_append", ssd_kv8_append_rows_kernel<T, D, V>, grid, 128, 0, s, p) \
                             : op_launch("ssd_kv8_append", ssd_kv8_append_kernel<T, D, V>, grid, 256, 0, s, p))
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
  if (n < 0 || n > 1 << 30) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_read: %d slots", n);
  if (n == 0) return SSD_OK;
  if (!k || !v || !slot) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_read: null buffer");
  if ((reinterpret_cast<uintptr_t>(k) | reinterpret_cast<uintptr_t>(v)) % 16)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_read: k and v must be 16-byte aligned");
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
  // a tile per warp where that fills the GPU no more than once (latency), else four
  const int in_window = n < kWindow ? n : kWindow;
  p.takers = n <= 4096 ? in_window / 16 + 1 : in_window / 64;
  const dim3 grid((n + kWindow - 1) / kWindow * p.takers, (c->n_kv_heads + 3) / 4);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  const char* what = "ssd_kv8_read";
  if (type == SSD_TYPE_FP32)
    return c->head_dim == 128 ? op_launch(what, ssd_kv8_read_kernel<float, 128>, grid, 256, 0, s, p)
                              : op_launch(what, ssd_kv8_read_kernel<float, 64>, grid, 256, 0, s, p);
  return c->head_dim == 128 ? op_launch(what, ssd_kv8_read_kernel<__nv_bfloat16, 128>, grid, 256, 0, s, p)
                            : op_launch(what, ssd_kv8_read_kernel<__nv_bfloat16, 64>, grid, 256, 0, s, p);
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
