// Shared definitions of the low-bit operators (paged 8-bit K/V cache, 4-bit weights): the byte
// order of a cache tile, typed loads and stores, and the context-free error message.
#pragma once

#include <cuda_fp16.h>

#include <atomic>

#include "common.cuh"

namespace ssd {

// Records the calling thread's message (a fixed buffer: nothing here throws) and returns `s`.
ssd_status op_fail(ssd_status s, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
// Raises a kernel's shared-memory limit, once per device (`ready`: a bit for each).
template <typename K>
ssd_status op_smem(K* kernel, int bytes, std::atomic<uint64_t>& ready, const char* what) {
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  const uint64_t bit = 1ull << (dev & 63);
  if (e == cudaSuccess && ready.load(std::memory_order_relaxed) & bit) return SSD_OK;
  if (e == cudaSuccess)
    e = cudaFuncSetAttribute(reinterpret_cast<const void*>(kernel), cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
  if (e != cudaSuccess) return op_fail(SSD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
  ready.fetch_or(bit, std::memory_order_relaxed);
  return SSD_OK;
}
// Launch that may begin while the launch before it drains: every kernel launched so waits for that one
// (griddepcontrol.wait) before it touches memory, and lets the next begin early.
template <typename... P, typename... A>
ssd_status op_launch(const char* what, void (*kernel)(P...), dim3 grid, int threads, int smem, cudaStream_t s, A... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute at[1];
  at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = at;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, args...);
  return e == cudaSuccess ? SSD_OK : op_fail(SSD_ERR_CUDA, "%s: %s", what, cudaGetErrorString(e));
}
// The status of a launch that has just been made.
ssd_status op_launched(const char* what);

// ------------------------------------------------------------------ operands that share memory

// Elements p + r * row + h * head + [0, width) of a buffer, r < rows, h < heads.
struct OpRows {
  const void* p;
  int64_t rows, heads, row, head, width;
};
// Whether two of them, of elements of `size` bytes, share an element.  Almost always the address ranges are apart;
// else rows that lie between each other (slices of one buffer) are told from rows that overlap.
inline bool op_overlap(OpRows a, OpRows b, int size) {
  using Int = __int128;
  auto span = [](const OpRows& x, Int& lo, Int& hi) {  // elements from x.p on
    const Int r = static_cast<Int>(x.rows - 1) * x.row, h = static_cast<Int>(x.heads - 1) * x.head;
    lo = (r < 0 ? r : 0) + (h < 0 ? h : 0);
    hi = (r > 0 ? r : 0) + (h > 0 ? h : 0) + x.width;
  };
  Int alo, ahi, blo, bhi;
  span(a, alo, ahi);
  span(b, blo, bhi);
  const Int delta = (static_cast<Int>(reinterpret_cast<uintptr_t>(b.p)) - reinterpret_cast<uintptr_t>(a.p)) / size;
  if (delta + bhi <= alo || ahi <= delta + blo) return false;
  for (OpRows* x : {&a, &b})
    if (x->head == x->width) x->width *= x->heads, x->heads = 1, x->head = 0;  // one piece per row
  // whether -b.width < c + r * s < a.width for a whole r in [lo, hi]
  auto meets = [&](Int c, Int s, Int lo, Int hi) -> bool {
    if (s < 0) {
      s = -s;
      const Int t = lo;
      lo = -hi, hi = -t;
    }
    if (s == 0) return lo <= hi && -b.width < c && c < a.width;
    auto floor_div = [](Int x, Int y) -> Int { return x / y - (x % y < 0 ? 1 : 0); };  // y > 0
    const Int first = floor_div(-b.width - c, s) + 1, last = -floor_div(c - a.width, s) - 1;
    return (first > lo ? first : lo) <= (last < hi ? last : hi);
  };
  if (a.row == b.row && a.head == b.head) {  // differences of rows and heads
    for (int64_t h = 1 - a.heads; h < b.heads; ++h)
      if (meets(delta + static_cast<Int>(h) * a.head, a.row, 1 - a.rows, b.rows - 1)) return true;
    return false;
  }
  for (int64_t r = 0; r < a.rows; ++r)
    for (int64_t h = 0; h < a.heads; ++h)
      for (int64_t g = 0; g < b.heads; ++g)
        if (meets(delta + static_cast<Int>(g) * b.head - static_cast<Int>(h) * a.head - static_cast<Int>(r) * a.row, b.row,
                  0, b.rows - 1))
          return true;
  return false;
}

// ------------------------------------------------------------------ cache layout
//
// A tile is 16 tokens of one block and kv head: 16 * D bytes of K, then 16 * D of V, a code c
// held as the byte c + 128.  With mma.m16n8k16 a lane (g = lane / 4, t = lane % 4) needs, of K, the
// keys of matrix rows g and g + 8 at four dimensions per 16-wide step, and of V, four keys at the
// dimensions g and g + 8 of each 16.  Both are kept as one 4-byte word per lane and step, a lane's
// words in 16-byte chunks, the 32 lanes' chunks next to each other: every 16-byte load of a warp is
// one contiguous 512 bytes, and a lane reads back from shared memory the bytes it copied itself.
//
// Matrix row r of the score tile is token tile_token(r); the inverse is below.  Row r and r + 1
// (r even) and r + 8, r + 9 are four consecutive tokens, which is what lets a V word hold them.

constexpr int kTileTokens = 16;

__host__ __device__ constexpr int kv8_tile_token(int r) {  // matrix row -> token of the tile
  return 4 * ((r & 7) >> 1) + 2 * (r >> 3) + (r & 1);
}

// Byte of (token, dim) in the K half (resp. V half) of a tile.
__host__ __device__ __forceinline__ constexpr int kv8_k_byte(int token, int d, int dim) {
  const int row = 2 * (token >> 2) + (token & 1);  // matrix row modulo 8
  const int j = (token >> 1) & 1;                  // 1: rows 8..15
  const int word = j * (dim / 16) + (d >> 4);
  const int lane = row * 4 + ((d >> 2) & 3);
  return (word >> 2) * 512 + lane * 16 + (word & 3) * 4 + (d & 3);
}
__host__ __device__ __forceinline__ constexpr int kv8_v_byte(int token, int d) {
  const int word = d >> 3;
  const int lane = (d & 7) * 4 + (token >> 2);
  return (word >> 2) * 512 + lane * 16 + (word & 3) * 4 + (token & 3);
}

// ------------------------------------------------------------------ typed access

template <typename T>
__device__ __forceinline__ float to_f32(T v);
template <>
__device__ __forceinline__ float to_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }

template <typename T>
__device__ __forceinline__ T from_f32(float v);
template <>
__device__ __forceinline__ float from_f32<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Four consecutive elements.  VEC: p is aligned to them all.
template <bool VEC>
__device__ __forceinline__ float4 load4(const float* p) {
  if constexpr (VEC) return *reinterpret_cast<const float4*>(p);
  return make_float4(p[0], p[1], p[2], p[3]);
}
template <bool VEC>
__device__ __forceinline__ float4 load4(const __nv_bfloat16* p) {
  if constexpr (VEC) {
    const uint2 w = *reinterpret_cast<const uint2*>(p);
    const float2 a = bf16x2_to_float2(w.x), b = bf16x2_to_float2(w.y);
    return make_float4(a.x, a.y, b.x, b.y);
  }
  return make_float4(to_f32(p[0]), to_f32(p[1]), to_f32(p[2]), to_f32(p[3]));
}

// Whether rows at `p` with these strides (in elements of `size` bytes) can be read 4 elements at a time.
inline bool aligned4(const void* p, int size, int64_t a, int64_t b) {
  return reinterpret_cast<uintptr_t>(p) % (4 * size) == 0 && a % 4 == 0 && b % 4 == 0;
}

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v = fmaxf(v, __shfl_xor_sync(~0u, v, o));
  return v;
}
// ------------------------------------------------------------------ the cache's workspace
//
// [64 ints: status word, plan ticket][attention tickets][attention partial states]

constexpr int kKv8WorkHead = 64;  // ints

inline bool kv8_shape_ok(const ssd_kv8* c) {
  if (!c) return false;
  const bool bs = c->block_tokens == 16 || c->block_tokens == 32 || c->block_tokens == 64 || c->block_tokens == 128;
  if (!bs || (c->head_dim != 64 && c->head_dim != 128) || c->n_layers < 1 || c->n_kv_heads < 1 || c->n_blocks < 1)
    return false;
  if (c->n_heads < c->n_kv_heads || c->n_heads % c->n_kv_heads) return false;
  if (c->max_batch < 1 || c->max_batch > SSD_KV8_MAX_BATCH || c->max_blocks < 1) return false;
  // slots, row numbers and positions fit 31 bits, with room to add a tile
  const int64_t lim = 1 << 30;
  const int64_t cap = static_cast<int64_t>(c->max_blocks) * c->block_tokens;
  if (static_cast<int64_t>(c->n_blocks) * c->block_tokens > lim || cap > lim || c->n_heads > 16384) return false;
  if (static_cast<int64_t>(c->n_blocks) * (c->block_tokens / 16) * c->n_kv_heads > lim) return false;
  return cap * c->max_batch <= 0x7fffffff;
}

}  // namespace ssd

namespace ssd {

// ------------------------------------------------------------------ a step's buffer
//
// Work of the attention is the flat list of 16-token tiles of all segments (request, kv head, row
// group), cut into one span per team of W warps.  The plan makes the cuts, once for all layers, so that
// an attention warp finds its place with one load.

constexpr int kAttnSms = 152;
constexpr int kAttnMaxTeams = 2 * kAttnSms * 8;

// Launch shape of the attention for items of 8, 16, 24 or 32 rows, by the registers that the output
// accumulators take (rows x dimensions / 32 a thread).
struct AttnShape {
  int warps, ctas, teams;  // per CTA, CTAs per SM, most teams per CTA
};
__host__ __device__ constexpr AttnShape attn_shape(int row_tile, int dim) {
  return row_tile * dim <= 1024   ? AttnShape{8, 2, row_tile == 8 ? 8 : 4}
         : row_tile * dim <= 2048 ? AttnShape{12, 1, 4}
                                  : AttnShape{8, 1, 2};
}

struct alignas(16) StepHead {
  int64_t span;  // tiles per team; cuts inside long segments are its multiples
  int warps;     // per team
  int n_rows;    // rows of all requests
  int pad[12];
};
// A team's span [u0, u1) of the list: it begins at tile `tile` of this segment.
struct alignas(16) TeamSpan {
  int b, head, rg, tile;
  int n, groups, row0, rows;  // tiles of the segment; row groups, first row and rows of the request
  int64_t u0, u1;
  int len, pad[3];
};
static_assert(sizeof(StepHead) == 64 && sizeof(TeamSpan) == 64, "layout");
static_assert(sizeof(StepHead) + kAttnMaxTeams * sizeof(TeamSpan) == SSD_KV8_STEP_HEAD * 4ull, "layout");

struct StepView {
  StepHead* head;
  TeamSpan* teams;  // [CTA][most teams per CTA]
  int32_t* seg_start;
  int32_t* row_start;
  int32_t* len;
  int32_t* slot;
};
__host__ __device__ __forceinline__ StepView step_view(int32_t* d, int batch) {
  StepView v;
  v.head = reinterpret_cast<StepHead*>(d);
  v.teams = reinterpret_cast<TeamSpan*>(v.head + 1);
  v.seg_start = d + SSD_KV8_STEP_HEAD;
  v.row_start = v.seg_start + batch + 1;
  v.len = v.row_start + batch + 1;
  v.slot = v.len + batch;
  return v;
}

// Query rows (of one kv head) one attention item takes.  Items of 8 have the most warps per SM and the
// fewest empty columns where requests differ, but more of them read the same tiles; so they are the choice
// where the tiles come from L2: a layer's cache of at most 128 MB, about L2's size (12 rows of a kv head, 75 MB:
// items of 8 rows 29 us, of 16 34; 16 rows, 89 MB: 31 and 44 us; 32 rows, 132 MB: 52 and 51).  Else as many as
// there usually are, in the fewest items of at most 32 (24 rows, 147 MB: of 24 50 us, of 8 58; 900 MB: 111 and
// 182).  Measured in caches as large as their content.  The host knows the capacity only, so a large pool that
// holds short contexts gets the larger items where 8 would be faster (256 requests of 300 tokens, 16 rows:
// 85 us, of 8 54).  Where the content is just above L2 either may be (64 requests of 2000 tokens, 16 rows,
// 186 MB: of 16 55 us, of 8 49).
constexpr int64_t kItemsOf8Bytes = 128ll << 20;
inline int step_row_tile(const ssd_kv8* c, const ssd_kv8_step* s) {
  if (s->row_tile) return s->row_tile;
  const int64_t all = static_cast<int64_t>(s->batch) * c->max_blocks, blocks = all < c->n_blocks ? all : c->n_blocks;
  if (blocks * c->block_tokens * c->n_kv_heads * c->head_dim * 2 <= kItemsOf8Bytes) return 8;
  const int64_t r = static_cast<int64_t>((s->rows > 0 ? s->rows + s->batch - 1 : s->batch) / s->batch) *
                    (c->n_heads / c->n_kv_heads);
  const int64_t items = (r + 31) / 32;
  return static_cast<int>(((r + items - 1) / items + 7) / 8 * 8);
}

ssd_status kv8_check(const ssd_kv8* c, int layer);
ssd_status kv8_check_step(const ssd_kv8* c, const ssd_kv8_step* s);

}  // namespace ssd
