// Attention of a step's query rows over the paged 8-bit cache (see ssd_kv8_attention).
//
// Mathematics.  For one kv head and up to 8 NB query rows r (rows x grouped heads) the kernel forms
// S^T = K Q^T and O^T = V^T P^T, 16 keys at a time, with m16n8k16 products: the keys (then the
// dimensions) are the 16 matrix rows, the query rows the 8 columns, so one row costs no more than
// eight need.  Codes are exact in fp16: a byte c + 128 becomes the half 1024 + (c + 128) by a byte
// permute, less 1152.  Queries are scaled by a power of two per row into [1, 2) and held as one half
// (bf16 rows: exact) or a high and a low half (fp32 rows, 22 bits).  The K scale, the row's power of
// two and the softmax scale multiply the fp32 scores.  Softmax is online, with the running maximum m
// and sum l in fp32: p = 2^(s - m).  The V scale vs of a tile goes into the weights w = p vs / B, which
// are rounded to one half (two for fp32 rows); B is a power of two per row, at least every p vs so
// far, so that neither tiny nor huge V blocks lose bits; O is kept in units of B.
//
// Bound: bytes.  A cached token costs 2 D bytes and 4 D rows flops, below the tensor rate up to about
// 16 rows; so the design is a stream of the cache at full width.  The tile layout (lowbit.cuh) lets
// each lane copy the 16-byte pieces that it alone reads, with cp.async into its warp's own ring: no
// barrier between the copies and their use, three steps of 8 KB a warp in flight or in use.
//
// Work is the flat list of 16-token tiles of all (request, kv head, row group) segments, cut into
// equal spans, one per team of W warps (8 warps share an SM).  Teams take a segment's steps in turn and
// merge their states in shared memory.  Few segments: W = 8, and long segments are cut between teams;
// the team that finishes such a segment last (an atomic ticket, never a wait) merges the states from
// global memory in team order, so the result does not depend on timing.  Many segments: smaller teams,
// down to single warps that merge nothing.
#include "lowbit.cuh"

namespace ssd {
namespace {

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxCtas = 152;
constexpr int kMaxTeams = kMaxCtas * kWarps;

struct Kv8AttnParams {
  const void* q;
  void* o;
  int64_t q_row, q_head, o_row, o_head;
  const uint32_t* row_mask;
  int32_t* step;
  int batch, rows, group, n_heads, n_kv_heads, shift, n_blocks, max_blocks;
  int q_vec;  // q rows can be read 4 elements at a time
  float scale_log2;
  const uint8_t* data;
  const float* scales;
  const int32_t* table;
  unsigned* tickets;  // [kMaxTeams], zero between launches
  float* part;        // [2 * teams][8 NB][D], then [2 * teams][8 NB][2] (maximum, sum)
};

template <int D, int NB>
struct Geo {
  static constexpr int kTile = 32 * D;                      // bytes of 16 tokens, K and V
  static constexpr int kStage = 2 * kTile;                  // a step: two tiles
  static constexpr int kStages = (NB == 4 ? 16384 : 24576) / kStage;
  static constexpr int kRing = kStages * kStage;            // per warp
  static constexpr int kPad = D + 4;                        // floats per row of a merge record
  static constexpr int kTeams = NB == 4 ? kMaxCtas : kMaxTeams;  // most teams a launch may have
  static constexpr bool kSharedQ = NB == 4;                 // query fragments in shared memory, one copy per CTA
  static constexpr int kRec = kWarps * kRing;
  static constexpr int kStat = kRec + kWarps * 8 * kPad * 4;
  static constexpr int kScale = kStat + kWarps * 8 * 2 * 4;
  static constexpr int kFlag = kScale + kWarps * kStages * 2 * 8;
  static constexpr int kQ = kFlag + kWarps * 4 + 16;
  static constexpr int kRs = kQ + (kSharedQ ? 2 * (D / 16) * NB * 32 * 8 : 0);
  static constexpr int kTotal = kRs + (kSharedQ ? 8 * NB * 4 : 0);
  static_assert(kRec % 16 == 0 && kStat % 16 == 0 && kScale % 16 == 0 && kQ % 16 == 0, "alignment");
  static_assert(kTotal <= 232448, "shared memory");
  static_assert((SSD_KV8_MAX_BATCH + 1) * 8 <= kStat - kRec, "the partition's prefix sums fit the merge records");
};

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Codes b0, b1 (HI: b2, b3) of a word of bytes c + 128, as halves.
template <bool HI>
__device__ __forceinline__ uint32_t codes2(uint32_t w) {
  uint32_t x, y;
  asm("prmt.b32 %0, %1, %2, %3;" : "=r"(x) : "r"(w), "r"(0x64646464u), "n"(HI ? 0x4342 : 0x4140));
  asm("sub.f16x2 %0, %1, %2;" : "=r"(y) : "r"(x), "r"(0x64806480u));
  return y;
}

__device__ __forceinline__ void mma16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                      uint32_t b1) {
  asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t half2_bits(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ float2 half2_floats(uint32_t h) {
  return __half22float2(*reinterpret_cast<const __half2*>(&h));
}
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}

__device__ __forceinline__ void cp_async8(void* dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(smem_u32(dst)), "l"(src) : "memory");
}

__device__ __forceinline__ uint4 lds128(const uint8_t* p) { return *reinterpret_cast<const uint4*>(p); }

// A place in the flat work list: tile `tile` of segment `seg` (kv head, row group) of request b.
struct Place {
  int b, seg, n_segs, n;  // segments of the request, tiles of each
  int tile;
};

struct Work {
  const int64_t* start;  // shared: prefix sums of tiles per request
  const int32_t *seg_start, *row_start, *len;
  int batch;
  int64_t cap;

  __device__ __forceinline__ void request(Place& p, int b) const {
    p.b = b;
    p.n_segs = __ldg(seg_start + b + 1) - __ldg(seg_start + b);
    const int64_t end = static_cast<int64_t>(__ldg(len + b)) + __ldg(row_start + b + 1) - __ldg(row_start + b);
    p.n = static_cast<int>((min(end, cap) + 15) >> 4);
  }
  // The place of flat tile u (0 <= u < total).
  __device__ __forceinline__ Place locate(int64_t u) const {
    int lo = 0, hi = batch;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (start[mid] <= u) lo = mid; else hi = mid;
    }
    Place p;
    request(p, lo);
    const int64_t d = u - start[lo];
    p.seg = static_cast<int>(d / p.n);
    p.tile = static_cast<int>(d - static_cast<int64_t>(p.seg) * p.n);
    return p;
  }
};

// A team's part of one segment: tiles [a, e).
struct Piece {
  Place p;
  int a, e;
  int64_t u;  // flat position of tile a
};

template <typename T, int D, int NB>
__global__ void __launch_bounds__(kThreads, 1) ssd_kv8_attn_kernel(const Kv8AttnParams p) {
  using G = Geo<D, NB>;
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;
  constexpr int KS = D / 16;  // 16-dimension steps of the scores, 16-dimension tiles of the output
  constexpr int RT = 8 * NB;
  extern __shared__ __align__(128) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const StepView st = step_view(p.step, p.batch);
  const int bs_tiles = 1 << (p.shift - 4);

  // rows past the last request's
  const int n_rows = st.row_start[p.batch];
  if (n_rows < p.rows) {
    const int64_t n = static_cast<int64_t>(p.rows - n_rows) * p.n_heads * D;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + tid; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) {
      const int64_t rh = i / D;
      static_cast<T*>(p.o)[(n_rows + rh / p.n_heads) * p.o_row + rh % p.n_heads * p.o_head + i % D] = from_f32<T>(0.0f);
    }
  }

  // ---- this team's span of the work
  Work work;
  int64_t* start_s = reinterpret_cast<int64_t*>(smem + G::kRec);
  int* max_s = reinterpret_cast<int*>(smem + G::kFlag);
  work.start = start_s;
  work.seg_start = st.seg_start;
  work.row_start = st.row_start;
  work.len = st.len;
  work.batch = p.batch;
  work.cap = static_cast<int64_t>(p.max_blocks) << p.shift;
  if (tid == 0) *max_s = 0;
  __syncthreads();
  {
    int most = 0;
    for (int b = tid; b <= p.batch; b += kThreads) {
      start_s[b] = st.work_start[b];
      if (b < p.batch) {
        Place q;
        work.request(q, b);
        if (q.n_segs > 0) most = max(most, q.n);
      }
    }
    if (most) atomicMax(max_s, most);
  }
  const int n_segs = st.seg_start[p.batch];
  __syncthreads();
  const int64_t total = start_s[p.batch];
  // Team size: with fewer than two segments per team of a size, the next larger size cuts less.
  const int W = NB == 4 ? 8 : n_segs >= 16 * static_cast<int>(gridDim.x) ? 1 : n_segs >= 8 * static_cast<int>(gridDim.x) ? 2 : n_segs >= 4 * static_cast<int>(gridDim.x) ? 4 : 8;
  const int teams = gridDim.x * (kWarps / W);
  const int sub = warp / W, wt = warp - sub * W;  // team of the CTA, warp of the team
  const int team = blockIdx.x * (kWarps / W) + sub;
  const int tt = tid - sub * W * 32;              // thread of the team
  const int64_t span = max((total + teams - 1) / teams, static_cast<int64_t>(4 * W));
  const int snap = static_cast<int>(min(span / 4, static_cast<int64_t>(1 << 30)));
  int64_t u0, u1;
  // Short contexts, a team for each: one segment per team, whatever its length, so that nothing is
  // merged through global memory (64 tiles take one SM about as long as that merge).
  if (n_segs <= teams && *max_s <= 64) {
    u0 = u1 = 0;
    if (team < n_segs) {
      int lo = 0, hi = p.batch;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (__ldg(st.seg_start + mid) <= team) lo = mid; else hi = mid;
      }
      Place q;
      work.request(q, lo);
      u0 = start_s[lo] + static_cast<int64_t>(team - __ldg(st.seg_start + lo)) * q.n;
      u1 = u0 + q.n;
    }
  } else {
    // Equal spans; a cut inside a segment that is short against the span moves to its nearer end.
    auto cut = [&](int c) -> int64_t {
      const int64_t x = c * span;
      if (x >= total) return total;
      const Place q = work.locate(x);
      if (q.n > snap) return x;
      return q.tile < q.n - q.tile ? x - q.tile : x - q.tile + q.n;
    };
    u0 = cut(team);
    u1 = cut(team + 1);
  }
  Piece c_piece;  // consumed
  if (u0 < u1) {
    c_piece.p = work.locate(u0);
    c_piece.u = u0;
    c_piece.a = c_piece.p.tile;
    c_piece.e = static_cast<int>(min(static_cast<int64_t>(c_piece.p.n), c_piece.a + (u1 - u0)));
  }
  __syncthreads();  // the prefix sums give way to the merge records
  if (u0 >= u1) return;

  auto next_piece = [&](Piece& x) -> bool {
    x.u += x.e - x.a;
    if (x.u >= u1) return false;
    if (++x.p.seg >= x.p.n_segs) {
      int b = x.p.b + 1;
      for (work.request(x.p, b); x.p.n_segs == 0; work.request(x.p, b)) ++b;  // u < u1: a later request has work
      x.p.seg = 0;
    }
    x.a = 0;
    x.e = static_cast<int>(min(static_cast<int64_t>(x.p.n), u1 - x.u));
    return true;
  };

  // ---- the stream of this warp's steps: tiles (tile, tile + 1), one block-table entry ahead
  const int row_groups_div = p.n_kv_heads;
  uint8_t* ring = smem + warp * G::kRing;
  float2* scale_s = reinterpret_cast<float2*>(smem + G::kScale) + warp * (G::kStages * 2);
  Piece i_piece = c_piece;
  int i_tile = i_piece.a + 2 * wt, i_head = 0, i_id = -1;
  bool i_more = true;
  auto lookup = [&]() {  // moves to the next step that exists and reads its table entries (lane & 1: which tile)
    while (i_tile >= i_piece.e) {
      if (!next_piece(i_piece)) {
        i_more = false;
        return;
      }
      i_tile = i_piece.a + 2 * wt;
    }
    i_head = i_piece.p.seg / (i_piece.p.n_segs / row_groups_div);
    const int tile = i_tile + (lane & 1);
    i_id = tile < i_piece.e ? __ldg(p.table + static_cast<size_t>(i_piece.p.b) * p.max_blocks + (tile >> (p.shift - 4))) : -1;
  };
  auto issue = [&](int stage) {
    if (i_more) {
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int id = __shfl_sync(~0u, i_id, k);
        float2* sc = scale_s + stage * 2 + k;
        if (id >= 0 && id < p.n_blocks) {
          const size_t rec = static_cast<size_t>(id) * p.n_kv_heads + i_head;
          const uint8_t* src = p.data + (rec * bs_tiles + ((i_tile + k) & (bs_tiles - 1))) * G::kTile + lane * 16;
          uint8_t* dst = ring + stage * G::kStage + k * G::kTile + lane * 16;
#pragma unroll
          for (int i = 0; i < G::kTile / 512; ++i) cp_async16(dst + i * 512, src + i * 512);
          if (lane == 0) cp_async8(sc, p.scales + rec * 2);
        } else if (lane == 0) {
          *sc = make_float2(-1.0f, 0.0f);  // no such tile: its keys are not seen
        }
      }
      i_tile += 2 * W;
      lookup();
    }
    cp_async_commit();
  };
  lookup();
  int i_stage = 0;
  for (; i_stage < G::kStages - 1; ++i_stage) issue(i_stage);
  int stage = 0;

  float* rec_s = reinterpret_cast<float*>(smem + G::kRec);
  float2* stat_s = reinterpret_cast<float2*>(smem + G::kStat);
  volatile int* flag_s = reinterpret_cast<volatile int*>(smem + G::kFlag);
  uint2* q_s = reinterpret_cast<uint2*>(smem + G::kQ);
  float* rs_s = reinterpret_cast<float*>(smem + G::kRs);

  for (bool more = true; more; more = next_piece(c_piece)) {
    const Place& pl = c_piece.p;
    const int groups = pl.n_segs / p.n_kv_heads;
    const int head = pl.seg / groups, rg = pl.seg - head * groups;
    const int row0 = __ldg(st.row_start + pl.b), rows_b = __ldg(st.row_start + pl.b + 1) - row0;
    const int len = __ldg(st.len + pl.b);
    const int r_valid = min(static_cast<int64_t>(rows_b) * p.group - static_cast<int64_t>(rg) * RT, static_cast<int64_t>(RT));
    // row r of the segment -> (step row of the request, query head of the kv head)
    auto row_of = [&](int r, int& i, int& hq) {
      const int R = rg * RT + r;
      i = R / p.group;
      hq = head * p.group + R - i * p.group;
    };

    // ---- query fragments: row nb * 8 + g, dimensions 16 s + 4 t .. + 3
    uint32_t qf[G::kSharedQ ? 1 : PARTS][G::kSharedQ ? 1 : KS][G::kSharedQ ? 1 : NB][2];
    float rs[NB][2];  // score factors of the rows 2t, 2t + 1 of each block
    auto load_q = [&](int nb, uint32_t (*f)[KS][2]) -> float {  // f[PARTS][KS][2]
      const int r = nb * 8 + g;
      float x[KS][4], amax = 0.0f;
      if (r < r_valid) {
        int i, hq;
        row_of(r, i, hq);
        const T* src = static_cast<const T*>(p.q) + (row0 + i) * p.q_row + hq * p.q_head + 4 * t;
#pragma unroll
        for (int s = 0; s < KS; ++s) {
          const float4 v = p.q_vec ? load4<true>(src + 16 * s) : load4<false>(src + 16 * s);
          x[s][0] = v.x, x[s][1] = v.y, x[s][2] = v.z, x[s][3] = v.w;
        }
      } else {
#pragma unroll
        for (int s = 0; s < KS; ++s) x[s][0] = x[s][1] = x[s][2] = x[s][3] = 0.0f;
      }
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) amax = fmaxf(amax, fabsf(x[s][e]));
      amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 1));
      amax = fmaxf(amax, __shfl_xor_sync(~0u, amax, 2));
      uint32_t ex = __float_as_uint(amax) & 0x7f800000u;
      if (ex == 0x7f800000u) ex = 127u << 23;  // an infinite query: its row comes out NaN or infinite
      if (ex == 0) ex = 1u << 23;
      const float inv = __uint_as_float((254u << 23) - ex);
#pragma unroll
      for (int s = 0; s < KS; ++s) {
#pragma unroll
        for (int e = 0; e < 4; ++e) x[s][e] *= inv;
        f[0][s][0] = half2_bits(x[s][0], x[s][1]);
        f[0][s][1] = half2_bits(x[s][2], x[s][3]);
        if constexpr (PARTS == 2) {
          const float2 h0 = half2_floats(f[0][s][0]), h1 = half2_floats(f[0][s][1]);
          f[1][s][0] = half2_bits(x[s][0] - h0.x, x[s][1] - h0.y);
          f[1][s][1] = half2_bits(x[s][2] - h1.x, x[s][3] - h1.y);
        }
      }
      return __uint_as_float(ex) * p.scale_log2;
    };
    if constexpr (G::kSharedQ) {  // one team per CTA: warps 0 .. NB - 1 fetch one block of rows each
      if (warp < NB) {
        uint32_t f[PARTS][KS][2];
        const float sc = load_q(warp, f);
#pragma unroll
        for (int k = 0; k < PARTS; ++k)
#pragma unroll
          for (int s = 0; s < KS; ++s) q_s[((k * KS + s) * NB + warp) * 32 + lane] = make_uint2(f[k][s][0], f[k][s][1]);
        if (t == 0) rs_s[warp * 8 + g] = sc;
      }
      named_bar_sync(1, kThreads);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        rs[nb][0] = rs_s[nb * 8 + 2 * t];
        rs[nb][1] = rs_s[nb * 8 + 2 * t + 1];
      }
    } else {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        uint32_t f[PARTS][KS][2];
        const float sc = load_q(nb, f);
#pragma unroll
        for (int k = 0; k < PARTS; ++k)
#pragma unroll
          for (int s = 0; s < KS; ++s) {
            qf[k][s][nb][0] = f[k][s][0];
            qf[k][s][nb][1] = f[k][s][1];
          }
        rs[nb][0] = __shfl_sync(~0u, sc, 8 * t);
        rs[nb][1] = __shfl_sync(~0u, sc, 8 * t + 4);
      }
    }
    auto q_frag = [&](int k, int s, int nb) -> uint2 {
      if constexpr (G::kSharedQ) return q_s[((k * KS + s) * NB + nb) * 32 + lane];
      else return make_uint2(qf[k][s][nb][0], qf[k][s][nb][1]);
    };

    float o[NB][KS][4], m[NB][2], l[NB][2], unit[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int i = 0; i < KS; ++i) o[nb][i][0] = o[nb][i][1] = o[nb][i][2] = o[nb][i][3] = 0.0f;
      m[nb][0] = m[nb][1] = -INFINITY;
      l[nb][0] = l[nb][1] = unit[nb][0] = unit[nb][1] = 0.0f;
    }

    for (int tile = c_piece.a + 2 * wt; tile < c_piece.e; tile += 2 * W) {
      cp_async_wait_group<G::kStages - 2>();
      __syncwarp();
      issue(i_stage);
      if (++i_stage == G::kStages) i_stage = 0;
      const uint8_t* buf = ring + stage * G::kStage + lane * 16;
      const float2 sc0 = scale_s[stage * 2], sc1 = scale_s[stage * 2 + 1];
      if (++stage == G::kStages) stage = 0;

      // scores of 2 x 16 keys: keys g and g + 8 of each tile (matrix rows), query rows 2t and 2t + 1
      float s[2][NB][4];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[k][nb][0] = s[k][nb][1] = s[k][nb][2] = s[k][nb][3] = 0.0f;
      }
#pragma unroll
      for (int c = 0; c < KS / 4; ++c) {
        uint4 lo[2], hi[2];
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          lo[k] = lds128(buf + k * G::kTile + c * 512);
          hi[k] = lds128(buf + k * G::kTile + (KS / 4 + c) * 512);
        }
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t a[2][4];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint32_t x = (&lo[k].x)[w], y = (&hi[k].x)[w];
            a[k][0] = codes2<false>(x), a[k][1] = codes2<false>(y), a[k][2] = codes2<true>(x), a[k][3] = codes2<true>(y);
          }
#pragma unroll
          for (int part = 0; part < PARTS; ++part)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const uint2 f = q_frag(part, c * 4 + w, nb);
#pragma unroll
              for (int k = 0; k < 2; ++k) mma16(s[k][nb], a[k][0], a[k][1], a[k][2], a[k][3], f.x, f.y);
            }
        }
      }
      // masks: only where a tile reaches past the cached tokens, or does not exist
      const bool edge = (tile + 2) * 16 > len || sc0.x < 0.0f || sc1.x < 0.0f;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          s[0][nb][e] *= rs[nb][e & 1] * sc0.x;
          s[1][nb][e] *= rs[nb][e & 1] * sc1.x;
        }
      if (edge) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = nb * 8 + 2 * t + e;
            int i = 0, hq;
            if (r < r_valid) row_of(r, i, hq);
            const uint32_t bits = p.row_mask && r < r_valid ? __ldg(p.row_mask + row0 + i) : 0u;
#pragma unroll
            for (int k = 0; k < 2; ++k)
#pragma unroll
              for (int half = 0; half < 2; ++half) {
                const int j = (tile + k) * 16 + kv8_tile_token(g + 8 * half) - len;  // the step's own row j
                const bool seen = (k ? sc1.x : sc0.x) >= 0.0f &&
                                  (j < 0 || (p.row_mask ? j < 32 && (bits >> j & 1u) : j <= i && r < r_valid));
                if (!seen) s[k][nb][half * 2 + e] = -INFINITY;
              }
          }
      }
      // online softmax, then weights in halves, transposed into the second product's operand
      uint32_t pf[2][NB][PARTS][2];
      float scale_o[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        float vinv[2][2];
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float t0 = fmaxf(s[0][nb][e], s[0][nb][e + 2]), t1 = fmaxf(s[1][nb][e], s[1][nb][e + 2]);
#pragma unroll
          for (int x = 4; x <= 16; x <<= 1) {
            t0 = fmaxf(t0, __shfl_xor_sync(~0u, t0, x));
            t1 = fmaxf(t1, __shfl_xor_sync(~0u, t1, x));
          }
          const float m_new = fmaxf(m[nb][e], fmaxf(t0, t1));
          const float m_use = m_new == -INFINITY ? 0.0f : m_new;
          const float alpha = ex2(m[nb][e] - m_use);
          m[nb][e] = m_new;
          const float need = fmaxf(unit[nb][e] * alpha, fmaxf(ex2(t0 - m_use) * sc0.y, ex2(t1 - m_use) * sc1.y));
          uint32_t up = (__float_as_uint(need) + 0x7fffffu) & 0x7f800000u;
          up = max(up, 1u << 23);
          const float inv = __uint_as_float((254u << 23) - up);
          scale_o[nb][e] = alpha * (unit[nb][e] * inv);
          unit[nb][e] = __uint_as_float(up);
          vinv[0][e] = sc0.y * inv;
          vinv[1][e] = sc1.y * inv;
          float sum = 0.0f;
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              float& x = s[k][nb][half * 2 + e];
              x = ex2(x - m_use);
              sum += x;
            }
          l[nb][e] = l[nb][e] * alpha + sum;
        }
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int half = 0; half < 2; ++half) {
            const float w0 = s[k][nb][half * 2] * vinv[k][0], w1 = s[k][nb][half * 2 + 1] * vinv[k][1];
            const uint32_t h = half2_bits(w0, w1);
            pf[k][nb][0][half] = transpose8(h);
            if constexpr (PARTS == 2) {
              const float2 hf = half2_floats(h);
              pf[k][nb][1][half] = transpose8(half2_bits(w0 - hf.x, w1 - hf.y));
            }
          }
      }
      bool same = true;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) same &= scale_o[nb][0] == 1.0f && scale_o[nb][1] == 1.0f;
      if (!__all_sync(~0u, same)) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int i = 0; i < KS; ++i) {
            o[nb][i][0] *= scale_o[nb][0];
            o[nb][i][1] *= scale_o[nb][1];
            o[nb][i][2] *= scale_o[nb][0];
            o[nb][i][3] *= scale_o[nb][1];
          }
      }
#pragma unroll
      for (int c = 0; c < KS / 2; ++c) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint4 v = lds128(buf + k * G::kTile + 16 * D + c * 512);
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const uint32_t x = w ? v.z : v.x, y = w ? v.w : v.y;
            const uint32_t a0 = codes2<false>(x), a1 = codes2<false>(y), a2 = codes2<true>(x), a3 = codes2<true>(y);
#pragma unroll
            for (int part = 0; part < PARTS; ++part)
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) mma16(o[nb][c * 2 + w], a0, a1, a2, a3, pf[k][nb][part][0], pf[k][nb][part][1]);
          }
        }
      }
    }

    // ---- merge the team's warps, eight rows at a time
    const bool whole = c_piece.a == 0 && c_piece.e == pl.n;
    const int slot = team * 2 + (c_piece.a == 0 ? 1 : 0);
    float* part_o = p.part + static_cast<size_t>(slot) * RT * D;
    float2* part_s = reinterpret_cast<float2*>(p.part + static_cast<size_t>(2) * G::kTeams * RT * D) + slot * RT;
    auto write_row = [&](int r, int d, const float4& v, float sum) {
      if (r >= r_valid) return;
      int i, hq;
      row_of(r, i, hq);
      T* dst = static_cast<T*>(p.o) + (row0 + i) * p.o_row + hq * p.o_head + d;
      const float f = sum == 0.0f ? 0.0f : 1.0f / sum;
      dst[0] = from_f32<T>(v.x * f), dst[1] = from_f32<T>(v.y * f), dst[2] = from_f32<T>(v.z * f), dst[3] = from_f32<T>(v.w * f);
    };
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float* mine = rec_s + warp * (8 * G::kPad);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float sum = l[nb][e];
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1) sum += __shfl_xor_sync(~0u, sum, x);
        if (g == 0) stat_s[warp * 8 + 2 * t + e] = make_float2(m[nb][e], sum);
#pragma unroll
        for (int i = 0; i < KS; ++i) {
          mine[(2 * t + e) * G::kPad + 16 * i + g] = o[nb][i][e] * unit[nb][e];
          mine[(2 * t + e) * G::kPad + 16 * i + g + 8] = o[nb][i][e + 2] * unit[nb][e];
        }
      }
      named_bar_sync(1 + sub, W * 32);
      for (int x = tt; x < 8 * D / 4; x += W * 32) {
        const int r = x / (D / 4), d = (x % (D / 4)) * 4;
        float top = -INFINITY;
        for (int w = 0; w < W; ++w) top = fmaxf(top, stat_s[(sub * W + w) * 8 + r].x);
        const float use = top == -INFINITY ? 0.0f : top;
        float sum = 0.0f;
        float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int w = 0; w < W; ++w) {
          const float2 ms = stat_s[(sub * W + w) * 8 + r];
          const float f = ex2(ms.x - use);
          const float4 v = *reinterpret_cast<const float4*>(rec_s + ((sub * W + w) * 8 + r) * G::kPad + d);
          sum += ms.y * f;
          acc.x += v.x * f, acc.y += v.y * f, acc.z += v.z * f, acc.w += v.w * f;
        }
        if (whole) {
          write_row(nb * 8 + r, d, acc, sum);
        } else {
          *reinterpret_cast<float4*>(part_o + (nb * 8 + r) * D + d) = acc;
          if (d == 0) part_s[nb * 8 + r] = make_float2(top, sum);
        }
      }
      named_bar_sync(1 + sub, W * 32);
    }
    if (!whole) {
      // the teams that share the segment: those of the cuts inside it
      const int64_t s0 = c_piece.u - c_piece.a, s1 = s0 + pl.n;
      const int t0 = static_cast<int>(s0 / span), t1 = static_cast<int>((s1 - 1) / span);
      if (tt == 0) flag_s[sub] = atom_add_acq_rel_gpu(p.tickets + t0, 1u) == static_cast<unsigned>(t1 - t0);
      named_bar_sync(1 + sub, W * 32);
      if (flag_s[sub]) {
        if (tt == 0) p.tickets[t0] = 0;
        const float2* all_s = reinterpret_cast<const float2*>(p.part + static_cast<size_t>(2) * G::kTeams * RT * D);
        for (int x = tt; x < RT * D / 4; x += W * 32) {
          const int r = x / (D / 4), d = (x % (D / 4)) * 4;
          if (r >= r_valid) break;
          float top = -INFINITY;
          for (int c = t0; c <= t1; ++c) top = fmaxf(top, __ldcg(all_s + (2 * c + (c == t0)) * RT + r).x);
          const float use = top == -INFINITY ? 0.0f : top;
          float sum = 0.0f;
          float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
          for (int c = t0; c <= t1; ++c) {
            const int from = 2 * c + (c == t0);
            const float2 ms = __ldcg(all_s + from * RT + r);
            const float4 v = __ldcg(reinterpret_cast<const float4*>(p.part + (static_cast<size_t>(from) * RT + r) * D + d));
            const float f = ex2(ms.x - use);
            sum += ms.y * f;
            acc.x += v.x * f, acc.y += v.y * f, acc.z += v.z * f, acc.w += v.w * f;
          }
          write_row(r, d, acc, sum);
        }
      }
      named_bar_sync(1 + sub, W * 32);
    }
  }
  cp_async_wait_all();
}

template <typename T, int D, int NB>
ssd_status launch(const Kv8AttnParams& p, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  if (ssd_status e = op_smem(ssd_kv8_attn_kernel<T, D, NB>, Geo<D, NB>::kTotal, ready, "ssd_kv8_attention")) return e;
  ssd_kv8_attn_kernel<T, D, NB><<<kMaxCtas, kThreads, Geo<D, NB>::kTotal, s>>>(p);
  return op_launched("ssd_kv8_attention");
}

template <typename T, int D>
ssd_status launch_rows(int row_tile, const Kv8AttnParams& p, cudaStream_t s) {
  return row_tile == 8 ? launch<T, D, 1>(p, s) : row_tile == 16 ? launch<T, D, 2>(p, s) : launch<T, D, 4>(p, s);
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" {

int64_t ssd_kv8_work_bytes(const ssd_kv8* c) {
  if (!kv8_shape_ok(c)) return -1;
  // 32-row items always have teams of a whole CTA, so 16-row items of single-warp teams need most
  const int64_t rows16 = 2ll * kMaxTeams * 16 * (c->head_dim + 2) * 4;
  const int64_t rows32 = 2ll * kMaxCtas * 32 * (c->head_dim + 2) * 4;
  return kKv8WorkHead * 4 + kMaxTeams * 4 + (rows16 > rows32 ? rows16 : rows32);
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
  p.n_heads = c->n_heads;
  p.n_kv_heads = c->n_kv_heads;
  p.shift = 31 - __builtin_clz(c->block_tokens);
  p.n_blocks = c->n_blocks;
  p.max_blocks = c->max_blocks;
  p.q_vec = aligned4(q, size, q_row_stride, q_head_stride);
  p.scale_log2 = scale * 1.4426950408889634f;
  const size_t recs = static_cast<size_t>(layer) * c->n_blocks * c->n_kv_heads;
  p.data = static_cast<const uint8_t*>(c->data) + recs * c->block_tokens * c->head_dim * 2;
  p.scales = c->scales + recs * 2;
  p.table = c->table;
  p.tickets = static_cast<unsigned*>(c->work) + kKv8WorkHead;
  p.part = reinterpret_cast<float*>(p.tickets + kMaxTeams);
  const int tile = step_row_tile(c, step);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (type == SSD_TYPE_FP32)
    return c->head_dim == 128 ? launch_rows<float, 128>(tile, p, s) : launch_rows<float, 64>(tile, p, s);
  return c->head_dim == 128 ? launch_rows<__nv_bfloat16, 128>(tile, p, s) : launch_rows<__nv_bfloat16, 64>(tile, p, s);
}

}  // extern "C"
