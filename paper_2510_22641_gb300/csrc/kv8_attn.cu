// Attention of a step's query rows over the paged 8-bit cache (see ssd_kv8_attention).
//
// Mathematics.  For one kv head and up to 8 NB query rows r (rows x grouped heads) the kernel forms
// S^T = K Q^T and O^T = V^T P^T, 16 keys at a time, with m16n8k16 products: the keys (then the
// dimensions) are the 16 matrix rows, the query rows the 8 columns, so one row costs no more than
// eight need.  Codes are exact in fp16: a byte c + 128 becomes the half 1024 + (c + 128) by a byte
// permute, less 1152.  Queries are scaled by a power of two per row, the largest into [2^14, 2^15), and held
// as one half (bf16 rows: exact down to 2^-31 of the largest) or a high and a low half (fp32 rows: 22 bits,
// or 2^-39 of the largest).  The K scale, the row's power of two and the softmax scale multiply the fp32
// scores.  Softmax is online, in fp32: p = 2^(s - m) with a reference m per row that is raised, in whole
// steps, to the running maximum only when a p passes 2^8, and the sum l.  The V scale vs of a tile goes into
// the weights w = 2^7 p vs / B, which are rounded to one half (two for fp32 rows); B is a power of two per
// row, raised with m to at least every p vs, so that neither tiny nor huge V blocks lose bits; O is kept in
// units of B / 2^7.
//
// Bound: bytes.  A cached token of a kv head costs 2 D bytes and 4 D flops per query row (times grouped heads),
// below these products' rate up to about 16 rows; so the design is a stream of the cache at full width.  The
// tile layout (lowbit.cuh) lets each lane copy the 16-byte pieces that it alone reads, with cp.async into its
// warp's own ring of three tiles or more: no barrier between the copies and their use.  Measured: 64 requests
// of up to 8191 tokens, 32 / 8 heads, two bf16 rows 112 us, 6.0 TB/s; 16 of 1024, 40 heads, seven fp32 rows 32 us (3.5 TB/s:
// 12 tiles a warp, then the merge); two of 131072, six rows, 24 query rows a kv head 106 us (4.3 TB/s: the
// accumulators leave 8 warps an SM, which wait for dependent results: issue 45 %, DRAM 51 %, tensor pipe 38 %);
// one row over 640 tokens 9.7 us (latency).
//
// Work is the flat list of 16-token tiles of all (request, kv head, row group) segments, cut by the plan
// into equal spans, one per team of W warps, a CTA or less.  A team's warps take a segment's tiles in turn
// and merge their states in shared memory.  Long segments are cut between teams; the team that finishes
// such a segment last (an atomic ticket, never a wait) merges the states from global memory in team order,
// so the result does not depend on timing.
#include "lowbit.cuh"

namespace ssd {
namespace {

struct Kv8AttnParams {
  const void* q;
  void* o;
  int64_t q_row, q_head, o_row, o_head;
  const uint32_t* row_mask;
  int32_t* step;
  int batch, rows, group, n_heads, n_kv_heads, shift, n_blocks, max_blocks;
  int q_vec;           // q rows can be read 4 elements at a time
  unsigned group_inv;  // ceil(2^32 / group): high half of R * group_inv = R / group for R < 2^32 / group
  float scale_log2;
  const uint8_t* data;
  const float* scales;
  const int32_t* table;
  unsigned* tickets;  // [kAttnMaxTeams], zero between launches
  float* part;        // [2 * teams] states of 8 NB rows x D, then [2 * teams][8 NB][2] (maximum, sum)
};

// Up to 8 rows: query fragments in registers.  More: in shared memory, one copy per team.
template <int D, int NB>
struct Geo {
  static constexpr AttnShape kShape = attn_shape(8 * NB, D);
  static constexpr int kWarps = kShape.warps;
  static constexpr int kThreads = 32 * kWarps;
  static constexpr int kCtas = kShape.ctas;
  static constexpr bool kSharedQ = NB > 1;
  static constexpr int kTeams = kShape.teams;
  static constexpr int kTile = 32 * D;                      // bytes of 16 tokens, K and V: one step
  static constexpr int kRing = kCtas == 2 && kSharedQ ? 10240 : kWarps * kCtas > 8 ? 12288 : 20480;  // per warp
  static constexpr int kStages = kRing / kTile;
  static constexpr int kStat = kWarps * kRing;              // (maximum, sum, unit) of 8 rows per warp
  static constexpr int kOff = kStat + kWarps * 8 * 16;      // where each warp's state lies
  static constexpr int kFlag = kOff + kWarps * 4;
  static constexpr int kPlace = (kFlag + kWarps * 4 + 15) / 16 * 16;
  static constexpr int kScale = kPlace + kWarps * 16;
  static constexpr int kQ = kScale + kWarps * kStages * 8;
  static constexpr int kQTeam = kSharedQ ? 2 * (D / 16) * NB * 32 * 8 + 8 * NB * 4 : 0;  // fragments, row factors
  static constexpr int kTotal = kQ + kTeams * kQTeam;
  static_assert(kScale % 16 == 0 && kQ % 16 == 0 && kQTeam % 16 == 0, "alignment");
  static_assert(kTile >= 8 * D * 4, "a state of 8 rows fits one stage");
  static_assert(kTotal * kCtas <= 231424, "shared memory");
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

// A team's part of one segment (row group rg of kv head `head` of request b): tiles [a, e) of n.
struct Piece {
  int b, head, rg, groups, n, a, e;
  int u;  // position of tile a in the team's span
};

template <typename T, int D, int NB>
__global__ void __launch_bounds__(Geo<D, NB>::kThreads, Geo<D, NB>::kCtas) ssd_kv8_attn_kernel(const Kv8AttnParams p) {
  using G = Geo<D, NB>;
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;
  constexpr int KS = D / 16;  // 16-dimension steps of the scores, 16-dimension tiles of the output
  constexpr int RT = 8 * NB;
  constexpr int kWarps = G::kWarps, kThreads = G::kThreads;
  extern __shared__ __align__(128) uint8_t smem[];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const StepView st = step_view(p.step, p.batch);
  const int bs_tiles = 1 << (p.shift - 4);

  pdl_wait();
  pdl_trigger();
  // ---- this team's span: the CTA's records, a 16-byte quarter per lane
  const int4 quarter = reinterpret_cast<const int4*>(st.teams + blockIdx.x * G::kTeams)[min(lane, 4 * G::kTeams - 1)];
  const int4 head = *reinterpret_cast<const int4*>(st.head);
  const int64_t span = static_cast<int64_t>(static_cast<uint32_t>(head.x)) | static_cast<int64_t>(head.y) << 32;
  const int W = head.z, n_rows = head.w;

  // rows past the last request's
  if (n_rows < p.rows) {
    const int64_t n = static_cast<int64_t>(p.rows - n_rows) * p.n_heads * D;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * kThreads + tid; i < n; i += static_cast<int64_t>(gridDim.x) * kThreads) {
      const int64_t rh = i / D;
      static_cast<T*>(p.o)[(n_rows + rh / p.n_heads) * p.o_row + rh % p.n_heads * p.o_head + i % D] = from_f32<T>(0.0f);
    }
  }
  if (W < 1 || W > kWarps || kWarps % W != 0) return;  // no plan was made
  const int sub = warp / W, wt = warp - sub * W;  // team of the CTA, warp of the team
  const int team = blockIdx.x * (kWarps / W) + sub;
  const int tt = tid - sub * W * 32;              // thread of the team
  auto field = [&](int q, int i) -> int {
    const int v = i == 0 ? quarter.x : i == 1 ? quarter.y : i == 2 ? quarter.z : quarter.w;
    return __shfl_sync(~0u, v, 4 * sub + q);
  };
  Piece c_piece;  // consumed
  c_piece.b = field(0, 0);
  c_piece.head = field(0, 1);
  c_piece.rg = field(0, 2);
  c_piece.a = field(0, 3);
  c_piece.n = field(1, 0);
  c_piece.groups = field(1, 1);
  int row0 = field(1, 2), rows_b = field(1, 3), len = field(3, 0);  // of the consumed piece's request
  const int64_t u0 = static_cast<int64_t>(static_cast<uint32_t>(field(2, 0))) | static_cast<int64_t>(field(2, 1)) << 32;
  const int64_t u1 = static_cast<int64_t>(static_cast<uint32_t>(field(2, 2))) | static_cast<int64_t>(field(2, 3)) << 32;
  if (u0 >= u1) return;
  const int u_len = static_cast<int>(u1 - u0);  // a span is far below 2^31 tiles
  c_piece.u = 0;
  c_piece.e = c_piece.a + min(c_piece.n - c_piece.a, u_len);
  int64_t* place_s = reinterpret_cast<int64_t*>(smem + G::kPlace) + warp * 2;  // needed at merges only
  if (lane == 0) place_s[0] = u0, place_s[1] = span;

  const int64_t cap = static_cast<int64_t>(p.max_blocks) << p.shift;
  auto next_piece = [&](Piece& x) -> bool {
    x.u += x.e - x.a;
    if (x.u >= u_len) return false;
    if (++x.rg >= x.groups) {
      x.rg = 0;
      if (++x.head >= p.n_kv_heads) {
        x.head = 0;
        int segs;
        do {  // u < u_len: a later request has work
          ++x.b;
          segs = st.seg_start[x.b + 1] - st.seg_start[x.b];
        } while (segs == 0);
        const int rows = st.row_start[x.b + 1] - st.row_start[x.b];
        x.n = static_cast<int>((min(static_cast<int64_t>(st.len[x.b]) + rows, cap) + 15) >> 4);
        x.groups = segs / p.n_kv_heads;
      }
    }
    x.a = 0;
    x.e = min(x.n, u_len - x.u);
    return true;
  };

  // ---- the stream of this warp's steps, one block-table entry ahead
  uint8_t* ring = smem + warp * G::kRing;
  const uint8_t* data_lane = p.data + lane * 16;
  float2* scale_s = reinterpret_cast<float2*>(smem + G::kScale) + warp * G::kStages;
  Piece i_piece = c_piece;
  int i_tile = i_piece.a + wt, i_head = i_piece.head, i_id = -1;
  bool i_more = true;
  auto lookup = [&]() {  // moves to the next step that exists and reads its table entry
    while (i_tile >= i_piece.e) {
      if (!next_piece(i_piece)) {
        i_more = false;
        return;
      }
      i_tile = i_piece.a + wt;
      i_head = i_piece.head;
    }
    i_id = p.table[static_cast<size_t>(i_piece.b) * p.max_blocks + (i_tile >> (p.shift - 4))];
  };
  auto issue = [&](int stage) {
    if (i_more) {
      float2* sc = scale_s + stage;
      if (static_cast<unsigned>(i_id) < static_cast<unsigned>(p.n_blocks)) {
        const unsigned rec = static_cast<unsigned>(i_id) * p.n_kv_heads + i_head;  // blocks x heads < 2^32
        const unsigned tile = (rec << (p.shift - 4)) + (i_tile & (bs_tiles - 1));
        const uint8_t* src = data_lane + static_cast<uint64_t>(tile) * G::kTile;
        uint8_t* dst = ring + stage * G::kTile + lane * 16;
#pragma unroll
        for (int i = 0; i < G::kTile / 512; ++i) cp_async16(dst + i * 512, src + i * 512);
        if (lane == 0) cp_async8(sc, p.scales + static_cast<uint64_t>(rec) * 2);
      } else if (lane == 0) {
        *sc = make_float2(-1.0f, 0.0f);  // no such block: its keys are not seen
      }
      i_tile += W;
      lookup();
    }
    cp_async_commit();
  };
  lookup();
  int i_stage = 0;
  for (; i_stage < G::kStages - 1; ++i_stage) issue(i_stage);
  int stage = 0;

  float4* stat_s = reinterpret_cast<float4*>(smem + G::kStat);
  volatile int* off_s = reinterpret_cast<volatile int*>(smem + G::kOff);
  volatile int* flag_s = reinterpret_cast<volatile int*>(smem + G::kFlag);
  uint2* q_s = reinterpret_cast<uint2*>(smem + G::kQ + sub * G::kQTeam);
  float* rs_s = reinterpret_cast<float*>(smem + G::kQ + sub * G::kQTeam + 2 * KS * NB * 32 * 8);

  for (;;) {
    const int head = c_piece.head, rg = c_piece.rg;
    // a mask has bits for 32 rows of the step; others are seen by none, which the caller is told
    if (p.row_mask && rows_b > 32 && tt == 0) atomicOr(reinterpret_cast<int*>(p.tickets) - kKv8WorkHead, SSD_KV8_LENGTH);
    const int r_valid = static_cast<int>(min(static_cast<int64_t>(rows_b) * p.group - static_cast<int64_t>(rg) * RT,
                                             static_cast<int64_t>(RT)));
    // row r of the segment -> (step row of the request, query head of the kv head)
    auto row_of = [&](int r, int& i, int& hq) {
      const int R = rg * RT + r;
      i = p.group == 1 ? R : static_cast<int>(__umulhi(static_cast<unsigned>(R), p.group_inv));
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
      ex = max(ex, 15u << 23);                 // so that 2^(14 - e) is a normal number
      const float inv = __uint_as_float((268u << 23) - ex);
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
    if constexpr (G::kSharedQ) {  // the team's warps fetch a block of 8 rows each
      for (int nb = wt; nb < NB; nb += W) {
        uint32_t f[PARTS][KS][2];
        const float sc = load_q(nb, f);
#pragma unroll
        for (int k = 0; k < PARTS; ++k)
#pragma unroll
          for (int s = 0; s < KS; ++s) q_s[((k * KS + s) * NB + nb) * 32 + lane] = make_uint2(f[k][s][0], f[k][s][1]);
        if (t == 0) rs_s[nb * 8 + g] = sc;
      }
      named_bar_sync(1 + sub, W * 32);
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
      m[nb][0] = m[nb][1] = -3.402823466e38f;  // finite, so that masked scores give 2^-inf = 0 even if none is seen
      l[nb][0] = l[nb][1] = 0.0f;
      unit[nb][0] = unit[nb][1] = 0x1p126f;  // forgotten with the first key seen
    }

    for (int tile = c_piece.a + wt; tile < c_piece.e; tile += W) {
      cp_async_wait_group<G::kStages - 2>();
      __syncwarp();
      issue(i_stage);
      if (++i_stage == G::kStages) i_stage = 0;
      const uint8_t* buf = ring + stage * G::kTile + lane * 16;
      const float2 sc = scale_s[stage];
      if (++stage == G::kStages) stage = 0;

      // scores of 16 keys: keys g and g + 8 (matrix rows), query rows 2t and 2t + 1
      float s[NB][4];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.0f;
#pragma unroll
      for (int c = 0; c < KS / 4; ++c) {
        const uint4 lo = lds128(buf + c * 512), hi = lds128(buf + (KS / 4 + c) * 512);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const uint32_t x = (&lo.x)[w], y = (&hi.x)[w];
          const uint32_t a0 = codes2<false>(x), a1 = codes2<false>(y), a2 = codes2<true>(x), a3 = codes2<true>(y);
#pragma unroll
          for (int part = 0; part < PARTS; ++part)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              const uint2 f = q_frag(part, c * 4 + w, nb);
              mma16(s[nb], a0, a1, a2, a3, f.x, f.y);
            }
        }
      }
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[nb][e] *= rs[nb][e & 1] * (sc.x * 0x1p-14f);
      // masks: only where a tile reaches past the cached tokens, or does not exist
      if ((tile + 1) * 16 > len || sc.x < 0.0f) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const int r = nb * 8 + 2 * t + e;
            int i = 0, hq;
            if (r < r_valid) row_of(r, i, hq);
            const uint32_t bits = p.row_mask && r < r_valid ? p.row_mask[row0 + i] : 0u;
#pragma unroll
            for (int half = 0; half < 2; ++half) {
              const int j = tile * 16 + kv8_tile_token(g + 8 * half) - len;  // the step's own row j
              const bool seen = sc.x >= 0.0f && (j < 0 || (p.row_mask ? j < rows_b && (static_cast<uint64_t>(bits) >> min(j, 63) & 1u) : j <= i && r < r_valid));
              if (!seen) s[nb][half * 2 + e] = -INFINITY;
            }
          }
      }
      // Online softmax.  The row's reference m and unit stay as they are while no probability passes
      // 2^8 and no weight 2^15 (a half holds 65504); a tile that passes raises them to its maximum, where
      // weights are at most 2^7.  Only such tiles need a maximum across lanes.
      float w[NB][4], pr[NB][2];
      // 2^7 / unit times the V scale (finite: a V block far above the unit has no weight here)
      auto vscale = [&](int nb, int e) -> float {
        return fminf(sc.y * __uint_as_float((261u << 23) - __float_as_uint(unit[nb][e])), 3.402823466e38f);
      };
      auto weigh = [&]() -> bool {
        bool up = false;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float vinv = vscale(nb, e);
            const float p0 = ex2(s[nb][e] - m[nb][e]), p1 = ex2(s[nb][e + 2] - m[nb][e]);
            w[nb][e] = p0 * vinv;
            w[nb][e + 2] = p1 * vinv;
            pr[nb][e] = p0 + p1;
            up |= pr[nb][e] > 256.0f || w[nb][e] > 32768.0f || w[nb][e + 2] > 32768.0f;
          }
        return up;
      };
      if (__any_sync(~0u, weigh())) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float top = fmaxf(s[nb][e], s[nb][e + 2]);
#pragma unroll
            for (int k = 4; k <= 16; k <<= 1) top = fmaxf(top, __shfl_xor_sync(~0u, top, k));
            // whole steps: alpha is a power of two, so that rows raised often do not round their unit up each time
            const float m_new = fmaxf(m[nb][e], ceilf(top)), step = m_new - m[nb][e];
            const float alpha = step > 126.0f ? 0.0f : __uint_as_float((127u - static_cast<unsigned>(step)) << 23);
            const float need = fmaxf(unit[nb][e] * alpha, ex2(top - m_new) * sc.y);
            const uint32_t bits = max((__float_as_uint(need) + 0x7fffffu) & 0x7f800000u, 8u << 23);
            const float f = (alpha * unit[nb][e]) * __uint_as_float((254u << 23) - bits);
            m[nb][e] = m_new;
            unit[nb][e] = __uint_as_float(bits);
            l[nb][e] *= alpha;
#pragma unroll
            for (int i = 0; i < KS; ++i) {
              o[nb][i][e] *= f;
              o[nb][i][e + 2] *= f;
            }
          }
        weigh();
      }
      // weights in halves, transposed into the second product's operand
      uint32_t pf[NB][PARTS][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        l[nb][0] += pr[nb][0];
        l[nb][1] += pr[nb][1];
#pragma unroll
        for (int half = 0; half < 2; ++half) {
          const uint32_t h = half2_bits(w[nb][half * 2], w[nb][half * 2 + 1]);
          pf[nb][0][half] = transpose8(h);
          if constexpr (PARTS == 2) {
            const float2 hf = half2_floats(h);
            pf[nb][1][half] = transpose8(half2_bits(w[nb][half * 2] - hf.x, w[nb][half * 2 + 1] - hf.y));
          }
        }
      }
#pragma unroll
      for (int c = 0; c < KS / 2; ++c) {
        const uint4 v = lds128(buf + 16 * D + c * 512);
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const uint32_t x = w ? v.z : v.x, y = w ? v.w : v.y;
          const uint32_t a0 = codes2<false>(x), a1 = codes2<false>(y), a2 = codes2<true>(x), a3 = codes2<true>(y);
#pragma unroll
          for (int part = 0; part < PARTS; ++part)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) mma16(o[nb][c * 2 + w], a0, a1, a2, a3, pf[nb][part][0], pf[nb][part][1]);
        }
      }
    }

    // ---- merge.  States stay in the accumulators' layout: a lane holds, for each 16-dimension tile, the
    // dimensions g and g + 8 of its rows 2t and 2t + 1.
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e)
#pragma unroll
        for (int x = 4; x <= 16; x <<= 1) l[nb][e] += __shfl_xor_sync(~0u, l[nb][e], x);
    const bool whole = c_piece.a == 0 && c_piece.e == c_piece.n;
    const int slot = team * 2 + (c_piece.a == 0 ? 1 : 0);
    float4* part_o = reinterpret_cast<float4*>(p.part);                                          // [slot][NB][KS][lane]
    float2* part_s = reinterpret_cast<float2*>(p.part + static_cast<size_t>(2) * gridDim.x * G::kTeams * RT * D);
    // the rows 2t and 2t + 1 of block nb: where they go, or null
    auto out_row = [&](int nb, int e) -> T* {
      const int r = nb * 8 + 2 * t + e;
      if (r >= r_valid) return nullptr;
      int i, hq;
      row_of(r, i, hq);
      return static_cast<T*>(p.o) + (row0 + i) * p.o_row + hq * p.o_head + g;
    };
    auto write = [&](T* d0, T* d1, int i, const float4& v, float f0, float f1) {
      if (d0) {
        d0[16 * i] = from_f32<T>(v.x * f0);
        d0[16 * i + 8] = from_f32<T>(v.z * f0);
      }
      if (d1) {
        d1[16 * i] = from_f32<T>(v.y * f1);
        d1[16 * i + 8] = from_f32<T>(v.w * f1);
      }
    };
    auto over = [](float sum) -> float { return sum == 0.0f ? 0.0f : 1.0f / sum; };
    if (W == 1) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float b0 = unit[nb][0] * 0x1p-7f, b1 = unit[nb][1] * 0x1p-7f;
        if (whole) {
          T *d0 = out_row(nb, 0), *d1 = out_row(nb, 1);
          const float f0 = b0 * over(l[nb][0]), f1 = b1 * over(l[nb][1]);
#pragma unroll
          for (int i = 0; i < KS; ++i) write(d0, d1, i, make_float4(o[nb][i][0], o[nb][i][1], o[nb][i][2], o[nb][i][3]), f0, f1);
        } else {
#pragma unroll
          for (int i = 0; i < KS; ++i)
            part_o[((static_cast<size_t>(slot) * NB + nb) * KS + i) * 32 + lane] =
                make_float4(o[nb][i][0] * b0, o[nb][i][1] * b1, o[nb][i][2] * b0, o[nb][i][3] * b1);
          if (g == 0)
#pragma unroll
            for (int e = 0; e < 2; ++e) part_s[slot * RT + nb * 8 + 2 * t + e] = make_float2(m[nb][e], l[nb][e]);
        }
      }
    } else {
      // Through shared memory: the free stage of each warp's ring (the next to be filled, after the last
      // barrier here) holds its state of eight rows; each warp merges some of the 16-dimension tiles.
      __syncwarp();  // every lane has read that stage
      float4* mine = reinterpret_cast<float4*>(ring + i_stage * G::kTile);
      if (lane == 0) off_s[warp] = i_stage * G::kTile;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
        for (int i = 0; i < KS; ++i) mine[i * 32 + lane] = make_float4(o[nb][i][0], o[nb][i][1], o[nb][i][2], o[nb][i][3]);
        if (g == 0)
#pragma unroll
          for (int e = 0; e < 2; ++e)
            stat_s[warp * 8 + 2 * t + e] = make_float4(m[nb][e], l[nb][e], unit[nb][e] * 0x1p-7f, 0.0f);
        named_bar_sync(1 + sub, W * 32);
        if (wt < KS) {
          const float4* stat = stat_s + sub * W * 8 + 2 * t;
          float m0 = -3.402823466e38f, m1 = m0;
#pragma unroll 2
          for (int w = 0; w < W; ++w) {
            m0 = fmaxf(m0, stat[w * 8].x);
            m1 = fmaxf(m1, stat[w * 8 + 1].x);
          }
          T *d0 = nullptr, *d1 = nullptr;
          if (whole) d0 = out_row(nb, 0), d1 = out_row(nb, 1);
#pragma unroll 1
          for (int i = wt; i < KS; i += W) {
            float4 acc = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            float l0 = 0.0f, l1 = 0.0f;
#pragma unroll 2
            for (int w = 0; w < W; ++w) {
              const float4 s0 = stat[w * 8], s1 = stat[w * 8 + 1];
              const float4 v = reinterpret_cast<const float4*>(smem + (sub * W + w) * G::kRing + off_s[sub * W + w])[i * 32 + lane];
              const float f0 = ex2(s0.x - m0), f1 = ex2(s1.x - m1);
              l0 += s0.y * f0;
              l1 += s1.y * f1;
              const float b0 = f0 * s0.z, b1 = f1 * s1.z;
              acc.x += v.x * b0, acc.y += v.y * b1, acc.z += v.z * b0, acc.w += v.w * b1;
            }
            if (whole) {
              write(d0, d1, i, acc, over(l0), over(l1));
            } else {
              part_o[((static_cast<size_t>(slot) * NB + nb) * KS + i) * 32 + lane] = acc;
              if (i == 0 && g == 0) {
                part_s[slot * RT + nb * 8 + 2 * t] = make_float2(m0, l0);
                part_s[slot * RT + nb * 8 + 2 * t + 1] = make_float2(m1, l1);
              }
            }
          }
        }
        named_bar_sync(1 + sub, W * 32);
      }
    }
    if (!whole) {
      // the teams that share the segment: those of the cuts inside it
      const int64_t s0 = place_s[0] + c_piece.u - c_piece.a, s1 = s0 + c_piece.n, span = place_s[1];
      const int t0 = static_cast<int>(s0 / span), t1 = static_cast<int>((s1 - 1) / span);
      __syncwarp();  // a team of one warp: its states are written
      if (tt == 0) flag_s[sub] = atom_add_acq_rel_gpu(p.tickets + t0, 1u) == static_cast<unsigned>(t1 - t0);
      named_bar_sync(1 + sub, W * 32);
      const bool last = flag_s[sub];
      named_bar_sync(1 + sub, W * 32);
      if (last) {
        if (tt == 0) p.tickets[t0] = 0;
        auto slot_of = [&](int c) -> int { return 2 * c + (c == t0); };
        // One pass in team order, each state rescaled to the larger maximum; several states' loads in flight.
        auto stats = [&](int c, int nb) -> float4 {  // (m, l) of the rows 2t, 2t + 1
          return __ldcg(reinterpret_cast<const float4*>(part_s + slot_of(c) * RT + nb * 8 + 2 * t));
        };
        auto state = [&](int c, int nb, int i) -> float4 {
          return __ldcg(part_o + ((static_cast<size_t>(slot_of(c)) * NB + nb) * KS + i) * 32 + lane);
        };
        struct Sum {
          float m0, m1, l0, l1, old0, old1, new0, new1;
          __device__ __forceinline__ void begin() { m0 = m1 = -3.402823466e38f, l0 = l1 = 0.0f; }
          __device__ __forceinline__ void add(const float4& z) {
            const float a0 = fmaxf(m0, z.x), a1 = fmaxf(m1, z.z);
            old0 = ex2(m0 - a0), old1 = ex2(m1 - a1), new0 = ex2(z.x - a0), new1 = ex2(z.z - a1);
            l0 = l0 * old0 + z.y * new0;
            l1 = l1 * old1 + z.w * new1;
            m0 = a0, m1 = a1;
          }
          __device__ __forceinline__ void fold(float4& acc, const float4& v) const {
            acc.x = acc.x * old0 + v.x * new0;
            acc.y = acc.y * old1 + v.y * new1;
            acc.z = acc.z * old0 + v.z * new0;
            acc.w = acc.w * old1 + v.w * new1;
          }
        };
        if (NB == 1 && W == 1) {
          Sum z;
          float4 acc[KS];
          z.begin();
#pragma unroll
          for (int i = 0; i < KS; ++i) acc[i] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 2
          for (int c = t0; c <= t1; ++c) {
            z.add(stats(c, 0));
#pragma unroll
            for (int i = 0; i < KS; ++i) z.fold(acc[i], state(c, 0, i));
          }
          T *d0 = out_row(0, 0), *d1 = out_row(0, 1);
          const float f0 = over(z.l0), f1 = over(z.l1);
#pragma unroll
          for (int i = 0; i < KS; ++i) write(d0, d1, i, acc[i], f0, f1);
        } else {
#pragma unroll 1
          for (int i = wt; i < KS; i += W) {
            Sum z[NB];
            float4 acc[NB];
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) z[nb].begin(), acc[nb] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
            for (int c = t0; c <= t1; ++c)
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) {
                z[nb].add(stats(c, nb));
                z[nb].fold(acc[nb], state(c, nb, i));
              }
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) write(out_row(nb, 0), out_row(nb, 1), i, acc[nb], over(z[nb].l0), over(z[nb].l1));
          }
        }
      }
    }
    const int b = c_piece.b;
    if (!next_piece(c_piece)) break;
    if (c_piece.b != b) {
      row0 = st.row_start[c_piece.b];
      rows_b = st.row_start[c_piece.b + 1] - row0;
      len = st.len[c_piece.b];
    }
  }
  cp_async_wait_all();
}

template <typename T, int D, int NB>
ssd_status launch(const Kv8AttnParams& p, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  if (ssd_status e = op_smem(ssd_kv8_attn_kernel<T, D, NB>, Geo<D, NB>::kTotal, ready, "ssd_kv8_attention")) return e;
  using G = Geo<D, NB>;
  return op_launch("ssd_kv8_attention", ssd_kv8_attn_kernel<T, D, NB>, dim3(kAttnSms * G::kCtas), G::kThreads, G::kTotal, s, p);
}

template <typename T, int D>
ssd_status launch_rows(int row_tile, const Kv8AttnParams& p, cudaStream_t s) {
  return row_tile == 8    ? launch<T, D, 1>(p, s)
         : row_tile == 16 ? launch<T, D, 2>(p, s)
         : row_tile == 24 ? launch<T, D, 3>(p, s)
                          : launch<T, D, 4>(p, s);
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" {

int64_t ssd_kv8_work_bytes(const ssd_kv8* c) {
  if (!kv8_shape_ok(c)) return -1;
  // two partial states per team, [rows][D] and a (maximum, sum) per row
  int64_t most = 0;
  for (int rows = 8; rows <= 32; rows += 8) {
    const AttnShape sh = attn_shape(rows, c->head_dim);
    const int64_t bytes = 2ll * kAttnSms * sh.ctas * sh.teams * rows * (c->head_dim + 2) * 4;
    most = bytes > most ? bytes : most;
  }
  return kKv8WorkHead * 4 + kAttnMaxTeams * 4 + most;
}

ssd_status ssd_kv8_attention(const ssd_kv8* c, int layer, const ssd_kv8_step* step, const void* q, void* o, int type,
                             int64_t q_row_stride, int64_t q_head_stride, int64_t o_row_stride, int64_t o_head_stride,
                             float scale, const uint32_t* row_mask, void* cuda_stream) {
  if (ssd_status s = kv8_check(c, layer)) return s;
  if (ssd_status s = kv8_check_step(c, step)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  if (step->rows == 0) return SSD_OK;
  const int64_t g = c->n_heads / c->n_kv_heads;
  if (step->rows * g * g >= 1ll << 32) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_attention: %d rows", step->rows);
  if (!q || !o) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_attention: null buffer");
  const int size = type == SSD_TYPE_FP32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(q) | reinterpret_cast<uintptr_t>(o)) % size)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_attention: q and o must be aligned to their elements");
  const OpRows qr{q, step->rows, c->n_heads, q_row_stride, q_head_stride, c->head_dim},
      outr{o, step->rows, c->n_heads, o_row_stride, o_head_stride, c->head_dim};
  if (op_overlap(qr, outr, size)) return op_fail(SSD_ERR_INVALID_ARG, "ssd_kv8_attention: o overlaps q");
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
  p.group_inv = static_cast<unsigned>((0xffffffffull + p.group) / p.group);
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
  p.part = reinterpret_cast<float*>(p.tickets + kAttnMaxTeams);
  const int tile = step_row_tile(c, step);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (type == SSD_TYPE_FP32)
    return c->head_dim == 128 ? launch_rows<float, 128>(tile, p, s) : launch_rows<float, 64>(tile, p, s);
  return c->head_dim == 128 ? launch_rows<__nv_bfloat16, 128>(tile, p, s) : launch_rows<__nv_bfloat16, 64>(tile, p, s);
}

}  // extern "C"
