// 4-bit weights with group scales: packing, and products with 1..16 activation rows.
#include <stdlib.h>
#include "lowbit.cuh"

namespace ssd {
namespace {

// ------------------------------------------------------------------ layout
//
// [16-row tile][128-column chunk]: 1024 bytes of codes, then 16 rows x (128 / group) bf16 scales.
// A lane (g = lane / 4, t = lane % 4) of mma.m16n8k16 takes rows g and g + 8 at four columns of each
// 16-column step: 8 codes, one 32-bit word.  Its columns of steps 2 i and 2 i + 1 are 32 i + 8 t .. + 7,
// so that the matching activations are 16 contiguous bytes of a 16-bit row.  Nibble i of the low half
// and nibble i of the high half of the word form operand register i (even column in the low half), so
// one mask per register brings both codes into place.  Words of four steps make a lane's 16 bytes,
// lanes lie side by side.

constexpr int kChunk = 128;
constexpr int kCodeBytes = 16 * kChunk / 2;

__host__ __device__ constexpr int w4_record(int group) { return kCodeBytes + 16 * (kChunk / group) * 2; }
// Bit position of (row, column) in a tile's codes.
__host__ __device__ constexpr int w4_bit(int row, int col) {
  const int step = 2 * (col >> 5) + ((col >> 2) & 1), t = (col >> 3) & 3, c = col & 3;
  const int reg = (row >> 3) + 2 * (c >> 1);  // a0: row g, a1: row g + 8, a2 / a3: columns + 2
  const int nibble = reg + 4 * (c & 1);
  const int lane = (row & 7) * 4 + t;
  return (((step >> 2) * 32 + lane) * 16 + (step & 3) * 4) * 8 + nibble * 4;
}

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
    bool nan = false;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = lane + 32 * i, col = chunk * kChunk + grp * p.group + c;
      x[i] = 0.0f;
      if (c < p.group && n < p.n && col < p.k)
        x[i] = to_f32(static_cast<const T*>(p.w)[static_cast<int64_t>(n) * p.row_stride + col]);
      nan |= x[i] != x[i];
      amax = fmaxf(amax, fabsf(x[i]));
    }
    amax = warp_max(amax);
    if (__any_sync(~0u, nan)) amax = __int_as_float(0x7fc00000);
    const __nv_bfloat16 sb = __float2bfloat16_rn(amax / 7.0f);
    const float s = __bfloat162float(sb), inv = s > 0.0f ? 1.0f / s : 0.0f;
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

// ------------------------------------------------------------------ matmul
//
// y^T = W x^T by m16n8k16 products: 16 weight rows by 8 activation rows, 16 columns at a time.
//   bf16 rows are operands as they are, and codes become operands by shifts and masks alone: u = code + 8
//     goes into the mantissa of 128, 128 + u is exact in bf16, and one more product with the constant 136
//     gives what has to be taken off, sum (128 + u) x - sum 136 x = sum code x (the cancellation costs 5
//     of 24 bits, the output has 8);
//   fp32 rows are scaled per row and chunk by a power of two to 2^14 .. 2^15 and split into a high and a
//     low half (22 bits); u goes into the mantissa of the half 1024, and one subtraction (or fused
//     multiply) per pair gives the codes themselves, with no cancellation.  (u read as a subnormal half
//     would need no arithmetic, but the matrix unit aligns its sums by the exponents of the operands, so
//     a subnormal operand costs its leading zeros: 10 bits, measured 1e-5 of the result.)
// Each group's sum is multiplied by its scale in fp32 and added to the fp32 sums.
//
// Bound: bytes, n k / 2 of codes.  A chunk of 16 rows is one record of 1 KB + scales; a warp streams
// the records of MT row tiles at one chunk with cp.async into its own ring (lanes read back the bytes
// they copied; the scales are shared within the warp).  Work is the flat list of (segment of MT row
// tiles, chunk), cut into equal spans, one per team of W warps; a team's warps take a segment's chunks
// in turn and add up through shared memory.  Segments cut between teams are added in team order by the
// team that arrives last (an atomic ticket, never a wait).

constexpr int kWarps = 8;
constexpr int kThreads = 32 * kWarps;
constexpr int kMaxCtas = 304;  // two per SM
constexpr int kMaxTeams = kMaxCtas * kWarps;
constexpr int kMaxRec = kCodeBytes + 16 * 4 * 2;

struct W4Params {
  const uint8_t* packed;
  int n, chunks, per, rec, rows;  // per: groups in a chunk
  int warps;                              // per team
  const uint16_t* x;                      // 16-bit rows (bf16, or high and low halves), 16-byte aligned
  int64_t x_row, x_part;                  // elements between rows, between the high and low parts
  const float* x_scale;                   // fp32 rows: [chunk][16] powers of two
  void* y;
  const void* residual;
  int64_t y_row, r_row;
  unsigned* tickets;  // [kMaxTeams], zero between launches
  float* part;        // [2 * teams][8 NB][16 MT]
};

template <int PARTS, int NB, int MT>
struct W4Geo {
  static constexpr int kStage = MT * kMaxRec;
  static constexpr int kCtas = NB == 1 ? 2 : 1;  // per SM
  static constexpr int kStages = NB == 1 ? (MT == 1 ? 8 : MT == 2 ? 5 : 2) : (MT == 1 ? 16 : MT == 2 ? 10 : 5);
  static constexpr int kRing = kStage * kStages;
  static constexpr int kRT = 16 * MT;
  static constexpr int kPad = kRT + 4;
  static constexpr int kRec = kWarps * kRing;
  static constexpr int kFlag = kRec + kWarps * 8 * NB * kPad * 4;
  static constexpr int kTotal = kFlag + kWarps * 4;
  static_assert(kTotal * kCtas <= 231424, "shared memory");
};

template <bool BF16>
__device__ __forceinline__ void w4_mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if constexpr (BF16)
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t half2_sub(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t half2_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}

template <bool BF16>
__device__ __forceinline__ void w4_operand(uint32_t w, uint32_t (&a)[4]) {
  if constexpr (BF16) {
    a[0] = (w & 0x000f000fu) | 0x43004300u;
    a[1] = (w >> 4 & 0x000f000fu) | 0x43004300u;
    a[2] = (w >> 8 & 0x000f000fu) | 0x43004300u;
    a[3] = (w >> 12 & 0x000f000fu) | 0x43004300u;
  } else {
    const uint32_t h = w >> 8;
    a[0] = half2_sub((w & 0x000f000fu) | 0x64006400u, 0x64086408u);                  // 1024 + u - 1032
    a[1] = half2_fma((w & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, 0xd480d480u);     // (1024 + 16 u) / 16 - 72
    a[2] = half2_sub((h & 0x000f000fu) | 0x64006400u, 0x64086408u);
    a[3] = half2_fma((h & 0x00f000f0u) | 0x64006400u, 0x2c002c00u, 0xd480d480u);
  }
}

// T: type of y and the residual.  PARTS = 1: bf16 operands, 2: pairs of halves.
template <typename T, int NB, int MT, int per>  // per: groups in a chunk
__global__ void __launch_bounds__(kThreads, NB == 1 ? 2 : 1) ssd_w4_matmul_kernel(const W4Params p) {
  constexpr int PARTS = sizeof(T) == 4 ? 2 : 1;
  constexpr bool BF16 = PARTS == 1;
  using G = W4Geo<PARTS, NB, MT>;
  constexpr int RT = G::kRT;
  extern __shared__ __align__(128) uint8_t smem[];
  if constexpr (BF16) pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int W = p.warps, sub = warp / W, wt = warp - sub * W, tt = tid - sub * W * 32;
  const int teams = gridDim.x * (kWarps / W), team = blockIdx.x * (kWarps / W) + sub;
  const int n_tiles = (p.n + 15) >> 4, n_segs = (n_tiles + MT - 1) / MT, n_c = p.chunks;

  // ---- this team's span
  const int64_t total = static_cast<int64_t>(n_segs) * n_c;
  const int64_t span = n_segs <= teams ? n_c : (total + teams - 1) / teams;
  auto cut = [&](int c) -> int64_t {  // a cut in a segment short against the span moves to its nearer end
    const int64_t x = c * span;
    if (x >= total) return total;
    if (n_c > span / 4) return x;
    const int64_t in = x % n_c;
    return 2 * in < n_c ? x - in : x - in + n_c;
  };
  const int64_t u0 = cut(team), u1 = cut(team + 1);
  if (u0 >= u1) return;

  // ---- the stream of this warp's steps: MT records of one chunk
  uint8_t* ring = smem + warp * G::kRing;
  const int first_seg = static_cast<int>(u0 / n_c), first_a = static_cast<int>(u0 - static_cast<int64_t>(first_seg) * n_c);
  struct Step {
    int seg, chunk, end;  // end: of the team's part of the segment
    int64_t u;            // flat position of the segment's first chunk
  };
  auto begin = [&](Step& s) {
    s.seg = first_seg;
    s.u = u0 - first_a;
    s.end = static_cast<int>(min(static_cast<int64_t>(n_c), u1 - s.u));
    s.chunk = first_a + wt;
  };
  auto settle = [&](Step& s) -> bool {  // moves to a step that exists
    while (s.chunk >= s.end) {
      ++s.seg;
      s.u += n_c;
      if (s.u >= u1) return false;
      s.end = static_cast<int>(min(static_cast<int64_t>(n_c), u1 - s.u));
      s.chunk = wt;
    }
    return true;
  };
  Step is;
  begin(is);
  bool i_more = settle(is);
  auto issue = [&](int stage) {
    if (i_more) {
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const int tile = is.seg * MT + mt;
        if (tile < n_tiles) {
          const uint8_t* src = p.packed + (static_cast<size_t>(tile) * n_c + is.chunk) * p.rec;
          uint8_t* dst = ring + stage * G::kStage + mt * kMaxRec;
          cp_async16(dst + lane * 16, src + lane * 16);
          cp_async16(dst + 512 + lane * 16, src + 512 + lane * 16);
          if (lane < 2 * per) cp_async16(dst + kCodeBytes + lane * 16, src + kCodeBytes + lane * 16);
        }
      }
      is.chunk += W;
      i_more = settle(is);
    }
    cp_async_commit();
  };
  int i_stage = 0, stage = 0;
  for (; i_stage < G::kStages - 1; ++i_stage) issue(i_stage);
  if constexpr (!BF16) pdl_wait();  // the split rows come from the launch before, which waited for the weights
  pdl_trigger();

  // activations of one chunk: row nb * 8 + g, columns 32 i + 8 t .. + 7
  uint4 x[NB][PARTS][4];
  float2 xs[NB];
  auto load_x = [&](int chunk) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = nb * 8 + g;
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
        const uint16_t* src = p.x + k * p.x_part + r * p.x_row + static_cast<int64_t>(chunk) * kChunk + 8 * t;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          x[nb][k][i] = r < p.rows ? *reinterpret_cast<const uint4*>(src + 32 * i) : make_uint4(0, 0, 0, 0);
      }
      if constexpr (!BF16) xs[nb] = *reinterpret_cast<const float2*>(p.x_scale + chunk * 16 + nb * 8 + 2 * t);
    }
  };

  float* rec_s = reinterpret_cast<float*>(smem + G::kRec);
  volatile int* flag_s = reinterpret_cast<volatile int*>(smem + G::kFlag);
  Step cs;
  begin(cs);
  for (int a0 = first_a;; a0 = 0) {
    float y[MT][NB][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) y[mt][nb][0] = y[mt][nb][1] = y[mt][nb][2] = y[mt][nb][3] = 0.0f;
    for (; cs.chunk < cs.end; cs.chunk += W) {
      load_x(cs.chunk);
      cp_async_wait_group<G::kStages - 2>();
      __syncwarp();
      issue(i_stage);
      if (++i_stage == G::kStages) i_stage = 0;
      const uint8_t* buf = ring + stage * G::kStage;
      if (++stage == G::kStages) stage = 0;

      // what the constant offset of the codes adds, per group
      float off[4][NB][2];
      if constexpr (BF16) {
        const uint32_t a[4] = {0x43084308u, 0x43084308u, 0x43084308u, 0x43084308u};  // 136
        float s[NB][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if ((i & (4 / per - 1)) == 0)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) s[nb][0] = s[nb][1] = s[nb][2] = s[nb][3] = 0.0f;
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
            for (int k = 0; k < PARTS; ++k) {
              w4_mma<BF16>(s[nb], a, x[nb][k][i].x, x[nb][k][i].y);
              w4_mma<BF16>(s[nb], a, x[nb][k][i].z, x[nb][k][i].w);
            }
            off[i][nb][0] = s[nb][0];
            off[i][nb][1] = s[nb][1];
          }
        }
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        const uint8_t* rec = buf + mt * kMaxRec;
        const uint4 w01 = *reinterpret_cast<const uint4*>(rec + lane * 16);
        const uint4 w23 = *reinterpret_cast<const uint4*>(rec + 512 + lane * 16);
        const uint16_t* sc = reinterpret_cast<const uint16_t*>(rec + kCodeBytes);
        float c[NB][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // 32 columns
          if ((i & (4 / per - 1)) == 0)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) c[nb][0] = c[nb][1] = c[nb][2] = c[nb][3] = 0.0f;
          const uint32_t we = i == 0 ? w01.x : i == 1 ? w01.z : i == 2 ? w23.x : w23.z;
          const uint32_t wo = i == 0 ? w01.y : i == 1 ? w01.w : i == 2 ? w23.y : w23.w;
          uint32_t ae[4], ao[4];
          w4_operand<BF16>(we, ae);
          w4_operand<BF16>(wo, ao);
#pragma unroll
          for (int k = 0; k < PARTS; ++k)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              w4_mma<BF16>(c[nb], ae, x[nb][k][i].x, x[nb][k][i].y);
              w4_mma<BF16>(c[nb], ao, x[nb][k][i].z, x[nb][k][i].w);
            }
          if (((i + 1) & (4 / per - 1)) == 0) {  // end of a group
            const int grp = i / (4 / per);
            float s0 = __uint_as_float(static_cast<uint32_t>(sc[g * per + grp]) << 16);
            float s1 = __uint_as_float(static_cast<uint32_t>(sc[(g + 8) * per + grp]) << 16);
            if constexpr (!BF16) s0 *= 0x1p-14f, s1 *= 0x1p-14f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              if constexpr (BF16) {
                y[mt][nb][0] += (c[nb][0] - off[i][nb][0]) * s0;
                y[mt][nb][1] += (c[nb][1] - off[i][nb][1]) * s0;
                y[mt][nb][2] += (c[nb][2] - off[i][nb][0]) * s1;
                y[mt][nb][3] += (c[nb][3] - off[i][nb][1]) * s1;
              } else {
                y[mt][nb][0] += c[nb][0] * (s0 * xs[nb].x);
                y[mt][nb][1] += c[nb][1] * (s0 * xs[nb].y);
                y[mt][nb][2] += c[nb][2] * (s1 * xs[nb].x);
                y[mt][nb][3] += c[nb][3] * (s1 * xs[nb].y);
              }
            }
          }
        }
      }
    }

    // ---- add up the team's warps
    float* mine = rec_s + warp * (8 * NB * G::kPad);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int r = nb * 8 + 2 * t + e;
        if (r < p.rows)
#pragma unroll
          for (int mt = 0; mt < MT; ++mt) {
            mine[r * G::kPad + 16 * mt + g] = y[mt][nb][e];
            mine[r * G::kPad + 16 * mt + g + 8] = y[mt][nb][e + 2];
          }
      }
    const bool whole = a0 == 0 && cs.end == n_c;
    const int slot = team * 2 + (a0 == 0 ? 1 : 0);
    auto write_out = [&](int r, int col, const float4& v) {
      const int n0 = cs.seg * RT + col;
      const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (n0 + i < p.n) {
          const float add = p.residual ? to_f32(static_cast<const T*>(p.residual)[r * p.r_row + n0 + i]) : 0.0f;
          static_cast<T*>(p.y)[r * p.y_row + n0 + i] = from_f32<T>(e[i] + add);
        }
    };
    named_bar_sync(1 + sub, W * 32);
    for (int i = tt; i < p.rows * (RT / 4); i += W * 32) {
      const int r = i / (RT / 4), col = i % (RT / 4) * 4;
      float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
      for (int w = 0; w < W; ++w) {
        const float4 z = *reinterpret_cast<const float4*>(rec_s + ((sub * W + w) * 8 * NB + r) * G::kPad + col);
        v.x += z.x, v.y += z.y, v.z += z.z, v.w += z.w;
      }
      if (whole) write_out(r, col, v);
      else *reinterpret_cast<float4*>(p.part + (static_cast<size_t>(slot) * 8 * NB + r) * RT + col) = v;
    }
    named_bar_sync(1 + sub, W * 32);
    if (!whole) {
      const int t0 = static_cast<int>(cs.u / span), t1 = static_cast<int>((cs.u + n_c - 1) / span);
      if (tt == 0) flag_s[sub] = atom_add_acq_rel_gpu(p.tickets + t0, 1u) == static_cast<unsigned>(t1 - t0);
      named_bar_sync(1 + sub, W * 32);
      if (flag_s[sub]) {
        if (tt == 0) p.tickets[t0] = 0;
        for (int i = tt; i < p.rows * (RT / 4); i += W * 32) {
          const int r = i / (RT / 4), col = i % (RT / 4) * 4;
          float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
          for (int c = t0; c <= t1; ++c) {
            const float4 z = __ldcg(reinterpret_cast<const float4*>(
                p.part + (static_cast<size_t>(2 * c + (c == t0)) * 8 * NB + r) * RT + col));
            v.x += z.x, v.y += z.y, v.z += z.z, v.w += z.w;
          }
          write_out(r, col, v);
        }
      }
      named_bar_sync(1 + sub, W * 32);
    }
    cs.u += n_c;
    if (cs.u >= u1) break;
    ++cs.seg;
    cs.end = static_cast<int>(min(static_cast<int64_t>(n_c), u1 - cs.u));
    cs.chunk = wt;
  }
  cp_async_wait_all();
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

template <typename T, int NB, int MT, int PER>
ssd_status launch(const W4Params& p, cudaStream_t s) {
  using G = W4Geo<sizeof(T) == 4 ? 2 : 1, NB, MT>;
  static std::atomic<uint64_t> ready{0};
  if (ssd_status e = op_smem(ssd_w4_matmul_kernel<T, NB, MT, PER>, G::kTotal, ready, "ssd_w4_matmul")) return e;
  const int n_segs = ((p.n + 15) / 16 + MT - 1) / MT;
  const int teams_wanted = n_segs * ((p.chunks + 1) / 2);  // at least two chunks a team
  int grid = (teams_wanted + kWarps / p.warps - 1) / (kWarps / p.warps);
  const int one_each = (n_segs + kWarps / p.warps - 1) / (kWarps / p.warps);
  const int most = kMaxCtas / 2 * G::kCtas;
  grid = one_each <= most ? one_each : grid;
  return op_launch("ssd_w4_matmul", ssd_w4_matmul_kernel<T, NB, MT, PER>, dim3(grid > most ? most : grid), kThreads,
                   G::kTotal, s, p);
}

template <typename T, int NB, int MT>
ssd_status launch_group(const W4Params& p, cudaStream_t s) {
  return p.per == 1 ? launch<T, NB, MT, 1>(p, s) : p.per == 2 ? launch<T, NB, MT, 2>(p, s) : launch<T, NB, MT, 4>(p, s);
}

template <typename T, int NB>
ssd_status launch_tiles(const W4Params& p, cudaStream_t s) {
  const int tiles = (p.n + 15) / 16;
  int mt = tiles <= kMaxCtas ? 1 : tiles <= 2 * kMaxCtas ? 2 : 4;
  if (const char* e = getenv("W4_MT")) mt = atoi(e);
  return mt == 1 ? launch_group<T, NB, 1>(p, s) : mt == 2 ? launch_group<T, NB, 2>(p, s) : launch_group<T, NB, 4>(p, s);
}

ssd_status check_shape(int n, int k, int group) {
  if (group != 32 && group != 64 && group != 128) return op_fail(SSD_ERR_INVALID_ARG, "group %d", group);
  if (n < 1 || k < 1 || n > 16 * 65535 || k > (1 << 20))
    return op_fail(SSD_ERR_INVALID_ARG, "weight shape [%d][%d]", n, k);
  return SSD_OK;
}

// The workspace: tickets, partial sums of cut segments, activation rows in 16 bits, their scales.
struct WorkLayout {
  int64_t part, rows, scale, total;
};
WorkLayout work_layout(int k) {
  const int64_t chunks = (k + kChunk - 1) / kChunk;
  WorkLayout w;
  w.part = kMaxTeams * 4;
  w.rows = w.part + 2ll * kMaxTeams * 16 * 64 * 4;
  w.scale = w.rows + 2 * SSD_W4_MAX_ROWS * chunks * kChunk * 2;
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
  const WorkLayout lay = work_layout(k);
  uint8_t* wk = static_cast<uint8_t*>(work);
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  W4Params p = {};
  p.packed = static_cast<const uint8_t*>(packed);
  p.n = n;
  p.chunks = (k + kChunk - 1) / kChunk;
  p.per = kChunk / group;
  p.rec = w4_record(group);
  p.rows = rows;
  p.warps = p.chunks >= 16 ? 8 : p.chunks >= 8 ? 4 : p.chunks >= 4 ? 2 : 1;
  if (const char* e = getenv("W4_W")) p.warps = atoi(e);
  p.y = y;
  p.residual = residual;
  p.y_row = y_row_stride;
  p.r_row = res_row_stride;
  p.tickets = reinterpret_cast<unsigned*>(wk);
  p.part = reinterpret_cast<float*>(wk + lay.part);
  // bf16 rows that are whole chunks of aligned 16-byte pieces are operands as they lie
  if (type == SSD_TYPE_BF16 && k % kChunk == 0 && x_row_stride % 8 == 0 && reinterpret_cast<uintptr_t>(x) % 16 == 0) {
    p.x = static_cast<const uint16_t*>(x);
    p.x_row = x_row_stride;
  } else {
    p.x_row = static_cast<int64_t>(p.chunks) * kChunk;
    p.x_part = SSD_W4_MAX_ROWS * p.x_row;
    p.x_scale = reinterpret_cast<const float*>(wk + lay.scale);
    W4RowsParams r{x, x_row_stride, rows, k, p.chunks, reinterpret_cast<uint16_t*>(wk + lay.rows),
                   reinterpret_cast<float*>(wk + lay.scale)};
    p.x = r.out;
    const unsigned grid = static_cast<unsigned>((static_cast<int64_t>(rows) * p.chunks + 3) / 4);
    if (ssd_status e = type == SSD_TYPE_FP32
                           ? op_launch("ssd_w4_matmul", ssd_w4_rows_kernel<float>, dim3(grid), 128, 0, s, r)
                           : op_launch("ssd_w4_matmul", ssd_w4_rows_kernel<__nv_bfloat16>, dim3(grid), 128, 0, s, r))
      return e;
  }
  if (type == SSD_TYPE_FP32) return rows <= 8 ? launch_tiles<float, 1>(p, s) : launch_tiles<float, 2>(p, s);
  return rows <= 8 ? launch_tiles<__nv_bfloat16, 1>(p, s) : launch_tiles<__nv_bfloat16, 2>(p, s);
}

}  // extern "C"
