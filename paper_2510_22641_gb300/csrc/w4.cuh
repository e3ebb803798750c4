// 4-bit weights with group scales: the packed layout and the product kernel.
#pragma once

#include "lowbit.cuh"

namespace ssd {

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

// ------------------------------------------------------------------ matmul
//
// y^T = W x^T by m16n8k16 products: 16 weight rows by 8 activation rows, 16 columns at a time.
//   bf16 rows are operands as they are: u = code + 8 goes into the mantissa of 128, and one subtraction per
//     pair gives the codes.  (Products with 128 + u itself, less 136 times the row's sum, would save the
//     subtractions, but their rounding goes with the largest activation, seen by the weights or not: 3e-3
//     of the result beside one of 1e4, 0.4 beside 1e6.)
//   fp32 rows are scaled per row and chunk by a power of two to 2^14 .. 2^15 and split into a high and a
//     low half (22 bits, and to 2^-39 of the chunk's largest); u goes into the mantissa of the half 1024,
//     and one subtraction (or fused multiply) per pair gives the codes.  Integers put into a mantissa so are
//     a published way to unpack them (Kim et al., "Who Says Elephants Can't Run", 2022).  (u read as a
//     subnormal half would need no arithmetic, but the matrix unit aligns its sums by the exponents of the
//     operands, so a subnormal operand costs its leading zeros: 10 bits, measured 1e-5 of the result.)
// Each group's sum is multiplied by its scale in fp32 and added to the fp32 sums.
//
// Bound: bytes, n k / 2 of codes.  The row tiles are dealt out evenly, once, to the teams of W warps
// that fill the GPU; a team's warps take the chunks in turn, each for all of the team's tiles (up to MT
// at a time, sums in registers), so that a chunk's activations are fetched once per warp, and add up
// through shared memory.  No tile is shared between teams, so there are no partial sums in global memory.
// A warp streams its records (16 rows x 128 columns, 1 KB + scales) with cp.async into a ring of its own;
// lanes read back the bytes they copied, the scales are shared within the warp.
//
// Measured (device time, of the copy rate): 32000 x 4096, one bf16 row 17.3 us, 57 %; 16 rows 23.4 us, 42 %;
// one fp32 row 18.0 us, 55 %; 8 rows 22.4 us, 44 %; 16 rows 35.1 us, 28 %; 4096 x 4096, one bf16 row 4.6 us
// (launch, one round of loads, the sum).  162 to 195 instructions a record, about half of them unpacking,
// against the 180 issue slots that a record's bytes leave at the copy rate.  Neither is used up (issue 51 to
// 59 %, DRAM 37 to 48 %): 16 warps an SM (8 for 16 fp32 rows) wait for fixed latencies and the logic pipe.

constexpr int kW4Warps = 8;
constexpr int kW4Threads = 32 * kW4Warps;
constexpr int kW4MaxRec = kCodeBytes + 16 * 4 * 2;
constexpr int kW4Sms = 152;

struct W4Params {
  const uint8_t* packed;
  int n, chunks, rec, rows;
  int log_warps;      // warps per team, 1 << log_warps
  const uint16_t* x;  // 16-bit rows (bf16, or high and low halves), 16-byte aligned
  int64_t x_row, x_part;  // elements between rows, between the high and low parts
  const float* x_scale;   // fp32 rows: [chunk][16] powers of two
  void* y;
  const void* residual;
  int64_t y_row, r_row;
  int each, more;     // row tiles per team, teams that have one more
};

template <int PARTS, int NB, int MT>
struct W4Geo {
  // per SM: two, but for 16 fp32 rows, whose operands take the registers (32000 x 4096: one bf16 row with
  // one CTA 21.1 us, two 17.2; 16 bf16 rows 28.7 and 23.4; 8 fp32 rows 26.1 and 22.4)
  static constexpr int kCtas = PARTS * NB <= 2 ? 2 : 1;
  static constexpr int kStages = kCtas == 1 ? 18 : NB == 1 ? 9 : 8;  // records
  // whether the next chunk's activations are fetched ahead: where one CTA has the registers and few tiles
  // cover the wait (16 fp32 rows, 4096 x 4096: ahead 9.2 us, not ahead 9.6; 8 fp32 rows, 4096 x 4096, with
  // spills: 7.9 and 7.4; 16 bf16 rows, 32000 x 4096, with spills: 30.5 and 23.4)
  static constexpr bool kAhead = PARTS * NB == 4 && MT <= 4;
  static constexpr int kRing = kStages * kW4MaxRec;    // per warp
  static constexpr int kPart = MT > 4 ? MT / 2 : NB == 2 && MT > 2 ? 2 : MT;  // tiles merged at a time
  static constexpr int kPad = 16 * kPart + 4;
  static constexpr int kSum = kW4Warps * kRing;
  static constexpr int kTotal = kSum + kW4Warps * 8 * NB * kPad * 4;
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
__device__ __forceinline__ uint32_t bf2_sub(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t half2_fma(uint32_t a, uint32_t b, uint32_t c) {
  uint32_t r;
  asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(r) : "r"(a), "r"(b), "r"(c));
  return r;
}

// (w & mask) | bits in one instruction.
__device__ __forceinline__ uint32_t and_or(uint32_t w, uint32_t mask, uint32_t bits) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, %3, 0xEA;" : "=r"(r) : "r"(w), "r"(mask), "r"(bits));
  return r;
}

template <bool BF16>
__device__ __forceinline__ void w4_operand(uint32_t w, uint32_t (&a)[4]) {
  if constexpr (BF16) {
    a[0] = bf2_sub(and_or(w, 0x000f000fu, 0x43004300u), 0x43084308u);  // 128 + u - 136
    a[1] = bf2_sub(and_or(w >> 4, 0x000f000fu, 0x43004300u), 0x43084308u);
    a[2] = bf2_sub(and_or(w >> 8, 0x000f000fu, 0x43004300u), 0x43084308u);
    a[3] = bf2_sub(and_or(w >> 12, 0x000f000fu, 0x43004300u), 0x43084308u);
  } else {
    const uint32_t h = w >> 8;
    a[0] = half2_sub(and_or(w, 0x000f000fu, 0x64006400u), 0x64086408u);               // 1024 + u - 1032
    a[1] = half2_fma(and_or(w, 0x00f000f0u, 0x64006400u), 0x2c002c00u, 0xd480d480u);  // (1024 + 16 u) / 16 - 72
    a[2] = half2_sub(and_or(h, 0x000f000fu, 0x64006400u), 0x64086408u);
    a[3] = half2_fma(and_or(h, 0x00f000f0u, 0x64006400u), 0x2c002c00u, 0xd480d480u);
  }
}

// Parts of a row that are operands of their own products.
template <typename T, bool PAIR>
constexpr int kW4Parts = sizeof(T) == 4 && !PAIR ? 2 : 1;

// T: type of y and the residual.  bf16: bf16 operands; float: pairs of halves.  PAIR: up to four fp32 rows,
// whose high and low halves are columns r and r + 4 of one product (32000 x 4096, one row: two products
// 21.7 us, one 18.4).  per: groups in a chunk.
template <typename T, int NB, int MT, int per, bool PAIR>
__global__ void __launch_bounds__(kW4Threads, W4Geo<kW4Parts<T, PAIR>, NB, MT>::kCtas) ssd_w4_matmul_kernel(const W4Params p) {
  constexpr int PARTS = kW4Parts<T, PAIR>;
  constexpr bool BF16 = sizeof(T) == 2;
  static_assert(!PAIR || (NB == 1 && !BF16), "four rows of halves fill one block of columns");
  using G = W4Geo<PARTS, NB, MT>;
  extern __shared__ __align__(128) uint8_t smem[];
  if constexpr (BF16) pdl_wait();
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t = lane & 3;
  const int W = 1 << p.log_warps, sub = warp >> p.log_warps, wt = warp & (W - 1), tt = tid & (32 * W - 1);
  const int team = blockIdx.x * (kW4Warps >> p.log_warps) + sub;
  const int n_c = p.chunks;
  const int tile_begin = team * p.each + min(team, p.more), tile_end = tile_begin + p.each + (team < p.more);

  // ---- the stream of this warp's records: per pass of MT tiles, per chunk of the warp, the tiles
  uint8_t* ring = smem + warp * G::kRing;
  const int64_t tile_bytes = static_cast<int64_t>(n_c) * p.rec;
  int i_tile = tile_begin, i_chunk = wt, i_mt = 0;
  bool i_more = tile_begin < tile_end && wt < n_c;
  const uint8_t* i_src = p.packed + i_tile * tile_bytes + static_cast<int64_t>(i_chunk) * p.rec + lane * 16;
  auto issue = [&](int stage) {
    if (i_more) {
      uint8_t* dst = ring + stage * kW4MaxRec + lane * 16;
      cp_async16(dst, i_src);
      cp_async16(dst + 512, i_src + 512);
      if (lane < 2 * per) cp_async16(dst + kCodeBytes, i_src + kCodeBytes);
      i_src += tile_bytes;
      if (++i_mt == MT || i_tile + i_mt == tile_end) {
        i_mt = 0;
        i_chunk += W;
        if (i_chunk >= n_c) {
          i_chunk = wt;
          i_tile += MT;
          i_more = i_tile < tile_end;
        }
        i_src = p.packed + i_tile * tile_bytes + static_cast<int64_t>(i_chunk) * p.rec + lane * 16;
      }
    }
    cp_async_commit();
  };
  int i_stage = 0, stage = 0;
  for (; i_stage < G::kStages - 1; ++i_stage) issue(i_stage);
  if constexpr (!BF16) pdl_wait();  // the split rows come from the launch before, which waited for the weights
  pdl_trigger();

  // activations of one chunk: row nb * 8 + g, columns 32 i + 8 t .. + 7
  struct Rows {
    uint4 x[NB][PARTS][4];
    float2 scale[NB];
  };
  auto load_x = [&](Rows& r, int chunk) {
    if (chunk >= n_c) return;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int row = PAIR ? g & 3 : nb * 8 + g;
#pragma unroll
      for (int k = 0; k < PARTS; ++k) {
        const uint16_t* src = p.x + (PAIR ? g >> 2 : k) * p.x_part + row * p.x_row + static_cast<int64_t>(chunk) * kChunk + 8 * t;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          r.x[nb][k][i] = row < p.rows ? *reinterpret_cast<const uint4*>(src + 32 * i) : make_uint4(0, 0, 0, 0);
      }
      if constexpr (!BF16) r.scale[nb] = *reinterpret_cast<const float2*>(p.x_scale + chunk * 16 + (PAIR ? 2 * t & 3 : nb * 8 + 2 * t));
    }
  };

  float* sum_s = reinterpret_cast<float*>(smem + G::kSum);
  Rows cur, next;
  if constexpr (G::kAhead) load_x(next, wt);
  for (int tile0 = tile_begin; tile0 < tile_end; tile0 += MT) {
    const int cnt = min(MT, tile_end - tile0);
    float y[MT][NB][4];
#pragma unroll
    for (int mt = 0; mt < MT; ++mt)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) y[mt][nb][0] = y[mt][nb][1] = y[mt][nb][2] = y[mt][nb][3] = 0.0f;
    for (int chunk = wt; chunk < n_c; chunk += W) {
      if constexpr (G::kAhead) {
        cur = next;
        load_x(next, chunk + W < n_c ? chunk + W : wt);  // (the next pass begins again)
      } else {
        load_x(cur, chunk);
      }
#pragma unroll
      for (int mt = 0; mt < MT; ++mt) {
        if (mt >= cnt) break;
        cp_async_wait_group<G::kStages - 2>();
        __syncwarp();
        issue(i_stage);
        if (++i_stage == G::kStages) i_stage = 0;
        const uint8_t* rec = ring + stage * kW4MaxRec;
        if (++stage == G::kStages) stage = 0;
        const uint4 w01 = *reinterpret_cast<const uint4*>(rec + lane * 16);
        const uint4 w23 = *reinterpret_cast<const uint4*>(rec + 512 + lane * 16);
        const uint16_t* sc = reinterpret_cast<const uint16_t*>(rec + kCodeBytes);
        float c[PARTS][NB][4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {  // 32 columns
          if (i % (4 / per) == 0)
#pragma unroll
            for (int k = 0; k < PARTS; ++k)
#pragma unroll
              for (int nb = 0; nb < NB; ++nb) c[k][nb][0] = c[k][nb][1] = c[k][nb][2] = c[k][nb][3] = 0.0f;
          const uint32_t we = i == 0 ? w01.x : i == 1 ? w01.z : i == 2 ? w23.x : w23.z;
          const uint32_t wo = i == 0 ? w01.y : i == 1 ? w01.w : i == 2 ? w23.y : w23.w;
          uint32_t ae[4], ao[4];
          w4_operand<BF16>(we, ae);
          w4_operand<BF16>(wo, ao);
#pragma unroll
          for (int k = 0; k < PARTS; ++k)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) w4_mma<BF16>(c[k][nb], ae, cur.x[nb][k][i].x, cur.x[nb][k][i].y);
#pragma unroll
          for (int k = 0; k < PARTS; ++k)
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) w4_mma<BF16>(c[k][nb], ao, cur.x[nb][k][i].z, cur.x[nb][k][i].w);
          if ((i + 1) % (4 / per) == 0) {  // end of a group
            const int grp = i / (4 / per);
            float s0 = __uint_as_float(static_cast<uint32_t>(sc[g * per + grp]) << 16);
            float s1 = __uint_as_float(static_cast<uint32_t>(sc[(g + 8) * per + grp]) << 16);
            if constexpr (!BF16) s0 *= 0x1p-14f, s1 *= 0x1p-14f;
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) {
              float* v = c[0][nb];
              if constexpr (PARTS == 2)
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] += c[1][nb][e];
              if constexpr (BF16) {
                y[mt][nb][0] += v[0] * s0;
                y[mt][nb][1] += v[1] * s0;
                y[mt][nb][2] += v[2] * s1;
                y[mt][nb][3] += v[3] * s1;
              } else {
                y[mt][nb][0] += v[0] * (s0 * cur.scale[nb].x);
                y[mt][nb][1] += v[1] * (s0 * cur.scale[nb].y);
                y[mt][nb][2] += v[2] * (s1 * cur.scale[nb].x);
                y[mt][nb][3] += v[3] * (s1 * cur.scale[nb].y);
              }
            }
          }
        }
      }
    }

    // ---- add up the team's warps, kPart tiles at a time
#pragma unroll
    for (int m0 = 0; m0 < MT; m0 += G::kPart) {
      if (m0 >= cnt) break;
      float* mine = sum_s + warp * (8 * NB * G::kPad);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const int r = nb * 8 + 2 * t + e;
          if ((PAIR ? r & 3 : r) < p.rows)
#pragma unroll
            for (int mt = 0; mt < G::kPart; ++mt) {
              if (m0 + mt >= MT) break;
              mine[r * G::kPad + 16 * mt + g] = y[m0 + mt][nb][e];
              mine[r * G::kPad + 16 * mt + g + 8] = y[m0 + mt][nb][e + 2];
            }
        }
      named_bar_sync(1 + sub, W * 32);
      const int n0 = (tile0 + m0) * 16, width = min(min(cnt - m0, G::kPart) * 16, p.n - n0);
      for (int i = tt; i < p.rows * (4 * G::kPart); i += W * 32) {
        const int r = i / (4 * G::kPart), col = i % (4 * G::kPart) * 4;
        if (col >= width) continue;
        float4 v = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
        for (int w = 0; w < W; ++w)
#pragma unroll
          for (int q = PAIR ? 4 : 0; q >= 0; q -= 4) {  // low halves first
            const float4 z = *reinterpret_cast<const float4*>(sum_s + ((sub * W + w) * 8 * NB + r + q) * G::kPad + col);
            v.x += z.x, v.y += z.y, v.z += z.z, v.w += z.w;
          }
        const float e[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (col + j < width) {
            const float add = p.residual ? to_f32(static_cast<const T*>(p.residual)[r * p.r_row + n0 + col + j]) : 0.0f;
            static_cast<T*>(p.y)[r * p.y_row + n0 + col + j] = from_f32<T>(e[j] + add);
          }
      }
      named_bar_sync(1 + sub, W * 32);
    }
  }
  cp_async_wait_all();
}

template <typename T, int NB, int MT, int PER, bool PAIR>
ssd_status w4_launch(W4Params p, cudaStream_t s) {
  using G = W4Geo<kW4Parts<T, PAIR>, NB, MT>;
  static std::atomic<uint64_t> ready{0};
  if (ssd_status e = op_smem(ssd_w4_matmul_kernel<T, NB, MT, PER, PAIR>, G::kTotal, ready, "ssd_w4_matmul")) return e;
  const int tiles = (p.n + 15) / 16, per_cta = kW4Warps >> p.log_warps, most = kW4Sms * G::kCtas;
  int grid = (tiles + per_cta - 1) / per_cta;
  grid = grid < most ? grid : most;
  p.each = tiles / (grid * per_cta);
  p.more = tiles % (grid * per_cta);
  return op_launch("ssd_w4_matmul", ssd_w4_matmul_kernel<T, NB, MT, PER, PAIR>, dim3(grid), kW4Threads, G::kTotal, s, p);
}

template <typename T, int NB, int PER, bool PAIR>
ssd_status w4_launch_tiles(const W4Params& p, cudaStream_t s) {
  // the most tiles a team gets, in the fewest passes of at most kMost, evenly: a pass fetches the activations
  // anew (16 fp32 rows, 32000 x 4096: passes of 4 38.5 us, of 7 35.2; bf16: two CTAs leave 4 the registers)
  constexpr int kMost = NB == 1 || sizeof(T) == 4 ? 8 : 4;
  const int teams = kW4Sms * W4Geo<kW4Parts<T, PAIR>, NB, 1>::kCtas * (kW4Warps >> p.log_warps);
  const int tiles = ((p.n + 15) / 16 + teams - 1) / teams, passes = (tiles + kMost - 1) / kMost;
  const int mt = (tiles + passes - 1) / passes;
  if constexpr (kMost == 8) {
    if (mt > 6) return w4_launch<T, NB, 8, PER, PAIR>(p, s);
    if (mt > 4) return w4_launch<T, NB, 6, PER, PAIR>(p, s);
  }
  return mt > 3 ? w4_launch<T, NB, 4, PER, PAIR>(p, s)
         : mt > 2 ? w4_launch<T, NB, 3, PER, PAIR>(p, s)
         : mt > 1 ? w4_launch<T, NB, 2, PER, PAIR>(p, s)
                  : w4_launch<T, NB, 1, PER, PAIR>(p, s);
}

template <typename T, int NB, bool PAIR = false>
ssd_status w4_launch_group(int per, const W4Params& p, cudaStream_t s) {
  return per == 1   ? w4_launch_tiles<T, NB, 1, PAIR>(p, s)
         : per == 2 ? w4_launch_tiles<T, NB, 2, PAIR>(p, s)
                    : w4_launch_tiles<T, NB, 4, PAIR>(p, s);
}

// One translation unit each: products of bf16 / fp32 rows, up to so many of them.
ssd_status w4_matmul_bf16_8(int per, const W4Params& p, cudaStream_t s);
ssd_status w4_matmul_bf16_16(int per, const W4Params& p, cudaStream_t s);
ssd_status w4_matmul_fp32_4(int per, const W4Params& p, cudaStream_t s);
ssd_status w4_matmul_fp32_8(int per, const W4Params& p, cudaStream_t s);
ssd_status w4_matmul_fp32_16(int per, const W4Params& p, cudaStream_t s);

}  // namespace ssd
