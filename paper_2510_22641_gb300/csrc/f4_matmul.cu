// Products of rows and weights that are both packed to 4-bit floats.
#include "f4.cuh"

#include <type_traits>

#include "tcgen05_f4.cuh"

namespace ssd {
namespace {

struct F4MatmulParams {
  const uint8_t *w, *x;
  const uint32_t *w_rho, *x_rho;
  int n, rows, chunks;
  int early;  // the launch before writes x alone: w may be read ahead of it
  const void* rows_in;  // rows that are packed here (x is not looked at)
  int64_t rows_stride;
  int k, vec;
  void* y;
  const void* residual;
  int64_t y_row, r_row;
  long long limit;  // of a wait, in cycles of the SM's clock
  int hold;         // the first tile's first copy of w is left out
};

// sum * rho_x * rho_w by two powers of two with the same sign of exponent, so that neither step leaves the range
// unless the result does.  A NaN stays one.
__device__ __forceinline__ float f4_scaled(float sum, uint32_t rho_x, uint32_t rho_w) {
  const uint32_t e = (rho_x >> 23) + (rho_w >> 23), half = e >> 1;
  const float v = sum * __uint_as_float(half << 23) * __uint_as_float((e - half) << 23);
  return max(rho_x, rho_w) >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : v;
}

// Whether a scale is within 2^-60 .. 2^60, where a sum may be multiplied by one after the other.
__device__ __forceinline__ bool f4_plain(uint32_t rho) { return rho - (67u << 23) <= (120u << 23); }

// Bounded waits, of about two seconds: false when they run out.
template <typename F>
__device__ __forceinline__ bool f4_wait_for(F ready, long long limit) {
  long long start = 0;
  for (uint32_t i = 1;; ++i) {
    if (ready()) return true;
    if ((i & 1023u) != 0) continue;
    const long long now = clock64();
    if (start == 0) start = now;
    if (now - start > limit) return false;
  }
}
__device__ __forceinline__ bool f4_wait(uint64_t* bar, uint32_t parity, long long limit) {
  return f4_wait_for([&] { return mbar_try_wait(bar, parity); }, limit);
}

// N sums times their rows' scales (rho: of the x rows, in shared memory, 16-byte aligned); NaN where the sums are not
// valid.
template <int N>
__device__ __forceinline__ void f4_scale(float* v, const uint32_t* rho, uint32_t rho_w, bool plain, bool valid) {
  if (plain && valid) {
    const Float2x fw(__uint_as_float(rho_w));
#pragma unroll
    for (int j = 0; j < N; j += 4) {
      const float4 r = *reinterpret_cast<const float4*>(rho + j);
      const float2 a = (Float2x(v[j], v[j + 1]) * Float2x(r.x, r.y) * fw).get();
      const float2 b = (Float2x(v[j + 2], v[j + 3]) * Float2x(r.z, r.w) * fw).get();
      v[j] = a.x, v[j + 1] = a.y, v[j + 2] = b.x, v[j + 3] = b.y;
    }
  } else {
#pragma unroll
    for (int j = 0; j < N; ++j) v[j] = valid ? f4_scaled(v[j], rho[j], rho_w) : __uint_as_float(0x7fc00000u);
  }
}

// Stores N sums of weight row n and x rows m .. m + count - 1, res (0 where there is none) added.  rho: of the x rows, in
// shared memory.  plain: both rows' scales are f4_plain.
template <typename T, int N>
__device__ __forceinline__ void f4_store(const F4MatmulParams& p, int m, int n, int count, const float* v, const float* res,
                                         const uint32_t* rho, uint32_t rho_w, bool plain) {
  T* y = static_cast<T*>(p.y) + m * p.y_row + n;
  const float fw = __uint_as_float(rho_w);
  if (plain && count >= N) {
    T out[N];
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const float s = v[j] * __uint_as_float(rho[j]) * fw;
      out[j] = from_f32<T>(p.residual ? s + res[j] : s);
    }
#pragma unroll
    for (int j = 0; j < N; ++j, y += p.y_row) *y = out[j];
    return;
  }
#pragma unroll
  for (int j = 0; j < N; ++j, y += p.y_row) {
    if (j >= count) break;
    const float s = plain ? v[j] * __uint_as_float(rho[j]) * fw : f4_scaled(v[j], rho[j], rho_w);
    *y = from_f32<T>(p.residual ? s + res[j] : s);
  }
}
// Its residuals, all under way at once.
template <typename T, int N>
__device__ __forceinline__ void f4_residual(const F4MatmulParams& p, int m, int n, int count, float* res) {
  const T* r = static_cast<const T*>(p.residual) + m * p.r_row + n;
  T in[N] = {};
#pragma unroll
  for (int j = 0; j < N; ++j, r += p.r_row)
    if (j < count) in[j] = *r;
#pragma unroll
  for (int j = 0; j < N; ++j) res[j] = to_f32(in[j]);
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ float4 ld_cluster(uint32_t addr, uint32_t rank) {
  uint32_t a;
  float4 v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
  return v;
}

// ------------------------------------------------------------------ up to 128 rows
//
// A tile is 128 weight rows (the matrix rows, so that few x rows are few columns) by all x rows, up to BN.  The bytes of
// the weights bound it, in time the latency of 16 stages a CTA: 96 rows x 22016 x 4096 take 16.4 us with the packing of
// x (floor 9.0, two CTAs an SM; with one, in two turns, 23.6), 1 row x 4096 x 4096 6.6 us, of which the weights are 1.4.
// 33 to 64 rows have one CTA an SM, as two lack 1152 bytes of shared memory: 64 x 22016 x 4096 22.8 us, 32 rows 14.3.
template <int BN>
struct F4Tile {
  static constexpr int kStages = BN > 64 ? 3 : 4;  // two CTAs an SM, of 64 columns one
  static constexpr int kCodes = BN * kF4Cols / 2, kScales = kF4Record - kF4CodeBytes;
  static constexpr int kStage = kF4Record + kCodes + kScales;
  // tensor memory columns: the sums, then each stage's scales (16 of w, 16 of x)
  static constexpr int kSums = BN < 32 ? 32 : BN, kScaleCols = 32;
  static constexpr int kCols = 256;
  static constexpr int kSmem = 1024 + kStages * kStage + 256 + BN * 4 + 64;
  static_assert(BN <= kF4Rows && kSums + kStages * kScaleCols <= kCols, "tensor memory");
  static_assert(BN * kF4Rows * 4 <= kStages * kStage, "partial sums take the stages' place");
};

// Warp 0 copies records to shared memory, warp 1 issues the products, warps 2..5 read the sums.  The CTAs of a
// cluster split the columns and add up in rank order through shared memory.  X: void, or the type of up to four rows that
// are packed here: warps 2..5 find their largest magnitudes and write their codes and scales to the stages.
template <int BN, typename T, typename X>
__global__ void __launch_bounds__(192) ssd_f4_matmul_kernel(const F4MatmulParams p) {
  constexpr bool kPack = !std::is_void_v<X>;
  using S = F4Tile<BN>;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  uint8_t* smem = smem_raw + (((raw + 1023u) & ~1023u) - raw);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kStages * S::kStage);
  uint64_t* empty = full + S::kStages;
  uint64_t* done = empty + S::kStages;
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(done + 1);
  uint32_t* rho = reinterpret_cast<uint32_t*>(full) + 64;
  float* part = reinterpret_cast<float*>(smem);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const int n0 = blockIdx.x * kF4Rows, cols = p.rows, nn = (cols + 15) / 16 * 16;
  const int split = gridDim.z, rank = blockIdx.z;
  const int c0 = static_cast<int>(static_cast<int64_t>(p.chunks) * rank / split);
  const int c1 = static_cast<int>(static_cast<int64_t>(p.chunks) * (rank + 1) / split);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) mbar_init(&full[s], kPack ? 1 + cols : 1), mbar_init(&empty[s], 1);
    mbar_init(done, 1);
    fence_mbar_init();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)),
                 "r"(S::kCols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = *tmem_slot;
  bool ok = true;

  if (warp == 0) {
    if (lane == 0) {
      const uint8_t* w = p.w + static_cast<int64_t>(blockIdx.x) * p.chunks * kF4Record;
      const uint8_t* x = p.x;
      auto load_w = [&](int c) {
        const int s = (c - c0) % S::kStages;
        mbar_arrive_expect_tx(&full[s], kF4Record + (kPack ? 0 : nn * 128 + S::kScales));
        if (!p.hold || blockIdx.x + c > 0)
          bulk_load(smem + s * S::kStage, w + static_cast<int64_t>(c) * kF4Record, kF4Record, &full[s]);
      };
      auto load_x = [&](int c) {
        if (kPack) return;
        const int s = (c - c0) % S::kStages;
        uint8_t* at = smem + s * S::kStage + kF4Record;
        const uint8_t* rec = x + static_cast<int64_t>(c) * kF4Record;
        bulk_load(at, rec, nn * 128, &full[s]);
        bulk_load(at + S::kCodes, rec + kF4CodeBytes, S::kScales, &full[s]);
      };
      if (!p.early) pdl_wait();
      const int ahead = min(c1, c0 + S::kStages);
      for (int c = c0; c < ahead; ++c) load_w(c);
      if (p.early) pdl_wait();
      for (int c = c0; c < ahead; ++c) load_x(c);
      int c = ahead;
      for (; c < c1; ++c) {
        const int i = c - c0;
        if (!f4_wait(&empty[i % S::kStages], (i / S::kStages - 1) & 1, p.limit)) break;
        load_w(c);
        load_x(c);
      }
      if (c < c1) drain_ring(full, S::kStages, c - c0);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      pdl_wait();  // what the launch before still takes is not time that the waits below may run out in
      const uint32_t idesc = umma_idesc_f4(kF4Rows, nn);
      for (int c = c0; c < c1; ++c) {
        const int i = c - c0, s = i % S::kStages;
        if (!f4_wait(&full[s], (i / S::kStages) & 1, p.limit)) {
          ok = false;
          break;
        }
        tmem_fence_after();
        const uint32_t at = smem_u32(smem + s * S::kStage), sa = tmem + S::kSums + s * S::kScaleCols, sb = sa + 16;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          tmem_copy_scales(sa + 4 * kk, umma_desc_scales(at + kF4CodeBytes + 512 * kk));
          tmem_copy_scales(sb + 4 * kk, umma_desc_scales(at + kF4Record + S::kCodes + 512 * kk));
        }
        const uint64_t a = umma_desc_sw128(at), b = umma_desc_sw128(at + kF4Record);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)  // 64 columns are 32 bytes of the 128-byte rows
          umma_f4(tmem, a + 2 * kk, b + 2 * kk, idesc, sa + 4 * kk, sb + 4 * kk, i > 0 || kk > 0);
        umma_commit(&empty[s]);
      }
      if (ok) umma_commit(done);
    }
  } else {
    const int q = warp & 3, n = n0 + q * 32 + lane;
    pdl_wait();
    if constexpr (kPack) {
      using P = std::conditional_t<kPack, X, float>;
      const P* const x = static_cast<const P*>(p.rows_in);
      uint32_t* const part = rho + BN;  // [4 rows][4 warps]
      auto load = [&](Raw8<P>& v, int r, int c) {
        if (p.vec)
          v.template load<true>(x + r * p.rows_stride, c * kF4Cols + lane * 8, p.k);
        else
          v.template load<false>(x + r * p.rows_stride, c * kF4Cols + lane * 8, p.k);
      };
      for (int r = 0; r < cols; ++r) {
        uint32_t most = 0;
#pragma unroll 4
        for (int c = warp - 2; c < p.chunks; c += 4) {
          Raw8<P> v;
          load(v, r, c);
          most = max(most, v.amax());
        }
        most = __reduce_max_sync(~0u, most);
        if (lane == 0) part[4 * r + warp - 2] = most;
      }
      named_bar_sync(1, 128);
      int turn = 0;  // of the four warps
      for (int c = c0; c < c1 && ok; ++c) {
        const int i = c - c0, s = i % S::kStages;
        uint8_t* const at = smem + s * S::kStage + kF4Record;
        for (int r = 0; r < cols; ++r, ++turn) {
          if ((turn & 3) != warp - 2) continue;
          ok = __all_sync(~0u, i < S::kStages || f4_wait(&empty[s], (i / S::kStages - 1) & 1, p.limit));
          if (!ok) break;
          const F4Row f(max(max(part[4 * r], part[4 * r + 1]), max(part[4 * r + 2], part[4 * r + 3])));
          if (lane == 0) rho[r] = __float_as_uint(f.rho());
          Raw8<P> v;
          load(v, r, c);
          f4_put(v, v.amax(), f, at, at + S::kCodes, r);
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) mbar_arrive(&full[s]);
        }
      }
    } else {
      for (int i = threadIdx.x - 64; i < cols; i += 128) rho[i] = p.x_rho[i];
    }
    const uint32_t rho_w = n < p.n ? p.w_rho[n] : 0u;
    named_bar_sync(1, 128);
    bool plain = f4_plain(rho_w);
    for (int i = 0; i < cols; ++i) plain &= f4_plain(rho[i]);
    plain = __all_sync(~0u, plain || n >= p.n);
    float res[16] = {};
    const bool add = p.residual && split == 1 && n < p.n;
    if (add) f4_residual<T, 16>(p, 0, n, cols, res);
    ok = ok && f4_wait(done, 0, p.limit);
    if (!ok) drain_ring(full, S::kStages, c1 - c0);  // the copies under way land before their place is used or given up
    tmem_fence_after();
    for (int c = 0; c < nn; c += 16) {
      float v[16];
      tmem_ld16(tmem + (static_cast<uint32_t>(q * 32) << 16) + c, v);
      if (!ok)
        for (int j = 0; j < 16; ++j) v[j] = __uint_as_float(0x7fc00000u);
      if (split > 1) {
#pragma unroll
        for (int j = 0; j < 16; ++j) part[(c + j) * kF4Rows + q * 32 + lane] = v[j];
      } else if (n < p.n) {
        f4_store<T, 16>(p, c, n, cols - c, v, res, rho + c, rho_w, plain);
        if (add) f4_residual<T, 16>(p, c + 16, n, cols - c - 16, res);
      }
    }
  }
  pdl_trigger();
  tmem_fence_before();
  __syncthreads();
  if (split > 1) {
    // every CTA adds up a part of the x rows, four weight rows a lane, eight loads under way at a time
    cluster_barrier();
    const int i0 = cols * rank / split, i1 = cols * (rank + 1) / split, n = n0 + 4 * lane;
    const uint32_t at = smem_u32(part + 4 * lane);
    uint32_t rho_w[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) rho_w[j] = n + j < p.n ? p.w_rho[n + j] : 0;
    constexpr int kAhead = 4;
    for (int i = i0 + warp; i < i1; i += kAhead * 6) {
      float4 v[kAhead] = {};
      float res[kAhead][4] = {};
      if (p.residual)
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            if (i + 6 * k < i1 && n + j < p.n) f4_residual<T, 1>(p, i + 6 * k, n + j, 1, &res[k][j]);
      for (int r = 0; r < split; ++r) {
        float4 t[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (i + 6 * k < i1) t[k] = ld_cluster(at + (i + 6 * k) * kF4Rows * 4, r);
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          if (i + 6 * k < i1) v[k].x += t[k].x, v[k].y += t[k].y, v[k].z += t[k].z, v[k].w += t[k].w;
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (i + 6 * k >= i1) break;
        const float s[4] = {v[k].x, v[k].y, v[k].z, v[k].w};
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (n + j < p.n) f4_store<T, 1>(p, i + 6 * k, n + j, 1, s + j, &res[k][j], rho + i + 6 * k, rho_w[j], false);
      }
    }
    __syncwarp();
    cluster_barrier();  // the others still read this CTA's sums
  }
  if (warp == 1) {
    tmem_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(S::kCols) : "memory");
  }
}

// ------------------------------------------------------------------ many rows
//
// Pairs of CTAs, two SMs each, go over tiles of 256 weight rows by 256 x rows, x rows fastest, so that the pairs at work
// share few weight rows and weights are read from memory once.  A product of the pair takes 128 weight rows and half of the
// x rows from either CTA's shared memory, half the reading that 128 x 256 tiles need.  Warp 0 copies, warp 1 of the first
// CTA issues the products, warps 10..13 move the scales, warps 2..9 take a tile's sums into registers and give the tensor
// memory back before they store them.
//
// What bounds it is the matrix pipe (59 % busy) with the barriers around each stage: 5003 x 27648 x 5120 take 274 us with
// the packing of x (22), 5.2 PFLOP/s (a library bf16 product of that size at its best rate: 730).  Scales copied
// by tcgen05.cp: 386 (one CTA a tile of 128 x 256, sums read by eight warps; 507 with four, before).  640 x 4096 x 11008,
// 48 tiles for 76 pairs: 28 us, 51 before.

__device__ __forceinline__ uint32_t cluster_map(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
// Arrives at another CTA's barrier.  What it tells of lies in tensor memory (written, and fenced by tcgen05.fence) or came
// by bulk copies whose own barrier was waited for; no ordinary store is published, so cluster-wide release and acquire,
// which cost 700 cycles a stage, are not needed.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// The products issued so far arrive at this barrier of both CTAs when they are done.
__device__ __forceinline__ void umma_commit_pair(uint64_t* bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(smem_u32(bar)),
      "h"(static_cast<uint16_t>(3))
      : "memory");
}

constexpr int kF4PairThreads = 448;
struct F4Pair {
  static constexpr int kStages = 5;
  static constexpr int kCodes = 128 * 128, kScales = kF4Record - kF4CodeBytes;  // half of the x rows' codes; all their scales
  static constexpr int kStage = kF4Record + kCodes + 2 * kScales;
  static constexpr int kSums = 256, kScaleCols = 16 + 32;
  static constexpr int kSmem = 1024 + kStages * kStage + 256 + 2 * 256 * 4;
  static_assert(kSums + kStages * kScaleCols <= 512, "tensor memory");
};

template <typename T>
__global__ void __launch_bounds__(kF4PairThreads, 1) ssd_f4_matmul_pair_kernel(const F4MatmulParams p) {
  using S = F4Pair;
  constexpr int BN = 256;
  extern __shared__ uint8_t smem_raw[];
  const uint32_t raw = smem_u32(smem_raw);
  uint8_t* smem = smem_raw + (((raw + 1023u) & ~1023u) - raw);
  uint64_t* full = reinterpret_cast<uint64_t*>(smem + S::kStages * S::kStage);
  uint64_t* empty = full + S::kStages;
  uint64_t* scaled = empty + S::kStages;  // a stage's scales are in both CTAs' tensor memory (the first one's barrier)
  uint64_t* done = scaled + S::kStages;   // a tile's sums are complete
  uint64_t* taken = done + 1;             // and in registers, of both CTAs (the first one's barrier)
  uint32_t* tmem_slot = reinterpret_cast<uint32_t*>(taken + 1);
  volatile int* stop = reinterpret_cast<volatile int*>(tmem_slot + 1);
  uint32_t* rho = reinterpret_cast<uint32_t*>(full) + 64;  // [2][256]: of this tile and of the next
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, rank = cluster_rank();
  const int w_tiles = (p.n + kF4Rows - 1) / kF4Rows, tiles_m = (p.rows + BN - 1) / BN, tiles = tiles_m * ((w_tiles + 1) / 2);
  const int first = blockIdx.x / 2, step = gridDim.x / 2;

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) mbar_init(&full[s], 1), mbar_init(&empty[s], 1), mbar_init(&scaled[s], 8);
    mbar_init(done, 1);
    mbar_init(taken, 16);
    *stop = 0;
    fence_mbar_init();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
  }
  tmem_fence_before();
  __syncthreads();
  cluster_barrier();
  tmem_fence_after();
  const uint32_t tmem = *tmem_slot;
  pdl_wait();
  pdl_trigger();

  // columns of a tile: a multiple of 32, as each CTA holds half of them
  auto tile_cols = [&](int m0) { return (min(BN, p.rows - m0) + 31) / 32 * 32; };
  if (warp == 0) {
    // ---- copies, one a lane: the weight record; the CTA's half of the x codes, from up to two records; their scales
    int s = 0, phase = 1;
    bool ok = true;
    for (int t = first; t < tiles && ok; t += step) {
      const int m0 = t % tiles_m * BN, nt = min(t / tiles_m * 2 + rank, w_tiles - 1);
      const int half = tile_cols(m0) / 2, records = (2 * half + kF4Rows - 1) / kF4Rows;
      const int r0 = rank * half, r = (lane - 1) & 1;                                      // this CTA's first x row; record
      const int a = max(r0 - r * kF4Rows, 0), e = min(r0 + half - r * kF4Rows, kF4Rows);   // its rows of that record
      const uint8_t* src = p.x + (static_cast<int64_t>(m0 / kF4Rows) + r) * p.chunks * kF4Record;
      int to = 0;
      uint32_t size = 0;
      if (lane == 0) {
        src = p.w + static_cast<int64_t>(nt) * p.chunks * kF4Record;
        size = kF4Record;
      } else if (lane < 3 && a < e) {
        src += a * 128;
        to = kF4Record + (r * kF4Rows + a - r0) * 128;
        size = (e - a) * 128;
      } else if ((lane == 3 || lane == 4) && r < records) {
        src += kF4CodeBytes;
        to = kF4Record + S::kCodes + r * S::kScales;
        size = S::kScales;
      }
      const uint32_t bytes = kF4Record + half * 128 + records * S::kScales;
      for (int c = 0; c < p.chunks; ++c, src += kF4Record) {
        ok = __all_sync(~0u, !*stop && f4_wait(&empty[s], phase, p.limit));
        if (!ok) break;
        if (lane == 0) mbar_arrive_expect_tx(&full[s], bytes);
        __syncwarp();
        if (size && (!p.hold || blockIdx.x + t + c + lane > 0))
          bulk_load(smem + s * S::kStage + to, src, size, &full[s]);
        if (++s == S::kStages) s = 0, phase ^= 1;
      }
    }
    if (!ok) *stop = 1;
    // The copies under way land before the CTA leaves, whoever gave up waiting for them.
    for (int i = 0; i < S::kStages; ++i) mbar_wait_for(&full[i], i < s ? phase ^ 1 : phase, 100000000ull);
  } else if (warp == 1) {
    if (lane == 0 && rank == 0) {
      int s = 0, phase = 0, it = 0;
      bool ok = true;
      const uint64_t a0 = umma_desc_sw128(smem_u32(smem)), b0 = umma_desc_sw128(smem_u32(smem) + kF4Record);
      for (int t = first; t < tiles && ok; t += step, ++it) {
        const uint32_t idesc = umma_idesc_f4(2 * kF4Rows, tile_cols(t % tiles_m * BN));
        if (*stop || !f4_wait(taken, (it & 1) ^ 1, p.limit)) break;
        tmem_fence_after();
        uint32_t more = 0;
        for (int c = 0; c < p.chunks; ++c) {
          ok = f4_wait(&full[s], phase, p.limit) && f4_wait(&scaled[s], phase, p.limit);
          if (!ok) break;
          tmem_fence_after();
          const uint32_t sa = tmem + S::kSums + s * S::kScaleCols, sb = sa + 16;
          const uint64_t a = a0 + s * (S::kStage >> 4), b = b0 + s * (S::kStage >> 4);
#pragma unroll
          for (int kk = 0; kk < 4; ++kk) {
            umma_f4<2>(tmem, a + 2 * kk, b + 2 * kk, idesc, sa + 4 * kk, sb + 8 * kk, more);
            more = 1;
          }
          umma_commit_pair(&empty[s]);
          if (++s == S::kStages) s = 0, phase ^= 1;
        }
        if (ok) umma_commit_pair(done);
      }
    }
  } else if (warp >= 10) {
    // ---- the scales, from shared to tensor memory by way of registers: as copies (tcgen05.cp) they go through the
    // products' pipe, 48 cycles for 512 bytes, 12 of them a stage whose four products take 512
    const uint32_t quarter = static_cast<uint32_t>((warp & 3) * 32) << 16;
    int s = 0, phase = 0;
    bool ok = true;
    const uint32_t arrive0 = cluster_map(scaled, 0);
    for (int t = first; t < tiles && ok; t += step)
      for (int c = 0; c < p.chunks; ++c) {
        ok = __all_sync(~0u, !*stop && f4_wait(&full[s], phase, p.limit));
        if (!ok) break;
        const uint8_t* at = smem + s * S::kStage + kF4CodeBytes + lane * 16;
        const uint32_t to = tmem + quarter + S::kSums + s * S::kScaleCols;
        uint4 v[4];
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) v[kk] = *reinterpret_cast<const uint4*>(at + 512 * kk);
        tmem_st16(to, reinterpret_cast<const uint32_t*>(v));
        at += kF4Record - kF4CodeBytes + S::kCodes;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
          for (int kk = 0; kk < 4; ++kk)
            v[kk] = *reinterpret_cast<const uint4*>(at + (kk & 1) * S::kScales + 512 * (2 * h + (kk >> 1)));
          tmem_st16(to + 16 + 16 * h, reinterpret_cast<const uint32_t*>(v));
        }
        tmem_wait_st();
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(arrive0 + 8 * s);
        if (++s == S::kStages) s = 0, phase ^= 1;
      }
  } else {
    const int q = warp & 3, half = (warp - 2) >> 2, i = threadIdx.x - 64;
    const uint32_t taken_bar = cluster_map(taken, 0);
    int it = 0;
    for (int t = first; t < tiles; t += step, ++it) {
      const int m0 = t % tiles_m * BN, n = (t / tiles_m * 2 + rank) * kF4Rows + q * 32 + lane, cols = min(BN, p.rows - m0);
      uint32_t* rx = rho + (it & 1) * BN;
      const uint32_t mine = i < cols ? p.x_rho[m0 + i] : 127u << 23;
      rx[i] = mine;
      const uint32_t rho_w = n < p.n ? p.w_rho[n] : 127u << 23;
      int plain;
      asm volatile(
          "{\n .reg .pred p, q;\n setp.ne.b32 p, %1, 0;\n barrier.cta.red.and.pred q, 1, 256, p;\n selp.b32 %0, 1, 0, q;\n}"
          : "=r"(plain)
          : "r"(static_cast<int>(f4_plain(mine) && f4_plain(rho_w)))
          : "memory");
      // 128 columns a warp
      const int left = cols - half * (BN / 2);
      const bool store = n < p.n;
      [[maybe_unused]] uint32_t h[sizeof(T) == 2 ? BN / 4 : 1];  // pairs of bf16: the residual's, then the results
      if constexpr (sizeof(T) == 2) {
        if (p.residual) {
          const uint16_t* r = static_cast<const uint16_t*>(p.residual) + (m0 + half * (BN / 2)) * p.r_row + n;
#pragma unroll
          for (int j = 0; j < BN / 2; j += 2, r += 2 * p.r_row) {
            const uint32_t a = store && j < left ? *r : 0u, b = store && j + 1 < left ? r[p.r_row] : 0u;
            h[j / 2] = a | b << 16;
          }
        }
      }
      // of fp32 residuals 16 are under way ahead of the 16 that are added
      [[maybe_unused]] float ahead[sizeof(T) == 4 ? 16 : 1];
      [[maybe_unused]] const T* res = static_cast<const T*>(p.residual) + (m0 + half * (BN / 2)) * p.r_row + n;
      auto fetch = [&](int from) {
#pragma unroll
        for (int j = 0; j < static_cast<int>(sizeof(ahead) / sizeof(float)); ++j)
          ahead[j] = store && from + j < left ? to_f32(res[(from + j) * p.r_row]) : 0.0f;
      };
      if (sizeof(T) == 4 && p.residual) fetch(0);
      const bool ok = !*stop && f4_wait(done, it & 1, p.limit);  // after a failure the rest is NaN
      tmem_fence_after();
      // bf16 results are scaled and packed as they are read, 32 at a time, fp32 ones take two turns of 64: the registers of
      // 14 warps hold no more.  The tensor memory is given back after the last read.
      const uint32_t from = tmem + (static_cast<uint32_t>(q * 32) << 16) + half * (BN / 2);
      auto release = [&] {
        tmem_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive_cluster(taken_bar);
      };
      if (!ok) *stop = 1;
      rx += half * (BN / 2);
      if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int c = 0; c < BN / 2; c += 32) {
          float v[32];
          tmem_ld32(from + c, v);
          f4_scale<32>(v, rx + c, rho_w, plain, ok);
#pragma unroll
          for (int j = 0; j < 32; j += 2) {
            if (p.residual) {
              const float2 r = bf16x2_to_float2(h[(c + j) / 2]);
              v[j] += r.x, v[j + 1] += r.y;
            }
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[j], v[j + 1]);
            h[(c + j) / 2] = *reinterpret_cast<const uint32_t*>(&b);
          }
        }
        release();
        if (store) {
          __nv_bfloat16* y = static_cast<__nv_bfloat16*>(p.y) + (m0 + half * (BN / 2)) * p.y_row + n;
          if (left >= BN / 2) {
#pragma unroll
            for (int j = 0; j < BN / 2; ++j, y += p.y_row) *y = __ushort_as_bfloat16(static_cast<uint16_t>(h[j / 2] >> (16 * (j & 1))));
          } else {
#pragma unroll
            for (int j = 0; j < BN / 2; ++j, y += p.y_row)
              if (j < left) *y = __ushort_as_bfloat16(static_cast<uint16_t>(h[j / 2] >> (16 * (j & 1))));
          }
        }
      } else {
#pragma unroll
        for (int c = 0; c < BN / 2; c += 64) {
          float v[64];
          tmem_ld32(from + c, v);
          tmem_ld32(from + c + 32, v + 32);
          if (c + 64 == BN / 2) release();
          f4_scale<64>(v, rx + c, rho_w, plain, ok);
          T* y = static_cast<T*>(p.y) + (m0 + half * (BN / 2) + c) * p.y_row + n;
#pragma unroll
          for (int b = 0; b < 64; b += 16) {
            if (p.residual) {
#pragma unroll
              for (int j = 0; j < 16; ++j) v[b + j] += ahead[j];
              if (c + b + 16 < BN / 2) fetch(c + b + 16);
            }
#pragma unroll
            for (int j = 0; j < 16; ++j, y += p.y_row)
              if (store && c + b + j < left) *y = v[b + j];
          }
        }
      }
    }
  }
  tmem_fence_before();
  __syncthreads();
  cluster_barrier();  // neither CTA leaves while the pair's products or arrivals may touch it
  if (warp == 1) {
    tmem_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512) : "memory");
  }
}

template <typename T>
ssd_status f4_launch_pair(const F4MatmulParams& p, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  if (ssd_status e = op_smem(ssd_f4_matmul_pair_kernel<T>, F4Pair::kSmem, ready, "ssd_f4_matmul")) return e;
  const int64_t tiles = static_cast<int64_t>((p.n + 255) / 256) * ((p.rows + 255) / 256);
  if (tiles > 0x3fffffff) return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: %d rows of %d", p.rows, p.n);
  return op_launch_cluster("ssd_f4_matmul", ssd_f4_matmul_pair_kernel<T>, dim3(tiles < 76 ? 2 * static_cast<unsigned>(tiles) : 152u),
                           kF4PairThreads, F4Pair::kSmem, dim3(2), s, p);
}

template <int BN, typename T, typename X = void>
ssd_status f4_launch(const F4MatmulParams& p, int split, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  constexpr int smem = F4Tile<BN>::kSmem;
  if (ssd_status e = op_smem(ssd_f4_matmul_kernel<BN, T, X>, smem, ready, "ssd_f4_matmul")) return e;
  const dim3 grid((p.n + kF4Rows - 1) / kF4Rows, 1, split);
  return op_launch_cluster("ssd_f4_matmul", ssd_f4_matmul_kernel<BN, T, X>, grid, 192, smem, dim3(1, 1, split), s, p);
}

template <typename T>
ssd_status f4_dispatch(const F4MatmulParams& p, int x_type, cudaStream_t s) {
  if (p.rows > 128) return f4_launch_pair<T>(p, s);
  const int bn = p.rows <= 16 ? 16 : p.rows <= 32 ? 32 : p.rows <= 64 ? 64 : 128;
  const int tiles = (p.n + kF4Rows - 1) / kF4Rows;
  // A cluster shares a tile's columns as long as that leaves a CTA an SM (1 x 4096 x 4096: one CTA a tile 11.2 us, four
  // 7.1; with more CTAs than places the clusters wait for each other: 64 x 11008 x 4096, where an SM takes one CTA, one a
  // tile 12.4, two 20.5.  Between one and two CTAs an SM the sizes that have room for two were not measured).
  int split = 1;
  while (split < 8 && tiles * split * 2 <= 152 && split * 2 <= p.chunks) split *= 2;
  if (p.rows_in)
    return x_type == SSD_TYPE_FP32 ? f4_launch<16, T, float>(p, split, s) : f4_launch<16, T, __nv_bfloat16>(p, split, s);
  switch (bn) {
    case 16: return f4_launch<16, T>(p, split, s);
    case 32: return f4_launch<32, T>(p, split, s);
    case 64: return f4_launch<64, T>(p, split, s);
    default: return f4_launch<128, T>(p, split, s);
  }
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" {

ssd_status ssd_f4_matmul(const void* w, int n, int k, const void* x, int x_type, int rows, int64_t x_row_stride, void* y,
                         int type, int64_t y_row_stride, const void* residual, int64_t res_row_stride, void* work,
                         void* cuda_stream) {
  if (ssd_status s = f4_check_shape(n, k)) return s;
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  const bool packed = x_type == SSD_TYPE_F4;
  if (!packed && x_type != SSD_TYPE_BF16 && x_type != SSD_TYPE_FP32)
    return op_fail(SSD_ERR_INVALID_ARG, "x_type %d", x_type);
  if (rows == 0) return SSD_OK;
  if (ssd_status s = f4_check_shape(rows, k)) return s;
  const bool inside = !packed && f4_packs_inside(rows, k);
  const void* xp = packed || inside ? x : work;
  if (!w || !x || !y || !xp || reinterpret_cast<uintptr_t>(w) % 16 || (!inside && reinterpret_cast<uintptr_t>(xp) % 16))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: null or unaligned buffer");
  const int size = type == SSD_TYPE_FP32 ? 4 : 2, xsize = x_type == SSD_TYPE_FP32 ? 4 : 2;
  if ((reinterpret_cast<uintptr_t>(y) | reinterpret_cast<uintptr_t>(residual)) % size ||
      (!packed && reinterpret_cast<uintptr_t>(x) % xsize))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: rows must be aligned to their elements");
  const int64_t wbytes = ssd_f4_bytes(n, k), xbytes = ssd_f4_bytes(rows, k);
  const OpRows yb{y, rows, 1, y_row_stride * size, 0, static_cast<int64_t>(n) * size}, wb{w, 1, 1, 0, 0, wbytes},
      pb{xp, 1, 1, 0, 0, xbytes}, xb{x, rows, 1, x_row_stride * xsize, 0, static_cast<int64_t>(k) * xsize},
      rb{residual, rows, 1, res_row_stride * size, 0, static_cast<int64_t>(n) * size};
  if (!op_apart(yb)) return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: rows of y overlap");
  if (op_overlap(yb, wb, 1) || (!inside && op_overlap(yb, pb, 1)) || (!packed && op_overlap(yb, xb, 1)))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: y overlaps x, w or work");
  if (!packed && !inside && (op_overlap(pb, xb, 1) || op_overlap(pb, wb, 1) || (residual && op_overlap(pb, rb, 1))))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: work overlaps x, w or the residual");
  const bool in_place = residual == y && (rows == 1 || res_row_stride == y_row_stride);
  if (residual && !in_place && op_overlap(rb, yb, 1))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: y overlaps the residual and is not the same rows");
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (!packed && !inside)
    if (ssd_status e = f4_pack_rows("ssd_f4_matmul", x, x_type, rows, k, x_row_stride, work, s)) return e;
  F4MatmulParams p{};
  p.w = static_cast<const uint8_t*>(w);
  p.x = static_cast<const uint8_t*>(xp);
  p.w_rho = reinterpret_cast<const uint32_t*>(p.w + f4_scales_at(n, k));
  p.x_rho = reinterpret_cast<const uint32_t*>(p.x + f4_scales_at(rows, k));
  p.n = n, p.rows = rows, p.chunks = f4_chunks(k), p.early = !packed && !inside, p.k = k;
  if (inside) {
    p.rows_in = x, p.rows_stride = x_row_stride;
    p.vec = reinterpret_cast<uintptr_t>(x) % 16 == 0 && (rows == 1 || x_row_stride % (16 / xsize) == 0);
  }
  p.y = y, p.residual = residual, p.y_row = y_row_stride, p.r_row = res_row_stride;
  const OpWait wait = op_wait();
  p.limit = 2 * wait.ns, p.hold = wait.hold;
  return type == SSD_TYPE_FP32 ? f4_dispatch<float>(p, x_type, s) : f4_dispatch<__nv_bfloat16>(p, x_type, s);
}

}  // extern "C"
