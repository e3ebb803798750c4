// Products of rows and weights that are both packed to 4-bit floats.
#include "f4.cuh"

#include "tcgen05.cuh"

namespace ssd {
namespace {

struct F4MatmulParams {
  const uint8_t *w, *x;
  const uint32_t *w_rho, *x_rho;
  int n, rows, chunks;
  int early;  // the launch before writes x alone: w may be read ahead of it
  void* y;
  const void* residual;
  int64_t y_row, r_row;
};

// sum * rho_x * rho_w by two powers of two with the same sign of exponent, so that neither step leaves the range
// unless the result does.  A NaN stays one.
__device__ __forceinline__ float f4_scaled(float sum, uint32_t rho_x, uint32_t rho_w) {
  const uint32_t e = (rho_x >> 23) + (rho_w >> 23), half = e >> 1;
  const float v = sum * __uint_as_float(half << 23) * __uint_as_float((e - half) << 23);
  return max(rho_x, rho_w) >= 0x7f800000u ? __uint_as_float(0x7fc00000u) : v;
}

template <typename T>
__device__ __forceinline__ void f4_store(const F4MatmulParams& p, int m, int n, float v) {
  if (p.residual) v += to_f32(static_cast<const T*>(p.residual)[m * p.r_row + n]);
  static_cast<T*>(p.y)[m * p.y_row + n] = from_f32<T>(v);
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_barrier() {
  asm volatile("barrier.cluster.arrive.aligned;\nbarrier.cluster.wait.aligned;" ::: "memory");
}
__device__ __forceinline__ float ld_cluster(uint32_t addr, uint32_t rank) {
  uint32_t a;
  float v;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
  return v;
}

// A tile is 128 weight rows (the matrix rows, so that few x rows are few columns) by up to BN x rows.
template <int BN>
struct F4Tile {
  static constexpr int kRecords = (BN + kF4Rows - 1) / kF4Rows;  // of x
  static constexpr int kStages = BN > 128 ? 4 : BN > 64 ? 5 : 4;
  static constexpr int kCodes = BN * kF4Cols / 2, kScales = kF4Record - kF4CodeBytes;
  static constexpr int kStage = kF4Record + kCodes + kRecords * kScales;
  // tensor memory columns: the sums, then each stage's scales (16 of w, 16 of each x record)
  static constexpr int kSums = BN < 32 ? 32 : BN, kScaleCols = 16 + 16 * kRecords;
  static constexpr int kCols = kSums + kStages * kScaleCols <= 256 ? 256 : 512;
  static constexpr int kSmem = 1024 + kStages * kStage + 256 + BN * 4;
  static_assert(kSums + kStages * kScaleCols <= kCols && kCols <= 512, "tensor memory");
  static_assert(BN * kF4Rows * 4 <= kStages * kStage, "partial sums take the stages' place");
};

// Warp 0 copies records to shared memory, warp 1 issues the products, warps 2..5 read the sums.  The CTAs of a
// cluster split the columns and add up in rank order through shared memory.
template <int BN, typename T>
__global__ void __launch_bounds__(192) ssd_f4_matmul_kernel(const F4MatmulParams p) {
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
  const int n0 = blockIdx.x * kF4Rows, m0 = blockIdx.y * BN, cols = min(BN, p.rows - m0), nn = (cols + 15) / 16 * 16;
  const int split = gridDim.z, rank = blockIdx.z;
  const int c0 = static_cast<int>(static_cast<int64_t>(p.chunks) * rank / split);
  const int c1 = static_cast<int>(static_cast<int64_t>(p.chunks) * (rank + 1) / split);

  if (threadIdx.x == 0) {
    for (int s = 0; s < S::kStages; ++s) mbar_init(&full[s], 1), mbar_init(&empty[s], 1);
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
      const uint8_t* x = p.x + static_cast<int64_t>(m0 / kF4Rows) * p.chunks * kF4Record;
      const int records = (nn + kF4Rows - 1) / kF4Rows, last = nn - (records - 1) * kF4Rows;
      const uint32_t x_bytes = nn * 128 + records * S::kScales;
      auto load_w = [&](int c) {
        const int s = (c - c0) % S::kStages;
        mbar_arrive_expect_tx(&full[s], kF4Record + x_bytes);
        bulk_load(smem + s * S::kStage, w + static_cast<int64_t>(c) * kF4Record, kF4Record, &full[s]);
      };
      auto load_x = [&](int c) {
        const int s = (c - c0) % S::kStages;
        uint8_t* at = smem + s * S::kStage + kF4Record;
        for (int r = 0; r < records; ++r) {
          const uint8_t* rec = x + (static_cast<int64_t>(r) * p.chunks + c) * kF4Record;
          bulk_load(at + r * kF4CodeBytes, rec, (r + 1 < records ? kF4Rows : last) * 128, &full[s]);
          bulk_load(at + S::kCodes + r * S::kScales, rec + kF4CodeBytes, S::kScales, &full[s]);
        }
      };
      if (!p.early) pdl_wait();
      const int ahead = min(c1, c0 + S::kStages);
      for (int c = c0; c < ahead; ++c) load_w(c);
      if (p.early) pdl_wait();
      for (int c = c0; c < ahead; ++c) load_x(c);
      int c = ahead;
      for (; c < c1; ++c) {
        const int i = c - c0;
        if (!mbar_wait(&empty[i % S::kStages], (i / S::kStages - 1) & 1)) break;
        load_w(c);
        load_x(c);
      }
      if (c < c1) drain_ring(full, S::kStages, c - c0);
    }
  } else if (warp == 1) {
    if (lane == 0) {
      const uint32_t idesc = umma_idesc_f4(kF4Rows, nn);
      for (int c = c0; c < c1; ++c) {
        const int i = c - c0, s = i % S::kStages;
        if (!mbar_wait(&full[s], (i / S::kStages) & 1)) {
          ok = false;
          break;
        }
        tmem_fence_after();
        const uint32_t at = smem_u32(smem + s * S::kStage), sa = tmem + S::kSums + s * S::kScaleCols, sb = sa + 16;
#pragma unroll
        for (int kk = 0; kk < 4; ++kk) {
          tmem_copy_scales(sa + 4 * kk, umma_desc_scales(at + kF4CodeBytes + 512 * kk));
#pragma unroll
          for (int r = 0; r < S::kRecords; ++r)
            tmem_copy_scales(sb + 4 * (S::kRecords * kk + r),
                             umma_desc_scales(at + kF4Record + S::kCodes + r * S::kScales + 512 * kk));
        }
        const uint64_t a = umma_desc_sw128(at), b = umma_desc_sw128(at + kF4Record);
#pragma unroll
        for (int kk = 0; kk < 4; ++kk)  // 64 columns are 32 bytes of the 128-byte rows
          umma_f4(tmem, a + 2 * kk, b + 2 * kk, idesc, sa + 4 * kk, sb + 4 * S::kRecords * kk, i > 0 || kk > 0);
        umma_commit(&empty[s]);
      }
      if (ok) umma_commit(done);
    }
  } else {
    const int q = warp & 3, n = n0 + q * 32 + lane;
    pdl_wait();
    for (int i = threadIdx.x - 64; i < cols; i += 128) rho[i] = p.x_rho[m0 + i];
    const uint32_t rho_w = n < p.n ? p.w_rho[n] : 0u;
    named_bar_sync(1, 128);
    ok = mbar_wait(done, 0);
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
#pragma unroll
        for (int j = 0; j < 16; ++j)
          if (c + j < cols) f4_store<T>(p, m0 + c + j, n, f4_scaled(v[j], rho[c + j], rho_w));
      }
    }
  }
  pdl_trigger();
  tmem_fence_before();
  __syncthreads();
  if (split > 1) {
    cluster_barrier();
    const int i0 = cols * rank / split, i1 = cols * (rank + 1) / split, n = n0 + (threadIdx.x & 127);
    if (threadIdx.x < 128 && n < p.n) {
      const uint32_t rho_w = p.w_rho[n];
      for (int i = i0; i < i1; ++i) {
        float v = 0.0f;
        const uint32_t at = smem_u32(&part[i * kF4Rows + threadIdx.x]);
        for (int r = 0; r < split; ++r) v += ld_cluster(at, r);
        f4_store<T>(p, m0 + i, n, f4_scaled(v, rho[i], rho_w));
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

template <int BN, typename T>
ssd_status f4_launch(const F4MatmulParams& p, int split, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  constexpr int smem = F4Tile<BN>::kSmem;
  if (ssd_status e = op_smem(ssd_f4_matmul_kernel<BN, T>, smem, ready, "ssd_f4_matmul")) return e;
  const dim3 grid((p.n + kF4Rows - 1) / kF4Rows, (p.rows + BN - 1) / BN, split);
  return op_launch_cluster("ssd_f4_matmul", ssd_f4_matmul_kernel<BN, T>, grid, 192, smem, dim3(1, 1, split), s, p);
}

template <typename T>
ssd_status f4_dispatch(const F4MatmulParams& p, cudaStream_t s) {
  const int bn = p.rows <= 16 ? 16 : p.rows <= 32 ? 32 : p.rows <= 64 ? 64 : p.rows <= 128 ? 128 : 256;
  const int64_t tiles = static_cast<int64_t>((p.n + kF4Rows - 1) / kF4Rows) * ((p.rows + bn - 1) / bn);
  const int64_t slots = 152 * (bn <= 64 ? 2 : 1);
  int split = 1;
  while (split < 8 && tiles * split * 2 <= slots && split * 2 <= p.chunks) split *= 2;
  switch (bn) {
    case 16: return f4_launch<16, T>(p, split, s);
    case 32: return f4_launch<32, T>(p, split, s);
    case 64: return f4_launch<64, T>(p, split, s);
    case 128: return f4_launch<128, T>(p, split, s);
    default: return f4_launch<256, T>(p, split, s);
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
  const void* xp = packed ? x : work;
  if (!w || !x || !y || !xp || reinterpret_cast<uintptr_t>(w) % 16 || reinterpret_cast<uintptr_t>(xp) % 16)
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
  if (op_overlap(yb, wb, 1) || op_overlap(yb, pb, 1) || (!packed && op_overlap(yb, xb, 1)))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: y overlaps x, w or work");
  if (!packed && (op_overlap(pb, xb, 1) || op_overlap(pb, wb, 1) || (residual && op_overlap(pb, rb, 1))))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: work overlaps x, w or the residual");
  const bool in_place = residual == y && (rows == 1 || res_row_stride == y_row_stride);
  if (residual && !in_place && op_overlap(rb, yb, 1))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_f4_matmul: y overlaps the residual and is not the same rows");
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  if (!packed)
    if (ssd_status e = f4_pack_rows("ssd_f4_matmul", x, x_type, rows, k, x_row_stride, work, s)) return e;
  F4MatmulParams p{};
  p.w = static_cast<const uint8_t*>(w);
  p.x = static_cast<const uint8_t*>(xp);
  p.w_rho = reinterpret_cast<const uint32_t*>(p.w + f4_scales_at(n, k));
  p.x_rho = reinterpret_cast<const uint32_t*>(p.x + f4_scales_at(rows, k));
  p.n = n, p.rows = rows, p.chunks = f4_chunks(k), p.early = !packed;
  p.y = y, p.residual = residual, p.y_row = y_row_stride, p.r_row = res_row_stride;
  return type == SSD_TYPE_FP32 ? f4_dispatch<float>(p, s) : f4_dispatch<__nv_bfloat16>(p, s);
}

}  // extern "C"
