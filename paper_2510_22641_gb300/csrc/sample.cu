// Sampling: temperature, top-k, top-p, min-p and the draw by a given random number, one pass of rules per row.
#include <float.h>

#include "lowbit.cuh"

namespace ssd {
namespace {

// ------------------------------------------------------------------ masses
//
// The mass of a token is exp((l - top) / T) as an integer with 44 bits after the point, so that sums are exact in any
// order.  With y = -1024 log2(e) (top - l) / T held as a pair of floats and N = floor(y - 1/16), f = y - N,
//   2^(y / 1024) = 2^(N >> 10) * 2^((N & 1023) / 1024) * 2^(f / 1024):
// a table of 1024 values, a polynomial for 2^(f / 1024) - 1 < 2^-10, one multiplication, one shift.

constexpr int kExpBits = 10, kExpSize = 1 << kExpBits;
struct ExpTable {
  uint32_t v[kExpSize];
};
// 2^(j / 1024) * 2^31, a little less so that a value times 2^(1.07 / 1024) still fits 32 bits (the common factor
// cancels).  The Taylor series of e^x, x < ln 2, in 64 bits when this is compiled.
constexpr ExpTable make_exp_table() {
  ExpTable t = {};
  for (int j = 0; j < kExpSize; ++j) {
    const double x = 0.693147180559945309417232 * j / kExpSize;
    double sum = 1.0, term = 1.0;
    for (int i = 1; i < 24; ++i) {
      term *= x / i;
      sum += term;
    }
    t.v[j] = static_cast<uint32_t>(sum * 2147483648.0 * 0.999 + 0.5);
  }
  return t;
}
__device__ constexpr ExpTable kExpTable = make_exp_table();

// Tokens 44 octaves below the largest have none.
constexpr int kMassPlaces = 44 << kExpBits;

struct MassOf {
  float half_top, c_hi, c_lo;  // top / 2; the pair -2048 log2(e) / T

  // ~N, 65536 or more (also of a NaN) where there is no mass.  It does not fall as l falls.
  __device__ __forceinline__ int place(float l) const {
    const float t = fmaf(fmaf(-0.5f, l, half_top), c_hi, -0.0625f);
    return t > -65536.0f ? ~(__float_as_int(__fadd_rd(t, 12582912.0f)) - 0x4B400000) : 65536;
  }
  // The mass as a 32-bit number that belongs 12 - (place >> 10) places to the left.
  __device__ __forceinline__ uint32_t digits(float l, int place, const uint32_t* table) const {
    const float b = -0.5f * l, d = half_top + b, bb = d - half_top;
    const float lo = (half_top - (d - bb)) + (b - bb);  // d + lo = (top - l) / 2 exactly
    const float y = d * c_hi;
    const float e = fmaf(lo, c_hi, fmaf(d, c_lo, fmaf(d, c_hi, -y)));
    const float f = (y + static_cast<float>(place + 1)) + e;
    // 2^32 (2^(f / 1024) - 1) = f a + f^2 a^2 / 2! ..  with a = ln 2 / 1024, times 2^32
    const float q = fmaf(f, fmaf(f, fmaf(f, 0.2220f, 983.9678f), 2907270.0f), 8388608.0f);
    const uint32_t t = table[~place & (kExpSize - 1)];
    return t + __umulhi(t, __float_as_uint(q) - 0x4B000000u);
  }
  __device__ __forceinline__ uint64_t operator()(float l, const uint32_t* table) const {
    const int at = place(l);
    return at < kMassPlaces ? (static_cast<uint64_t>(digits(l, at, table)) << 12) >> (at >> kExpBits) : 0ull;
  }
};

__device__ __forceinline__ float key_value(uint32_t key) {  // the inverse of orderable
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
constexpr uint32_t kKeyNone = 0x007fffffu, kKeyInf = 0xff800000u;  // orderable(-inf), orderable(inf)

// floor(a * b / 2^64) of b = 2^64 * f, f in [0, 1); up: the ceiling.
__device__ __forceinline__ uint64_t times_fraction(uint64_t a, float f, bool up) {
  const uint64_t b = static_cast<uint64_t>(static_cast<double>(f) * 0x1p64);
  return __umul64hi(a, b) + (up && a * b != 0 ? 1 : 0);
}

struct SampleParams {
  const void* logits;
  int64_t row_stride;
  int vocab;
  const float* u;
  ssd_sampling how;
  int32_t* token;
  float* prob;
};

// ------------------------------------------------------------------ the kernel
//
// A cluster of CTAs holds a row in shared memory, read from global memory once, with the largest logit found on the way.
// A rule's border is found by counting: tokens (or their masses) are added up in 704 bins of a sixteenth of an octave of
// mass each; the bin in which the rule's count or mass is reached is split by the logits' bits into up to 704 again until
// one value is left.  All sums are of integers, so neither the atomics' order nor the cut into CTAs matters.

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32, kBins = kMassPlaces >> 6, kSegUnits = 64, kSegs = 256;
constexpr int kUses = 8;  // values that CTAs send each other, each at a place of its own

struct SampleShared {
  uint32_t table[kExpSize];
  uint64_t bin[2][kBins];   // of one search step, and of the next
  uint64_t seg[kSegs];
  uint64_t part[kSampleWarps];
  uint64_t sent[kUses][8];  // written by the CTA of that rank
  uint64_t before, at;      // what find_bin found
  int border;
};

__device__ __forceinline__ uint32_t cluster_addr(const void* p, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
  return a;
}
__device__ __forceinline__ void cluster_store(uint64_t* p, uint32_t rank, uint64_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(cluster_addr(p, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ void cluster_load2(const uint64_t* p, uint32_t rank, uint64_t& a, uint64_t& b) {
  asm volatile("ld.shared::cluster.v2.u64 {%0, %1}, [%2];" : "=l"(a), "=l"(b) : "r"(cluster_addr(p, rank)) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}

// Inclusive sum over the lanes below.
__device__ __forceinline__ uint64_t warp_scan(uint64_t v) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t t = __shfl_up_sync(~0u, v, o);
    if (lane >= o) v += t;
  }
  return v;
}
__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
#pragma unroll
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  return v;
}

template <typename T>
struct Logits16 {  // 16 bytes of a row
  static constexpr int kN = 16 / sizeof(T);
  union {
    uint4 w;
    T v[kN];
  };
};

template <typename T>
__global__ void __launch_bounds__(kSampleThreads) ssd_sample_kernel(const SampleParams p) {
  constexpr int E = Logits16<T>::kN, KS = sizeof(T) == 2 ? 16 : 0;  // keys of bf16 logits have 16 bits
  extern __shared__ __align__(16) uint8_t smem[];
  SampleShared& sh = *reinterpret_cast<SampleShared*>(smem);
  Logits16<T>* const data = reinterpret_cast<Logits16<T>*>(smem + (sizeof(SampleShared) + 15) / 16 * 16);
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int ctas = gridDim.x, rank = blockIdx.x, row = blockIdx.y, vocab = p.vocab;
  cluster_arrive();
  for (int i = tid; i < kExpSize; i += kSampleThreads) sh.table[i] = kExpTable.v[i];
  for (int i = tid; i < 2 * kBins; i += kSampleThreads) sh.bin[0][i] = 0;
  pdl_wait();
  pdl_trigger();

  // ---- this CTA's tokens [v0, v1), in units that lie in shared memory as they do in global memory; the places of the
  // first and the last unit that are not of the row hold -infinity
  const int per = (vocab + ctas - 1) / ctas, v0 = min(rank * per, vocab), v1 = min(v0 + per, vocab);
  const T* const src = static_cast<const T*>(p.logits) + row * p.row_stride + v0;
  const int phase = static_cast<int>(reinterpret_cast<uintptr_t>(src) / sizeof(T) % E);
  const int units = v1 > v0 ? (phase + v1 - v0 + E - 1) / E : 0, first_index = v0 - phase;
  float most = -INFINITY;
  auto take = [&](int u, const Logits16<T>& x) {
    data[u] = x;
#pragma unroll
    for (int e = 0; e < E; ++e) most = fmaxf(most, to_f32(x.v[e]));
  };
  if (tid < 2 && (tid == 0 || units > 1) && units > 0) {
    const int u = tid == 0 ? 0 : units - 1;
    Logits16<T> x;
    for (int e = 0; e < E; ++e) {
      const int i = u * E + e - phase;
      x.v[e] = i >= 0 && i < v1 - v0 ? src[i] : from_f32<T>(-INFINITY);
    }
    take(u, x);
  }
  {
    const uint4* in = reinterpret_cast<const uint4*>(src - phase);
    constexpr int kAhead = 4;
    for (int u = 1 + tid; u < units - 1; u += kAhead * kSampleThreads) {
      Logits16<T> x[kAhead];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (u + i * kSampleThreads < units - 1) x[i].w = in[u + i * kSampleThreads];
#pragma unroll
      for (int i = 0; i < kAhead; ++i)
        if (u + i * kSampleThreads < units - 1) take(u + i * kSampleThreads, x[i]);
    }
  }
#pragma unroll
  for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
  if (lane == 0) sh.part[warp] = __float_as_uint(most);
  cluster_wait();  // every CTA of the cluster runs
  __syncthreads();
  if (tid < ctas) {
    for (int i = 0; i < kSampleWarps; ++i) most = fmaxf(most, __uint_as_float(static_cast<uint32_t>(sh.part[i])));
    cluster_store(&sh.sent[0][rank], tid, __float_as_uint(most));
  }
  cluster_sync();
  float top = -INFINITY;
  for (int i = 0; i < ctas; ++i) top = fmaxf(top, __uint_as_float(static_cast<uint32_t>(sh.sent[0][i])));
  const uint32_t top_key = orderable(top + 0.0f);

  const ssd_sampling& h = p.how;
  const float temp = h.temperature_rows ? h.temperature_rows[row] : h.temperature;
  const float top_p = h.top_p_rows ? h.top_p_rows[row] : h.top_p;
  const float min_p = h.min_p_rows ? h.min_p_rows[row] : h.min_p;
  const int top_k = h.top_k_rows ? h.top_k_rows[row] : h.top_k;
  if (top_key <= kKeyNone) {
    if (rank == 0 && tid == 0) {
      p.token[row] = -1;
      if (p.prob) p.prob[row] = 0.0f;
    }
    return;
  }
  const bool one = !(temp >= 0x1p-100f) || top_k == 1 || top_p <= 0.0f || min_p > 1.0f;  // the first-ranked token
  const bool infinite = top_key == kKeyInf;  // only its equals have mass
  MassOf mass;
  {
    const double c = -2048.0 * 1.4426950408889634074 / static_cast<double>(one ? 1.0f : temp);
    mass.half_top = 0.5f * top;
    mass.c_hi = static_cast<float>(c);
    mass.c_lo = static_cast<float>(c - mass.c_hi);
  }
  // kept: logits above `cut`, and of those equal to it the tokens up to `last`
  float cut = infinite ? top : -FLT_MAX;
  int last = vocab - 1;
  auto kept = [&](float l, int index) { return l >= cut && (l != cut || index <= last); };
  auto place_of = [&](float l) { return infinite ? 0 : mass.place(l); };
  auto mass_of = [&](float l) -> uint64_t { return infinite ? 1ull << 44 : mass(l, sh.table); };

  // The first token in vocabulary order whose running measure exceeds aim(all of it): calls found(index, logit, all) in
  // one thread of the cluster.
  int uses = 1;
  auto walk = [&](auto measure, auto aim, auto found) {
    const int segs = (units + kSegUnits - 1) / kSegUnits;
    for (int s = warp; s < segs; s += kSampleWarps) {
      uint64_t sum = 0;
#pragma unroll
      for (int i = 0; i < kSegUnits / 32; ++i) {
        const int u = s * kSegUnits + 32 * i + lane;
        if (u < units) {
          const Logits16<T> x = data[u];
#pragma unroll
          for (int e = 0; e < E; ++e) sum += measure(to_f32(x.v[e]), first_index + u * E + e);
        }
      }
      sum = warp_sum(sum);
      if (lane == 0) sh.seg[s] = sum;
    }
    __syncthreads();
    const int each = (segs + 31) / 32;
    uint64_t mine = 0, run = 0;
    if (warp == 0) {
      for (int i = 0; i < each; ++i) mine += lane * each + i < segs ? sh.seg[lane * each + i] : 0;
      run = warp_scan(mine);
      const uint64_t sum = __shfl_sync(~0u, run, 31);
      if (lane < ctas) cluster_store(&sh.sent[uses][rank], lane, sum);
    }
    cluster_sync();
    if (warp == 0) {
      uint64_t base = 0, all = 0;
      for (int i = 0; i < ctas; ++i) {
        if (i == rank) base = all;
        all += sh.sent[uses][i];
      }
      const uint64_t goal = aim(all);
      run += base - mine;  // before this lane's segments
      const uint32_t owner = __ballot_sync(~0u, run <= goal && goal < run + mine);
      if (owner) {
        int s = 0;
        if (owner >> lane & 1)
          for (s = lane * each; goal >= run + sh.seg[s]; ++s) run += sh.seg[s];
        const int from = __ffs(owner) - 1;
        s = __shfl_sync(~0u, s, from);
        run = __shfl_sync(~0u, run, from);
        // a lane's neighbouring units
        uint64_t sum = 0;
        constexpr int kEach = kSegUnits / 32;
        const int u0 = s * kSegUnits + lane * kEach, u1 = min(u0 + kEach, units);
        for (int u = u0; u < u1; ++u)
          for (int e = 0; e < E; ++e) sum += measure(to_f32(data[u].v[e]), first_index + u * E + e);
        run += warp_scan(sum) - sum;
        if (run <= goal && goal < run + sum) {
          for (int u = u0; u < u1; ++u)
            for (int e = 0; e < E; ++e) {
              const float l = to_f32(data[u].v[e]);
              const uint64_t m = measure(l, first_index + u * E + e);
              if (run <= goal && goal < run + m) found(first_index + u * E + e, l, all);
              run += m;
            }
        }
      }
    }
    ++uses;
  };
  if (one) {
    walk([&](float l, int) -> uint64_t { return l == top; }, [](uint64_t) { return 0ull; },
         [&](int index, float, uint64_t) {
           p.token[row] = index;
           if (p.prob) p.prob[row] = 1.0f;
         });
    return;
  }

  // Adds up the cluster's bins of this step, finds the one in which the running measure reaches goal(all of it) (1 or
  // more; 0: none) and returns the goal.
  int step = 0;
  auto find_bin = [&](auto goal_of) -> uint64_t {
    cluster_sync();
    uint64_t a = 0, b = 0;
    if (tid < kBins / 2)
      for (int r = 0; r < ctas; ++r) {
        uint64_t x, y;
        cluster_load2(&sh.bin[step & 1][2 * tid], r, x, y);
        a += x, b += y;
      }
    // the other CTAs have read the bins of the step before
    for (int i = tid; i < kBins; i += kSampleThreads) sh.bin[~step & 1][i] = 0;
    uint64_t run = warp_scan(a + b);
    if (lane == 31) sh.part[warp] = run;
    __syncthreads();
    uint64_t all = 0;
    for (int i = 0; i < kSampleWarps; ++i) {
      if (i == warp) run += all;
      all += sh.part[i];
    }
    const uint64_t goal = goal_of(all), before = run - a - b;
    if (before < goal && goal <= run) {
      const bool in_b = goal > before + a;
      sh.border = 2 * tid + in_b;
      sh.before = in_b ? before + a : before;
      sh.at = in_b ? b : a;
    }
    __syncthreads();
    ++step;
    return goal;
  };
  // Shrinks the kept tokens to the shortest prefix of the ranking whose measure reaches goal_of(all of it).
  auto shrink = [&](auto measure, auto goal_of) {
    for (int u = tid; u < units; u += kSampleThreads) {
      const Logits16<T> x = data[u];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float l = to_f32(x.v[e]);
        const int at = kept(l, first_index + u * E + e) ? place_of(l) : kMassPlaces;
        if (at < kMassPlaces) atomicAdd(reinterpret_cast<unsigned long long*>(&sh.bin[step & 1][at >> 6]), measure(l));
      }
    }
    uint64_t goal = find_bin(goal_of);
    if (goal == 0) return;
    goal -= sh.before;
    // logits that the bin can hold, a place more at either end than it has
    const int bin = sh.border;
    const double unit = static_cast<double>(temp) / (1024.0 * 1.4426950408889634074);
    float low = top, high = top;
    if (!infinite) {
      low = fmaxf(__double2float_rd(top - unit * (64.0 * bin + 65.0)), -FLT_MAX);
      high = fminf(__double2float_ru(top - unit * (64.0 * bin - 1.5)), top);
    }
    uint32_t kmin = orderable(low) >> KS, kmax = orderable(high + 0.0f) >> KS;
    for (bool ready = false; !ready;) {
      const uint32_t width = kmax - kmin;  // one less than the keys
      const int shift = width < kBins ? 0 : 32 - __clz(width / kBins);
      for (int u = tid; u < units; u += kSampleThreads) {
        const Logits16<T> x = data[u];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float l = to_f32(x.v[e]);
          if (!(l >= low && l <= high)) continue;
          const uint32_t key = orderable(l + 0.0f) >> KS;
          if (key < kmin || key > kmax || !kept(l, first_index + u * E + e) || place_of(l) >> 6 != bin) continue;
          atomicAdd(reinterpret_cast<unsigned long long*>(&sh.bin[step & 1][(kmax - key) >> shift]), measure(l));
        }
      }
      find_bin([&](uint64_t) { return goal; });
      goal -= sh.before;
      kmax -= static_cast<uint32_t>(sh.border) << shift;
      kmin = max(kmin, kmax - ((1u << shift) - 1));
      ready = shift == 0;
    }
    // kmax is the border's key; its equals fall by index
    const float value = key_value(kmax & (0x80000000u >> KS) ? kmax << KS : kmax << KS | ((1u << KS) - 1));
    const uint64_t m = measure(value), wanted = (goal + m - 1) / m;
    const bool all = wanted * m >= sh.at;
    int end = vocab - 1;
    if (!all) {
      walk([&](float l, int) -> uint64_t { return l == value; }, [&](uint64_t) { return wanted - 1; },
           [&](int index, float, uint64_t) {
             for (int r = 0; r < ctas; ++r) cluster_store(&sh.sent[uses + 1][0], r, index);
           });
      cluster_sync();
      end = static_cast<int>(sh.sent[uses][0]);
      ++uses;
    } else if (value == cut) {
      end = last;
    }
    cut = value;
    last = end;
  };
  if (top_k > 1 && top_k < vocab)
    shrink([](float) { return 1ull; },
           [&](uint64_t all) -> uint64_t { return all > static_cast<uint64_t>(top_k) ? top_k : 0; });
  if (top_p < 1.0f)
    shrink([&](float l) { return mass_of(l); },
           [&](uint64_t all) -> uint64_t { return max(times_fraction(all, top_p, true), static_cast<uint64_t>(1)); });
  if (min_p > 0.0f && !infinite) {
    const double border = static_cast<double>(top) + static_cast<double>(temp) * log(static_cast<double>(min_p));
    const float b = __double2float_ru(border < top ? border : top);
    if (b > cut) cut = b, last = vocab - 1;
  }
  walk([&](float l, int index) -> uint64_t { return kept(l, index) ? mass_of(l) : 0; },
       [&](uint64_t all) -> uint64_t {
         const float u = p.u[row];
         return u >= 1.0f ? all - 1 : u > 0.0f ? times_fraction(all, u, false) : 0;
       },
       [&](int index, float l, uint64_t all) {
         p.token[row] = index;
         if (p.prob) {
           double share = 0x1p44;
           if (!infinite) {
             const int at = mass.place(l);
             share = ldexp(static_cast<double>(mass.digits(l, at, sh.table)), 12 - (at >> kExpBits));
           }
           p.prob[row] = static_cast<float>(share / static_cast<double>(all));
         }
       });
}

template <typename T>
ssd_status sample_launch(const SampleParams& p, int rows, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  constexpr int kHead = (sizeof(SampleShared) + 15) / 16 * 16, kMost = 200 << 10;
  if (ssd_status e = op_smem(ssd_sample_kernel<T>, kHead + kMost, ready, "ssd_sample")) return e;
  // CTAs of a row: as many as fill the SMs, a part of 2048 tokens or more each, and of a size that leaves room for two
  // CTAs an SM
  int ctas = 1;
  while (ctas < 8 && ((static_cast<int64_t>(rows) * ctas < 152 && p.vocab / ctas > 4096) ||
                      static_cast<int64_t>(p.vocab) * sizeof(T) / ctas > (88 << 10)))
    ctas *= 2;
  const int per = (p.vocab + ctas - 1) / ctas, bytes = per * static_cast<int>(sizeof(T)) + 32;
  for (int first = 0; first < rows; first += 65535) {  // what a grid's second dimension takes
    SampleParams q = p;
    const int n = rows - first < 65535 ? rows - first : 65535;
    q.logits = static_cast<const T*>(p.logits) + first * p.row_stride;
    q.u += first, q.token += first;
    if (q.prob) q.prob += first;
    if (q.how.temperature_rows) q.how.temperature_rows += first;
    if (q.how.top_p_rows) q.how.top_p_rows += first;
    if (q.how.min_p_rows) q.how.min_p_rows += first;
    if (q.how.top_k_rows) q.how.top_k_rows += first;
    if (ssd_status e = op_launch_cluster("ssd_sample", ssd_sample_kernel<T>, dim3(ctas, n), kSampleThreads, kHead + bytes,
                                         dim3(ctas), s, q))
      return e;
  }
  return SSD_OK;
}

}  // namespace
}  // namespace ssd

using namespace ssd;

extern "C" ssd_status ssd_sample(const void* logits, int type, int rows, int vocab, int64_t row_stride, const float* u,
                                 const ssd_sampling* how, int32_t* token, float* prob, void* cuda_stream) {
  if (type != SSD_TYPE_BF16 && type != SSD_TYPE_FP32) return op_fail(SSD_ERR_INVALID_ARG, "type %d", type);
  if (rows < 0 || vocab < 1 || vocab > SSD_SAMPLE_MAX_VOCAB)
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_sample: %d rows of %d logits", rows, vocab);
  if (rows == 0) return SSD_OK;
  if (!logits || !u || !how || !token) return op_fail(SSD_ERR_INVALID_ARG, "ssd_sample: null buffer");
  const uintptr_t words = reinterpret_cast<uintptr_t>(u) | reinterpret_cast<uintptr_t>(token) |
                          reinterpret_cast<uintptr_t>(prob) | reinterpret_cast<uintptr_t>(how->temperature_rows) |
                          reinterpret_cast<uintptr_t>(how->top_p_rows) | reinterpret_cast<uintptr_t>(how->min_p_rows) |
                          reinterpret_cast<uintptr_t>(how->top_k_rows);
  if (words % 4 || reinterpret_cast<uintptr_t>(logits) % (type == SSD_TYPE_FP32 ? 4 : 2))
    return op_fail(SSD_ERR_INVALID_ARG, "ssd_sample: buffers must be aligned to their elements");
  const SampleParams p{logits, row_stride, vocab, u, *how, token, prob};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return type == SSD_TYPE_FP32 ? sample_launch<float>(p, rows, s) : sample_launch<__nv_bfloat16>(p, rows, s);
}
