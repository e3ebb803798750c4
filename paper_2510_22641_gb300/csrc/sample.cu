// Sampling: temperature, top-k, top-p, min-p and the draw by a given random number.
#include <float.h>

#include "lowbit.cuh"

namespace ssd {
namespace {

// ------------------------------------------------------------------ masses
//
// The mass of a token is exp((l - top) / T) up to a factor that is the same for the whole row, as an integer with 44 bits
// after the point, so that sums are exact in any order.  With c = 1024 log2(e) / T as a pair of floats, n = l c_hi rounded
// to an integer, f = l c - n (by fused multiply-adds, to 2^-25) and a token's place n(top) - n(l),
//   exp(l / T) 2^(-n(top) / 1024) = 2^-(place >> 10) * 2^(-(place & 1023) / 1024) * 2^(f / 1024):
// a table of 1024 values, a polynomial, one multiplication, one shift.  |f| is at most 1/2 + |l c_lo|, and c_lo at most
// 1.22 * 2^-24 c, so with |l c| below 2^20 + 44 * 1024 it stays below 0.58.  (Up to 2^21 it reached 0.65, past the 0.6 that
// the polynomial is moved by, where a mass was off by 2^-9.)

constexpr int kExpBits = 10, kExpSize = 1 << kExpBits;
struct ExpTable {
  uint32_t v[kExpSize];
};
// 2^(-j / 1024) * 2^32, less so that a value times 2^((0.6 + f) / 1024), at most 2^(1.18 / 1024), fits 32 bits (the common
// factor cancels).  The Taylor series of e^x, 0 <= x < ln 2, in 64 bits when this is compiled.
constexpr ExpTable make_exp_table() {
  ExpTable t = {};
  for (int j = 0; j < kExpSize; ++j) {
    const double x = 0.693147180559945309417232 * (kExpSize - j) / kExpSize;
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

// Tokens 44 octaves below the largest have no mass.
constexpr uint32_t kMassPlaces = 44u << kExpBits;

struct MassOf {
  float origin;      // 0; the largest logit where c times it is 2^20 or more (then l - origin is exact wherever there is
                     // mass)
  float c_hi, c_lo;  // 1024 log2(e) / T
  uint32_t top;      // bits of the largest logit's `number`

  // 1.5 * 2^23 + n as a float; it does not fall as l rises.
  __device__ __forceinline__ float number(float l) const { return fmaf(l - origin, c_hi, 12582912.0f); }
  // kMassPlaces or more: no mass (also for -infinity and NaN, whose bits are far away).
  __device__ __forceinline__ uint32_t place(float l) const { return top - __float_as_uint(number(l)); }
  // The mass as a 32-bit number that belongs 12 - (place >> 10) places to the left.  Of infinite logits f is a NaN, whose
  // bits make the same digits for all of them.
  __device__ __forceinline__ uint32_t digits(float l, uint32_t place, const uint32_t* table) const {
    const float x = l - origin, n = number(l) - 12582912.0f;
    const float f = fmaf(x, c_lo, fmaf(x, c_hi, -n));
    // 2^32 (2^((f + 0.6) / 1024) - 1), the series at f = 0: with a = ln 2 / 1024, 2^32 e^(0.6 a) (1 + a f + a^2 f^2 / 2! ..) - 2^32
    const float q = fmaf(f, fmaf(f, fmaf(f, 0.22210662f, 984.36748f), 2908451.0f), 8388608.0f + 1744716.25f);
    const uint32_t t = table[place & (kExpSize - 1)];
    return t + __umulhi(t, __float_as_uint(q) & 0x7fffffu);
  }
  // Places and digits of two logits, the same bits.
  __device__ __forceinline__ void two(float l, float m, const uint32_t* table, uint32_t* place, uint32_t* w) const {
    const Float2x x = Float2x(l, m) + Float2x(-origin), c(c_hi), one(12582912.0f), n = fma2(x, c, one);
    const Float2x f = fma2(x, Float2x(c_lo), fma2(x, c, fma2(n, Float2x(-1.0f), one)));
    const Float2x q = fma2(f, fma2(f, fma2(f, Float2x(0.22210662f), Float2x(984.36748f)), Float2x(2908451.0f)),
                           Float2x(8388608.0f + 1744716.25f));
    const float2 ns = n.get(), qs = q.get();
    place[0] = top - __float_as_uint(ns.x), place[1] = top - __float_as_uint(ns.y);
    const uint32_t t = table[place[0] & (kExpSize - 1)], u = table[place[1] & (kExpSize - 1)];
    w[0] = t + __umulhi(t, __float_as_uint(qs.x) & 0x7fffffu);
    w[1] = u + __umulhi(u, __float_as_uint(qs.y) & 0x7fffffu);
  }
  // A mass in whole units of 2^-44 from its 12th octave on, where they fit 32 bits, and before that in digits, which are
  // exact: sums of these are sums of values, in any order and grouping.  (Digits added up and then shifted keep the bits
  // below 2^-44, as many as their sums are cut into: borders could move by a token with the number of CTAs.)
  static __device__ __forceinline__ uint32_t units(uint32_t w, uint32_t place) {
    return __funnelshift_rc(w, 0u, max(static_cast<int>(place >> kExpBits) - 12, 0));
  }
  static __device__ __forceinline__ int unit_bits(int bin) { return max(12 - (bin >> 4), 0); }  // of a bin's units
  static __device__ __forceinline__ uint64_t value(uint32_t w, uint32_t place) {
    const uint64_t v = static_cast<uint64_t>(w) << 12 >> (place >> kExpBits & 63);
    return place < kMassPlaces ? v : 0ull;
  }
  __device__ __forceinline__ uint64_t operator()(float l, const uint32_t* table) const {
    const uint32_t at = place(l);
    return value(digits(l, at, table), at);
  }
};

__device__ __forceinline__ float key_value(uint32_t key) {  // the inverse of orderable
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
constexpr uint32_t kKeyNone = 0x007fffffu;  // orderable(-infinity)

// floor(a * f) of f in [0, 1), f's digits below 2^-64 cut off; up: the ceiling.  In integers: a 64-bit float operation
// costs an SM of this GPU 16 cycles a warp.
__device__ __forceinline__ uint64_t times_fraction(uint64_t a, float f, bool up) {
  const int e = static_cast<int>(__float_as_uint(f) >> 23);  // f = digits * 2^(e - 150)
  const uint64_t digits = (__float_as_uint(f) & 0x7fffffu) | 0x800000u;
  const uint64_t b = e >= 86 ? digits << (e - 86) : e > 86 - 24 ? digits >> (86 - e) : 0;
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
  uint64_t limit;  // of a wait, in nanoseconds
  int hold;        // the first row's first copy is left out
};

// ------------------------------------------------------------------ the kernel
//
// What bounds it: instructions (42 an element over mixed rows) and the barriers between the steps.
// 256 rows of 150001 bf16 logits: 33 us for the largest alone (floor 11.4), 50 with top_k 50, 83 when every mass is added
// up once, 197 with top_p 0.95 (twice, and the border's search); mixed rows 108 to 111 (bit by bit over a row that is
// read again for every bit: 5095).  One row of 32000: 12.3 to 12.9 us, of which clusters' barriers and the first fetch of
// the code are most.
//
// A cluster of CTAs holds a row in shared memory, read from global memory once, with the largest logit found on the way.
// A rule's border is found by counting: tokens (or their masses) are added up in 704 bins of a sixteenth of an octave of
// mass each; the bin in which the rule's count or mass is reached is split by the logits' bits into up to 704 again until
// one value is left.  All sums are of the masses as integers, exact, so neither the atomics' order nor the cut into CTAs
// matters, nor which of the searches a row takes.

constexpr int kSampleThreads = 512, kSampleWarps = kSampleThreads / 32, kBins = static_cast<int>(kMassPlaces >> 6), kGroup = kBins / kSampleWarps,
              kSegUnits = 64, kSegs = 256;
static_assert(kBins % kSampleWarps == 0 && kGroup % 2 == 0 && kGroup <= 64, "a warp adds up a group");
constexpr int kUses = 10;   // values that CTAs send each other, each at a place of its own
constexpr int kPieces = 4;  // copies of a CTA's part of the row
constexpr int kList = 512;  // tokens that one CTA ranks by comparing all with all

struct SampleShared {
  uint32_t table[kExpSize];
  alignas(16) uint64_t bin[2][kBins];        // of one search step, and of the next; read by twos
  uint64_t groups[2][8][kSampleWarps];       // their sums over kGroup bins, of every CTA
  uint64_t seg[kSegs];
  uint64_t part[2][kSampleWarps];
  uint64_t sent[kUses][8];                   // written by the CTA of that rank
  uint64_t list[kList];                      // key and inverted index of tokens that are ranked one by one
  alignas(16) uint64_t all[kList + 2];       // the cluster's lists as one; read by twos
  uint64_t by_rank[kList], sorted[kList];
  uint64_t before, at;
  uint64_t arrived[kPieces];                 // barriers of the row's pieces
  int border, listed, first, kept, failed;
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
  pdl_wait();
  pdl_trigger();

  // ---- this CTA's tokens [v0, v1), in units that lie in shared memory as they do in global memory; the places of the
  // first and the last unit that are not of the row hold -infinity
  const int per = (vocab + ctas - 1) / ctas, v0 = min(rank * per, vocab), v1 = min(v0 + per, vocab);
  const T* const src = static_cast<const T*>(p.logits) + row * p.row_stride + v0;
  const int phase = static_cast<int>(reinterpret_cast<uintptr_t>(src) / sizeof(T) % E);
  const int units = v1 > v0 ? (phase + v1 - v0 + E - 1) / E : 0, first_index = v0 - phase;
  // the units inside the row are copied in kPieces, and looked at as they arrive
  const int piece = (units + kPieces * kSampleThreads - 1) / (kPieces * kSampleThreads) * kSampleThreads;
  if (tid == 0) {
    for (int i = 0; i < kPieces; ++i) mbar_init(&sh.arrived[i], 1);
    sh.failed = 0;
    fence_mbar_init();
    const uint4* in = reinterpret_cast<const uint4*>(src - phase);
    for (int i = 0; i < kPieces; ++i) {
      const int u0 = max(i * piece, 1), u1 = min((i + 1) * piece, units - 1);
      mbar_arrive_expect_tx(&sh.arrived[i], u0 < u1 ? (u1 - u0) * 16 : 0);
      if (u0 < u1 && (!p.hold || rank + row + i > 0)) bulk_load(data + u0, in + u0, (u1 - u0) * 16, &sh.arrived[i]);
    }
  }
  if (warp == 1 && lane < 2 * E) {  // the first and the last unit
    const int u = lane < E ? 0 : units - 1, i = u * E + lane % E - phase;
    if (u >= 0) data[u].v[lane % E] = i >= 0 && i < v1 - v0 ? src[i] : from_f32<T>(-INFINITY);
  }
  for (int i = tid; i < kExpSize; i += kSampleThreads) sh.table[i] = kExpTable.v[i];
  for (int i = tid; i < 2 * kBins; i += kSampleThreads) sh.bin[0][i] = 0;
  if (tid == 0) sh.first = vocab;
  __syncthreads();
  float most = -INFINITY;
  for (int i = 0; i < kPieces; ++i) {
    if (!mbar_wait_for(&sh.arrived[i], 0, p.limit)) sh.failed = 1;
#pragma unroll 2
    for (int u = i * piece + tid; u < min((i + 1) * piece, units); u += kSampleThreads) {
      const Logits16<T> x = data[u];
#pragma unroll
      for (int e = 0; e < E; ++e) most = fmaxf(most, to_f32(x.v[e]));
    }
  }
  const float most_of_thread = most;
#pragma unroll
  for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(~0u, most, o));
  if (lane == 0) sh.part[0][warp] = __float_as_uint(most);
  cluster_wait();  // every CTA of the cluster runs
  __syncthreads();
  if (tid < ctas) {
    for (int i = 0; i < kSampleWarps; ++i) most = fmaxf(most, __uint_as_float(static_cast<uint32_t>(sh.part[0][i])));
    cluster_store(&sh.sent[0][rank], tid, static_cast<uint64_t>(sh.failed) << 32 | __float_as_uint(most));
  }
  cluster_sync();
  float top = -INFINITY;
  bool failed = false;
  for (int i = 0; i < ctas; ++i) {
    top = fmaxf(top, __uint_as_float(static_cast<uint32_t>(sh.sent[0][i])));
    failed |= sh.sent[0][i] >> 32 != 0;
  }
  const uint32_t top_key = orderable(top + 0.0f);

  const ssd_sampling& h = p.how;
  const float temp = h.temperature_rows ? h.temperature_rows[row] : h.temperature;
  const float top_p = h.top_p_rows ? h.top_p_rows[row] : h.top_p;
  const float min_p = h.min_p_rows ? h.min_p_rows[row] : h.min_p;
  const int top_k = h.top_k_rows ? h.top_k_rows[row] : h.top_k;
  if (top_key <= kKeyNone || failed) {
    if (rank == 0 && tid == 0) {
      p.token[row] = -1;
      if (p.prob) p.prob[row] = failed ? NAN : 0.0f;
    }
    if (failed)  // the copies under way land before the CTA leaves
      for (int i = 0; i < kPieces; ++i) mbar_wait_for(&sh.arrived[i], 0, 100000000ull);
    return;
  }
  const bool one = !(temp >= 0x1p-100f) || top_k == 1 || top_p <= 0.0f || min_p > 1.0f;  // the first-ranked token
  MassOf mass;
  {
    // 1024 log2(e) / T by the remainder of the rounded quotient
    constexpr double kScale = 1024.0 * 1.4426950408889634074;
    constexpr float kHigh = static_cast<float>(kScale), kLow = static_cast<float>(kScale - static_cast<double>(kHigh));
    // Beside an infinite logit no finite one has mass, at any temperature: the largest keeps them all from infinity.
    const float t = one ? 1.0f : isinf(top) ? FLT_MAX : temp;
    mass.c_hi = kHigh / t;
    mass.c_lo = (fmaf(-mass.c_hi, t, kHigh) + kLow) / t;
    mass.origin = fabsf(top * mass.c_hi) < 1048576.0f || isinf(top) ? 0.0f : top;
    mass.top = __float_as_uint(mass.number(top));
  }
  // kept: logits above `cut`, and of those equal to it the tokens up to `last`
  float cut = -FLT_MAX;
  int last = vocab - 1;
  auto kept = [&](float l, int index) { return l >= cut && (l != cut || index <= last); };
  auto mass_of = [&](float l) { return mass(l, sh.table); };

  // what min_p leaves: exp(z - max z) >= min_p in masses
  const uint64_t least = min_p >= 1.0f ? mass_of(top) : min_p > 0.0f ? times_fraction(mass_of(top), min_p, true) : 0;
  auto aim = [&](uint64_t all) -> uint64_t {
    const float u = p.u[row];
    return u >= 1.0f ? all - 1 : u > 0.0f ? times_fraction(all, u, false) : 0;
  };
  auto put = [&](int index, float l, uint64_t all) {
    p.token[row] = index;
    if (!p.prob) return;
    // share / all, by a fp32 reciprocal that one step makes exact to 2^-44
    const uint32_t at = mass.place(l);
    const double share = static_cast<double>(mass.digits(l, at, sh.table)) *
                         __hiloint2double((1023 + 12 - static_cast<int>(at >> kExpBits)) << 20, 0);
    const double a = static_cast<double>(all), r = static_cast<double>(1.0f / static_cast<float>(all));
    p.prob[row] = static_cast<float>(share * fma(fma(-a, r, 1.0), r, r));
  };

  // Inclusive sums over the threads.  `turn` alternates, so that one barrier a sum is enough.
  auto scan = [&](uint64_t v, int turn, uint64_t& all) {
    v = warp_scan(v);
    if (lane == 31) sh.part[turn][warp] = v;
    __syncthreads();
    all = 0;
#pragma unroll
    for (int i = 0; i < kSampleWarps; ++i) {
      if (i == warp) v += all;
      all += sh.part[turn][i];
    }
    return v;
  };

  // The first token in vocabulary order whose running measure (0 of logits below `cut`) exceeds aim(all of it): calls
  // found(index, logit, all) in one thread of the cluster.  measure(l, m, index): of two neighbouring tokens together.
  int uses = 1;
  constexpr int kSeg = kSegUnits * E;
  static_assert(kSeg <= kSampleThreads, "a segment's tokens are looked at by a thread each");
  auto walk = [&](auto measure, auto aim, auto found) {
    const int segs = (units + kSegUnits - 1) / kSegUnits;
    for (int s = warp; s < segs; s += kSampleWarps) {
      uint64_t sum = 0;
#pragma unroll 1
      for (int u = s * kSegUnits + lane; u < min((s + 1) * kSegUnits, units); u += 32) {
        const Logits16<T> x = data[u];
        bool any = false;
#pragma unroll
        for (int e = 0; e < E; ++e) any |= to_f32(x.v[e]) >= cut;
        if (!any) continue;
#pragma unroll
        for (int e = 0; e < E; e += 2) sum += measure(to_f32(x.v[e]), to_f32(x.v[e + 1]), first_index + u * E + e);
      }
      sum = warp_sum(sum);
      if (lane == 0) sh.seg[s] = sum;
    }
    __syncthreads();
    uint64_t mine = tid < segs ? sh.seg[tid] : 0, sum, all = 0, base = 0;
    const uint64_t run = scan(mine, 0, sum);
    if (tid < ctas) cluster_store(&sh.sent[uses][rank], tid, sum);
    cluster_sync();
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      if (i == rank) base = all;
      if (i < ctas) all += sh.sent[uses][i];
    }
    ++uses;
    const uint64_t goal = aim(all);
    if (goal < base || goal >= base + sum) return;
    if (base + run - mine <= goal && goal < base + run) sh.border = tid, sh.before = base + run - mine;
    __syncthreads();
    const int i = sh.border * kSeg + tid, index = first_index + i;
    float l = 0.0f;
    mine = 0;
    if (tid < kSeg && i < units * E) {
      l = to_f32(reinterpret_cast<const T*>(data)[i]);
      mine = measure(l, -INFINITY, index);
    }
    const uint64_t from = sh.before + scan(mine, 1, sum) - mine;
    if (from <= goal && goal < from + mine) found(index, l, all);
  };
  if (one) {
    if (most_of_thread == top)
      for (int u = tid; u < units; u += kSampleThreads)
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (to_f32(data[u].v[e]) == top) atomicMin(&sh.first, first_index + u * E + e);
    __syncthreads();
    if (tid == 0) cluster_store(&sh.sent[1][rank], 0, sh.first);
    cluster_sync();
    if (rank == 0 && tid == 0) {
      int first = sh.first;
      for (int i = 1; i < ctas; ++i) first = min(first, static_cast<int>(sh.sent[1][i]));
      p.token[row] = first;
      if (p.prob) p.prob[row] = 1.0f;
    }
    return;
  }

  // Adds up the cluster's bins of this step, finds the one in which the running measure reaches goal_of(all of it) (1 or
  // more; 0: none) and returns the goal.  masses: the bins hold MassOf::units.  Every CTA gets the others' sums over groups
  // of bins, and reads one group.
  int step = 0;
  auto find_bin = [&](bool masses, auto goal_of) -> uint64_t {
    const int b = step & 1;
    auto value_of = [&](uint64_t v, int bin) { return masses ? v << MassOf::unit_bits(bin) : v; };
    __syncthreads();
    {
      uint64_t v = lane < kGroup ? value_of(sh.bin[b][warp * kGroup + lane], warp * kGroup + lane) : 0;
      if (lane + 32 < kGroup) v += value_of(sh.bin[b][warp * kGroup + lane + 32], warp * kGroup + lane + 32);
      v = warp_sum(v);
      if (lane < ctas) cluster_store(&sh.groups[b][rank][warp], lane, v);
    }
    cluster_sync();
    // the other CTAs have read the bins of the step before
    for (int i = tid; i < kBins; i += kSampleThreads) sh.bin[b ^ 1][i] = 0;
    uint64_t mine = 0;
#pragma unroll
    for (int r = 0; r < 8; ++r)
      if (r < ctas && lane < kSampleWarps) mine += sh.groups[b][r][lane];
    uint64_t run = warp_scan(mine);
    const uint64_t goal = goal_of(__shfl_sync(~0u, run, 31));
    const uint32_t owner = __ballot_sync(~0u, run - mine < goal && goal <= run);
    if (warp == 0 && owner) {
      const int group = __ffs(owner) - 1;
      const uint64_t base = __shfl_sync(~0u, run - mine, group);
      uint64_t x[8], y[8], v = 0, w = 0;  // all of them under way at once
#pragma unroll
      for (int r = 0; r < 8; ++r) {
        x[r] = y[r] = 0;
        if (r < ctas && lane < kGroup / 2) cluster_load2(&sh.bin[b][group * kGroup + 2 * lane], r, x[r], y[r]);
      }
#pragma unroll
      for (int r = 0; r < 8; ++r)
        v += value_of(x[r], group * kGroup + 2 * lane), w += value_of(y[r], group * kGroup + 2 * lane + 1);
      const uint64_t before = base + warp_scan(v + w) - v - w;
      if (before < goal && goal <= before + v + w) {
        const bool in_w = goal > before + v;
        sh.border = group * kGroup + 2 * lane + in_w;
        sh.before = in_w ? before + v : before;
        sh.at = in_w ? w : v;
      }
    }
    __syncthreads();
    ++step;
    return goal;
  };
  // logits that a bin can hold, with two places more at either end than it has (and what rounding takes)
  const float unit = temp * 6.7690154e-4f;  // of a place: T ln(2) / 1024
  auto low_of = [&](int bin) {
    return isinf(top) ? top : fmaxf(__fsub_rd(top, __fmul_ru(unit, 64.0f * bin + 66.1f)), -FLT_MAX);
  };
  auto high_of = [&](int bin) { return isinf(top) ? top : fminf(__fsub_ru(top, __fmul_rd(unit, 64.0f * bin - 2.1f)), top); };
  auto low_half = [&](int bin) { return reinterpret_cast<uint32_t*>(&sh.bin[step & 1][bin]); };

  // Lists the cluster's wanted tokens of logits in [low, high] in sh.all of every CTA, if they are kList at most, and
  // returns how many there are, or -1.
  auto collect = [&](float low, float high, auto wanted) -> int {
    if (tid == 0) sh.listed = 0;
    __syncthreads();
    for (int u = tid; u < units; u += kSampleThreads) {
      const Logits16<T> x = data[u];
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float l = to_f32(x.v[e]);
        if (!(l >= low && l <= high) || !wanted(l, first_index + u * E + e)) continue;
        const int i = atomicAdd(&sh.listed, 1);
        if (i < kList)
          sh.list[i] = static_cast<uint64_t>(orderable(l + 0.0f)) << 32 | ~static_cast<uint32_t>(first_index + u * E + e);
      }
    }
    __syncthreads();
    if (tid < ctas) cluster_store(&sh.sent[uses][rank], tid, sh.listed);
    cluster_sync();
    int n = 0, from = 0, at = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < ctas) {
        const int c = static_cast<int>(sh.sent[uses][i]);
        if (tid >= n && tid < n + c) from = i, at = tid - n;  // entry tid of all is entry `at` of CTA `from`
        n += c;
      }
    ++uses;
    if (n > kList) return -1;
    uint64_t v = 0;  // one past the end as well: two entries are compared at a time
    if (tid < n) asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(cluster_addr(&sh.list[at], from)) : "memory");
    if (tid <= n) sh.all[tid] = v;
    __syncthreads();
    return n;
  };
  // Entry tid / each of the list and its places by rank and by index, from comparing all with all: `each` neighbouring
  // lanes share an entry's comparisons.
  auto rank_list = [&](int n, int each, int& by_rank, int& by_index) -> uint64_t {
    const uint64_t mine = tid / each < n ? sh.all[tid / each] : 0;
    int better = 0, earlier = 0;
#pragma unroll 4
    for (int j = 2 * (tid & (each - 1)); j < n; j += 2 * each) {
      const ulonglong2 v = *reinterpret_cast<const ulonglong2*>(&sh.all[j]);
      better += (v.x > mine) + (v.y > mine);
      earlier += (static_cast<uint32_t>(v.x) > static_cast<uint32_t>(mine)) + (static_cast<uint32_t>(v.y) > static_cast<uint32_t>(mine));
    }
    for (int d = each / 2; d; d >>= 1)
      better += __shfl_xor_sync(~0u, better, d), earlier += __shfl_xor_sync(~0u, earlier, d);
    by_rank = better, by_index = earlier;
    return mine;
  };
  auto share_of = [&](int n) {
    int each = 1;
    while (each < 32 && n * each * 2 <= kSampleThreads) each *= 2;
    return each;
  };

  // Shrinks the kept tokens to the shortest prefix of the ranking whose count or mass reaches goal_of(all of it).
  bool limited = false;
  auto shrink = [&](bool counting, auto goal_of) {
    for (int u = tid; u < units; u += kSampleThreads) {
      const Logits16<T> x = data[u];
      uint32_t v[E], old[E], place[E];
      bool on[E];
#pragma unroll
      for (int e = 0; e < E; e += 2) {
        const float l = to_f32(x.v[e]), m = to_f32(x.v[e + 1]);
        mass.two(l, m, sh.table, place + e, v + e);
        on[e] = place[e] < kMassPlaces && (!limited || kept(l, first_index + u * E + e));
        on[e + 1] = place[e + 1] < kMassPlaces && (!limited || kept(m, first_index + u * E + e + 1));
        v[e] = counting ? 1 : MassOf::units(v[e], place[e]);
        v[e + 1] = counting ? 1 : MassOf::units(v[e + 1], place[e + 1]);
      }
      // low halves, and then what they carry: a 64-bit atomic on shared memory is a loop
#pragma unroll
      for (int e = 0; e < E; ++e) old[e] = on[e] ? atomicAdd(low_half(place[e] >> 6), v[e]) : 0;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (on[e] && old[e] > ~v[e]) atomicAdd(low_half(place[e] >> 6) + 1, 1u);
    }
    uint64_t goal = find_bin(!counting, goal_of);
    if (goal == 0) return;
    goal -= sh.before;
    const int bin = sh.border;
    // within the bin masses are in its units
    const int bits = counting ? 0 : MassOf::unit_bits(bin);
    goal = (goal + (1u << bits) - 1) >> bits;
    auto measure = [&](float l) -> uint64_t {
      const uint32_t at = mass.place(l);
      return counting ? 1u : MassOf::units(mass.digits(l, at, sh.table), at);
    };
    const float low = low_of(bin), high = high_of(bin);
    auto in_bin = [&](float l, int index) { return mass.place(l) >> 6 == static_cast<uint32_t>(bin) && kept(l, index); };
    limited = true;
    // fp32 logits in a bin are few and all different; bf16 ones are many equals of two or three values
    const int n = KS == 0 ? collect(low, high, in_bin) : -1;
    if (n >= 0) {
      const int each = share_of(n);
      int better, earlier;
      const uint64_t mine = rank_list(n, each, better, earlier);
      if (tid / each < n && (tid & (each - 1)) == 0) {
        sh.by_rank[better] = measure(key_value(static_cast<uint32_t>(mine >> 32)));
        sh.sorted[better] = mine;
      }
      __syncthreads();
      const uint64_t v = tid < n ? sh.by_rank[tid] : 0;
      uint64_t all;
      const uint64_t run = scan(v, 0, all);
      if (run - v < goal && goal <= run) sh.at = sh.sorted[tid];
      __syncthreads();
      cut = key_value(static_cast<uint32_t>(sh.at >> 32));
      last = static_cast<int>(~static_cast<uint32_t>(sh.at));
      return;
    }
    // more tokens than the list takes: the bin is split by the logits' keys until one is left
    uint32_t kmin = orderable(low) >> KS, kmax = orderable(high + 0.0f) >> KS;
    for (bool ready = false; !ready;) {
      const uint32_t width = kmax - kmin;  // one less than the keys
      const int shift = width < kBins ? 0 : 32 - __clz(width / kBins);
#pragma unroll 1
      for (int u = tid; u < units; u += kSampleThreads) {
        const Logits16<T> x = data[u];
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float l = to_f32(x.v[e]);
          if (!(l >= low && l <= high)) continue;
          const uint32_t key = orderable(l + 0.0f) >> KS;
          if (key >= kmin && key <= kmax && in_bin(l, first_index + u * E + e))
          {
            const uint32_t v = static_cast<uint32_t>(measure(l));
            uint32_t* const at = low_half((kmax - key) >> shift);
            if (atomicAdd(at, v) > ~v) atomicAdd(at + 1, 1u);
          }
        }
      }
      find_bin(false, [&](uint64_t) { return goal; });
      goal -= sh.before;
      kmax -= static_cast<uint32_t>(sh.border) << shift;
      kmin = max(kmin, kmax - ((1u << shift) - 1));
      ready = shift == 0;
    }
    // kmax is the border's key; its equals fall by index
    const float value = key_value(kmax & (0x80000000u >> KS) ? kmax << KS : kmax << KS | ((1u << KS) - 1));
    const uint64_t m = measure(value), wanted = (goal + m - 1) / m;
    int end = value == cut ? last : vocab - 1;
    if (wanted * m < sh.at) {
      walk([&](float l, float m, int) -> uint64_t { return (l == value) + (m == value); }, [&](uint64_t) { return wanted - 1; },
           [&](int index, float, uint64_t) {
             for (int r = 0; r < ctas; ++r) cluster_store(&sh.sent[uses][0], r, index);
           });
      cluster_sync();
      end = static_cast<int>(sh.sent[uses][0]);
      ++uses;
    }
    cut = value;
    last = end;
  };

  if (top_k > 1 && top_k < vocab) {
    // At least top_k tokens are in or above the bin that the top_k-th of the threads' largest is in; usually few more.
    // The first CTA ranks them, applies the rules to the sorted masses and draws.
    if (top_k <= kList / 2) {
      const uint32_t place = mass.place(most_of_thread);
      if (place < kMassPlaces) atomicAdd(low_half(place >> 6), 1u);
      const uint64_t found = find_bin(false, [&](uint64_t all) -> uint64_t { return all >= static_cast<uint64_t>(top_k) ? top_k : 0; });
      const int n = found ? collect(low_of(sh.border), top, [](float, int) { return true; }) : -1;
      if (n >= 0) {
        cluster_sync();
        if (rank != 0) return;
        const int each = share_of(n), most_kept = min(top_k, n);
        int better, earlier;
        const uint64_t mine = rank_list(n, each, better, earlier);
        const float logit = key_value(static_cast<uint32_t>(mine >> 32));
        const bool lead = tid / each < n && (tid & (each - 1)) == 0;
        const uint64_t w = lead ? mass_of(logit) : 0;
        if (lead) sh.by_rank[better] = w;
        __syncthreads();
        uint64_t v = tid < most_kept ? sh.by_rank[tid] : 0, all;
        uint64_t run = scan(v, 0, all);
        int keep = most_kept;
        if (top_p < 1.0f) {
          const uint64_t goal = max(times_fraction(all, top_p, true), static_cast<uint64_t>(1));
          if (run - v < goal && goal <= run) sh.kept = tid + 1;
          __syncthreads();
          keep = sh.kept;
        }
        if (lead) {
          sh.list[earlier] = better < keep && w >= least ? w : 0;
          sh.sorted[earlier] = mine;
        }
        __syncthreads();
        v = tid < n ? sh.list[tid] : 0;
        run = scan(v, 1, all);
        const uint64_t goal = aim(all);
        if (run - v <= goal && goal < run)
          put(static_cast<int>(~static_cast<uint32_t>(sh.sorted[tid])), key_value(static_cast<uint32_t>(sh.sorted[tid] >> 32)), all);
        return;
      }
    }
    shrink(true, [&](uint64_t all) -> uint64_t { return all > static_cast<uint64_t>(top_k) ? top_k : 0; });
  }
  if (top_p < 1.0f)
    shrink(false, [&](uint64_t all) -> uint64_t { return max(times_fraction(all, top_p, true), static_cast<uint64_t>(1)); });
  walk(
      [&](float l, float m, int index) -> uint64_t {
        uint32_t place[2], w[2];
        mass.two(l, m, sh.table, place, w);
        const uint64_t a = MassOf::value(w[0], place[0]), b = MassOf::value(w[1], place[1]);
        return (kept(l, index) && a >= least ? a : 0) + (kept(m, index + 1) && b >= least ? b : 0);
      },
      aim, put);
}

template <typename T>
ssd_status sample_launch(const SampleParams& p, int rows, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};
  constexpr int kHead = (sizeof(SampleShared) + 15) / 16 * 16, kMost = SSD_SAMPLE_MAX_VOCAB / 8 * 4 + 32;
  if (ssd_status e = op_smem(ssd_sample_kernel<T>, kHead + kMost, ready, "ssd_sample")) return e;
  // CTAs of a row: as many as fill the SMs, a part of 2048 tokens or more each, and of a size that leaves room for two
  // CTAs an SM
  int ctas = 1;
  while (ctas < 8 && ((static_cast<int64_t>(rows) * ctas < 152 && p.vocab / ctas > 4096) ||
                      static_cast<int64_t>(p.vocab) * sizeof(T) / ctas > (113 << 10) - kHead))
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
  const int size = type == SSD_TYPE_FP32 ? 4 : 2;
  const OpRows in{logits, rows, 1, row_stride * size, 0, static_cast<int64_t>(vocab) * size};
  auto row_words = [&](const void* a) { return OpRows{a, 1, 1, 0, 0, static_cast<int64_t>(rows) * 4}; };
  for (const void* y : {static_cast<const void*>(token), static_cast<const void*>(prob)}) {
    if (!y) continue;
    bool shared = op_overlap(row_words(y), in, 1) || (y == token && prob && op_overlap(row_words(y), row_words(prob), 1));
    for (const void* x : {static_cast<const void*>(u), static_cast<const void*>(how->temperature_rows),
                          static_cast<const void*>(how->top_p_rows), static_cast<const void*>(how->min_p_rows),
                          static_cast<const void*>(how->top_k_rows)})
      shared |= x && op_overlap(row_words(y), row_words(x), 1);
    if (shared) return op_fail(SSD_ERR_INVALID_ARG, "ssd_sample: an output overlaps another buffer");
  }
  const OpWait wait = op_wait();
  const SampleParams p{logits, row_stride, vocab, u, *how, token, prob, static_cast<uint64_t>(wait.ns), wait.hold};
  cudaStream_t s = static_cast<cudaStream_t>(cuda_stream);
  return type == SSD_TYPE_FP32 ? sample_launch<float>(p, rows, s) : sample_launch<__nv_bfloat16>(p, rows, s);
}
