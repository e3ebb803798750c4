// Sampling: temperature, top-k, top-p, min-p and the draw by a given random number, one pass of rules per row.
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

struct MassOf {
  float half_top, c_hi, c_lo;  // top / 2; the pair -2048 log2(e) / T

  // The mass as a 32-bit number and the places it is shifted to the right of 2^13 times it (64 or more: nothing).
  __device__ __forceinline__ void parts(float l, const uint32_t* table, uint32_t& w, int& shift) const {
    const float b = -0.5f * l, d = half_top + b, bb = d - half_top;
    const float lo = (half_top - (d - bb)) + (b - bb);  // d + lo = (top - l) / 2 exactly
    const float y = d * c_hi;
    const float e = fmaf(lo, c_hi, fmaf(d, c_lo, fmaf(d, c_hi, -y)));
    const float magic = __fadd_rd(fmaf(d, c_hi, -0.0625f), 12582912.0f);
    const int n = __float_as_int(magic) - 0x4B400000;
    const float f = (y - (magic - 12582912.0f)) + e;
    // 2^32 (2^(f / 1024) - 1) = f a + f^2 a^2 / 2! ..  with a = ln 2 / 1024, times 2^32
    const float q = fmaf(f, fmaf(f, fmaf(f, 0.2220f, 983.9678f), 2907270.0f), 8388608.0f);
    const uint32_t t = table[n & (kExpSize - 1)];
    w = t + __umulhi(t, __float_as_uint(q) - 0x4B000000u);
    shift = y > -65536.0f ? -(n >> kExpBits) : 64;  // also where y is NaN or n has no room
  }
  __device__ __forceinline__ uint64_t operator()(float l, const uint32_t* table) const {
    uint32_t w;
    int s;
    parts(l, table, w, s);
    return s >= 64 ? 0ull : (static_cast<uint64_t>(w) << 13) >> s;
  }
};

__device__ __forceinline__ float key_value(uint32_t key) {  // the inverse of orderable
  return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key);
}
// NaN ranks with -infinity, -0 with 0.
__device__ __forceinline__ uint32_t logit_key(float l) { return l != l ? 0x007fffffu : orderable(l + 0.0f); }
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

constexpr int kSampleThreads = 1024;

// Sum of a value over the CTA, in every thread.
__device__ __forceinline__ uint64_t cta_sum(uint64_t v, uint64_t* part) {
  for (int o = 16; o; o >>= 1) v += __shfl_xor_sync(~0u, v, o);
  __syncthreads();
  if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
  __syncthreads();
  v = 0;
  for (int i = 0; i < kSampleThreads / 32; ++i) v += part[i];
  return v;
}

// One CTA per row.  A rule's border is the largest key whose tokens at or above it reach the rule's count or mass,
// found bit by bit; the last equal tokens are told apart by index, found bit by bit as well.
template <typename T>
__global__ void __launch_bounds__(kSampleThreads) ssd_sample_kernel(const SampleParams p) {
  pdl_wait();
  pdl_trigger();
  __shared__ uint32_t table[kExpSize];
  __shared__ uint64_t part[kSampleThreads / 32];
  const int tid = threadIdx.x, row = blockIdx.x, vocab = p.vocab;
  table[tid] = kExpTable.v[tid];
  const T* logits = static_cast<const T*>(p.logits) + row * p.row_stride;
  auto key_at = [&](int i) { return logit_key(to_f32(logits[i])); };

  // the first-ranked token
  uint64_t best = 0;
  for (int i = tid; i < vocab; i += kSampleThreads) {
    const uint64_t k = static_cast<uint64_t>(key_at(i)) << 32 | (0xffffffffu - i);
    best = k > best ? k : best;
  }
  for (int o = 16; o; o >>= 1) {
    const uint64_t k = __shfl_xor_sync(~0u, best, o);
    best = k > best ? k : best;
  }
  if ((tid & 31) == 0) part[tid >> 5] = best;
  __syncthreads();
  for (int i = 0; i < kSampleThreads / 32; ++i) best = part[i] > best ? part[i] : best;
  const uint32_t top_key = static_cast<uint32_t>(best >> 32);
  const int first = static_cast<int>(0xffffffffu - static_cast<uint32_t>(best));

  const ssd_sampling& h = p.how;
  const float temp = h.temperature_rows ? h.temperature_rows[row] : h.temperature;
  float top_p = h.top_p_rows ? h.top_p_rows[row] : h.top_p;
  const float min_p = h.min_p_rows ? h.min_p_rows[row] : h.min_p;
  const int top_k = h.top_k_rows ? h.top_k_rows[row] : h.top_k;
  if (!(temp >= 0x1p-100f) || top_key <= kKeyNone) {
    if (tid == 0) {
      p.token[row] = top_key <= kKeyNone ? -1 : first;
      if (p.prob) p.prob[row] = top_key <= kKeyNone ? 0.0f : 1.0f;
    }
    return;
  }
  const float top = key_value(top_key);
  MassOf mass;
  {
    const double c = -2048.0 * 1.4426950408889634074 / static_cast<double>(temp);
    mass.half_top = 0.5f * top;
    mass.c_hi = static_cast<float>(c);
    mass.c_lo = static_cast<float>(c - mass.c_hi);
  }
  // where the largest is infinite only its equals have mass
  const uint32_t least = top_key == kKeyInf ? kKeyInf : kKeyNone + 1;
  auto mass_at = [&](int i) -> uint64_t {
    const uint32_t k = key_at(i);
    return k < least ? 0 : top_key == kKeyInf ? 1ull << 44 : mass(to_f32(logits[i]), table);
  };
  // kept: keys above `cut`, and of those equal to it the tokens up to `last`
  uint32_t cut = least;
  int last = vocab - 1;
  auto kept = [&](int i) {
    const uint32_t k = key_at(i);
    return k > cut || (k == cut && i <= last);
  };
  // Shrinks the kept set to the shortest prefix of the ranking whose measure reaches `goal`.
  auto shrink = [&](uint64_t goal, auto measure) {
    uint32_t c = 0;
    for (int bit = 31; bit >= 0; --bit) {
      const uint32_t t = c | 1u << bit;
      uint64_t sum = 0;
      for (int i = tid; i < vocab; i += kSampleThreads)
        if (kept(i) && key_at(i) >= t) sum += measure(i);
      if (cta_sum(sum, part) >= goal) c = t;
    }
    int end = -1;  // the largest index whose equals before it do not reach the goal
    for (int bit = 17; bit >= 0; --bit) {
      const int t = end + (1 << bit);
      uint64_t sum = 0;
      for (int i = tid; i < vocab; i += kSampleThreads)
        if (kept(i) && (key_at(i) > c || (key_at(i) == c && i <= t))) sum += measure(i);
      if (cta_sum(sum, part) < goal) end = t;
    }
    last = end + 1;
    cut = c;
  };
  if (top_k >= 1 && top_k < vocab) {
    uint64_t n = 0;
    for (int i = tid; i < vocab; i += kSampleThreads) n += kept(i);
    if (cta_sum(n, part) > static_cast<uint64_t>(top_k)) shrink(top_k, [](int) { return 1ull; });
  }
  if (top_p < 1.0f) {
    uint64_t all = 0;
    for (int i = tid; i < vocab; i += kSampleThreads) all += kept(i) ? mass_at(i) : 0;
    all = cta_sum(all, part);
    const uint64_t goal = top_p > 0.0f ? times_fraction(all, top_p, true) : 0;
    shrink(goal > 1 ? goal : 1, mass_at);
  }
  if (min_p > 1.0f) {
    cut = top_key, last = first;
  } else if (min_p > 0.0f && top_key != kKeyInf) {
    const double border = static_cast<double>(top) + static_cast<double>(temp) * log(static_cast<double>(min_p));
    const float b = __double2float_ru(border < top ? border : top);
    const uint32_t k = logit_key(b);
    if (k > cut) cut = k, last = vocab - 1;
  }
  // the draw: threads take neighbouring stretches of the vocabulary
  const int per = (vocab + kSampleThreads - 1) / kSampleThreads, from = min(tid * per, vocab), to = min(from + per, vocab);
  uint64_t mine = 0;
  for (int i = from; i < to; ++i) mine += kept(i) ? mass_at(i) : 0;
  uint64_t run = mine;
  for (int o = 1; o < 32; o <<= 1) {
    const uint64_t v = __shfl_up_sync(~0u, run, o);
    if ((tid & 31) >= o) run += v;
  }
  __syncthreads();
  if ((tid & 31) == 31) part[tid >> 5] = run;
  __syncthreads();
  uint64_t total = 0;
  for (int i = 0; i < kSampleThreads / 32; ++i) {
    if (i == tid >> 5) run += total;
    total += part[i];
  }
  const float u = p.u[row];
  const uint64_t aim = u >= 1.0f ? total - 1 : u > 0.0f ? times_fraction(total, u, false) : 0;
  if (run > aim && run - mine <= aim) {
    run -= mine;
    for (int i = from; i < to; ++i) {
      const uint64_t w = kept(i) ? mass_at(i) : 0;
      run += w;
      if (run <= aim) continue;
      p.token[row] = i;
      if (p.prob) {
        double share = 0x1p44;
        if (top_key != kKeyInf) {
          uint32_t v;
          int s;
          mass.parts(to_f32(logits[i]), table, v, s);
          share = ldexp(static_cast<double>(v), 13 - s);
        }
        p.prob[row] = static_cast<float>(share / static_cast<double>(total));
      }
      break;
    }
  }
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
  return type == SSD_TYPE_FP32
             ? op_launch("ssd_sample", ssd_sample_kernel<float>, dim3(rows), kSampleThreads, 0, s, p)
             : op_launch("ssd_sample", ssd_sample_kernel<__nv_bfloat16>, dim3(rows), kSampleThreads, 0, s, p);
}
