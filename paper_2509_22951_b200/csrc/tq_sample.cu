// One token for each row of logits (tq_sample): temperature, top-k, top-p, min-p, and the inverse of the distribution
// function at a given uniform number.
//
// Exact sums.  Every decision is a comparison of sums of weights w = 2^t, t = (x - max) log2(e) / temperature, with a bound: a
// weight is therefore an integer W = round(2^45 w), and sums of up to 2^18 of them are exact in 64 bits whatever their
// order, so that neither the split of a row nor the order of atomics can change a token.  With A a multiple of 1/32 next to max log2(e) / temperature,
// one fused multiply-add rounds t to 1/32 and another, which takes that from the exact product again, leaves the rest to 2^-31: the first is a
// place in a table of 2^(i/32) (a bank of shared memory for each entry) and an octave, the second goes into a polynomial: 26 bits and more in some
// 25 instructions, none of them a conversion; W is then a whole number (within 2^-26 of itself and half a unit).  W below 2^21 (t < -24) is the fp32
// exponential of an fp32 exponent: within five units (its three roundings, and c_low left out: 2^-20 of t each at most; ex2's 2^-22; a rounding).
//
// Order.  Tokens fall by (x, lower index first): as one integer, the logit's bits made to rise with it above the index turned
// round.  What is kept is all that is not below a border in that order, so every filter is a search for its border.
//
// A row is read once: a cluster of up to eight CTAs holds it in shared memory and speaks through distributed shared memory.  Then
//   top-k (up to 1024): the k-th largest of the threads' own maxima is a bound of the k-th logit that few others pass: those go to one CTA,
//          which does the rest: up to 128 tokens by comparing each with each, more by sums over parts of them;
//   top-p alone: a histogram of the weights over 32 bins an octave (exact: two integers a bin, as many atomics; one that returns, with a carry
//          now and then, takes as long, a 64-bit one longer) finds the bin of the border.  Where its sum is that of one token that is all;
//          else one CTA gets the bin's tokens and finds the one with which the sum is reached: over 128 of them by a finer histogram of
//          theirs, then each with each.  What is kept is in the CTAs' bins up to there: only the one that has the drawn token adds it up again;
//   neither, or min-p: the border is known; every CTA adds up what it keeps.
// Where so many logits are alike that a list does not hold them (2048), and for larger k, the border is found by bisection of the order.
//
// Bound: the bytes (a logit is read once) only for one row in 512; instructions otherwise, 25 to 60 of them a logit, issued in 55 % of the cycles
// (shared memory's data path 37 % busy), and for few rows the eight barriers of the cluster, 1500 to 2500 cycles each with what they wait for.
// One B200, 128256 logits in fp32, us: one row top-k 8.7, top-p 18.9, none 10.4; 64 rows with settings of all kinds 41; 512 rows greedy 99 (their
// bytes: 40), top-k 165, none 159 - 225, top-p 0.9 269 (peaked) - 450 (flat).
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "tq_attn_sm100.cuh"
#include "tq_internal.h"
#include "tq_ops_common.cuh"

namespace {

using namespace tq_ops;

constexpr uint32_t kThreads = 512, kWarps = kThreads / 32;
constexpr uint32_t kMaxCluster = 8;
constexpr uint32_t kIndexBits = 18;
static_assert((1u << kIndexBits) == TQ_SAMPLE_MAX_VOCAB, "a token's index fits its place in the order");
constexpr uint32_t kIndexMask = (1u << kIndexBits) - 1u;
constexpr int kOne = 45;      // W of the largest logit is 2^45
constexpr int kOctaves = 24;  // of the histogram, and of the weights that are computed to 26 bits; rounded to whole units, the least of them keep 22
constexpr int kTopPlace = 1;  // place of the largest logit at most (a is off by up to 1/64 and a little)
constexpr uint32_t kBins = kOctaves * 32u + kTopPlace + 1u;  // a place each
constexpr uint32_t kList = 2048;   // tokens that one CTA sorts
constexpr uint32_t kListK = 1024;  // largest k of the list: the threads' maxima bound it well up to a quarter of their number
constexpr uint32_t kKBins = 256;   // of the threads' maxima
constexpr uint32_t kSub = 256;     // parts of the bin with the border
constexpr uint32_t kParts = 768;   // of the list
constexpr uint32_t kNear = 128;    // tokens that are compared each with each

// 2^(i / 32) with 29 bits behind the point
struct Powers {
  uint32_t v[32];
};
constexpr Powers powers() {
  Powers p{};
  for (int i = 0; i < 32; ++i) {
    const double y = i * (0.69314718055994530942 / 32.0);
    double term = 1.0, sum = 1.0;
    for (int k = 1; k < 32; ++k) {
      term *= y / k;
      sum += term;
    }
    p.v[i] = (uint32_t)(sum * 536870912.0 + 0.5);
  }
  return p;
}
__constant__ Powers kPowers = powers();

struct SampleParams {
  const void* logits;
  int64_t row_stride;
  const float* uniform;
  const float* temperature;
  const int32_t* top_k;
  const float* top_p;
  const float* min_p;
  int32_t* token;
  float* logprob;
  uint32_t vocab, slice;  // slice: logits of a CTA
  uint32_t vectors;       // rows may be read 16 bytes at a time
};

struct Shared {
  uint64_t slots[2][kMaxCluster * kWarps];  // what the cluster's warps tell one another; two sets, used in turn
  uint64_t told[2];                         // by one CTA to all
  uint64_t found[2];                        // the warp whose piece has the token, and what is before it
  uint64_t warps[kWarps];                   // within a CTA
  uint32_t powers[32];                      // 2^(i / 32) with 29 bits behind the point
  uint32_t listed;                          // tokens in the list (of the first CTA)
  uint32_t near;                            // entries of `close`
  struct {
    uint32_t hi[kSub], lo[kSub];
  } sub;                                    // as bins, of parts of one bin
  uint64_t close[kNear], close_w[kNear];    // tokens next to the border, and their weights
  union {
    struct {
      uint32_t hi[kBins], lo[kBins];  // sums of the upper and lower 15 bits of the values of a bin
    } bins;
    uint32_t k_bins[kKBins];
    unsigned long long part[kParts];        // sums of parts of the list
  };
  uint64_t list[kList];
};
constexpr uint32_t kHead = (sizeof(Shared) + 15u) / 16u * 16u;  // the row's slice lies behind it

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
  uint32_t r;
  asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return r;
}
// The cluster's barriers in the form that whole warps execute together; lanes that have gone separate ways before come together first.
__device__ __forceinline__ void cluster_arrive() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_sync() {
  cluster_arrive();
  cluster_wait();
}
__device__ __forceinline__ uint32_t at_rank(const void* ptr, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tq_sm100::smem_u32(ptr)), "r"(rank));
  return a;
}
__device__ __forceinline__ void store_remote(const uint64_t* ptr, uint32_t rank, uint64_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at_rank(ptr, rank)), "l"(v) : "memory");
}
// (not volatile: several are asked for together; the cluster's barriers order them)
__device__ __forceinline__ uint32_t load_remote(const uint32_t* ptr, uint32_t rank) {
  uint32_t v;
  asm("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at_rank(ptr, rank)) : "memory");
  return v;
}
__device__ __forceinline__ uint32_t add_remote(uint32_t* ptr, uint32_t rank, uint32_t v) {
  uint32_t old;
  asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(at_rank(ptr, rank)), "r"(v) : "memory");
  return old;
}

// Bits that rise with the number (no NaN, no -0).
__device__ __forceinline__ uint32_t rising(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_rising(uint32_t r) { return __uint_as_float(r ^ (r >> 31 ? 0x80000000u : 0xFFFFFFFFu)); }
__device__ __forceinline__ uint64_t order_of(float x, uint32_t index) { return ((uint64_t)rising(x) << kIndexBits) | (kIndexMask - index); }
__device__ __forceinline__ uint32_t index_of(uint64_t order) { return kIndexMask - (uint32_t)(order & kIndexMask); }
__device__ __forceinline__ float logit_of(uint64_t order) { return from_rising((uint32_t)(order >> kIndexBits)); }

// Sums over a warp, in every lane, below 2^64: three pieces that 32 lanes cannot carry out of 32 bits.
__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
  const uint32_t a = __reduce_add_sync(kFull, (uint32_t)v & 0x3FFFFFu), b = __reduce_add_sync(kFull, (uint32_t)(v >> 22) & 0x3FFFFFu),
                 c = __reduce_add_sync(kFull, (uint32_t)(v >> 44));
  return (uint64_t)a + ((uint64_t)b << 22) + ((uint64_t)c << 44);
}
__device__ __forceinline__ uint64_t warp_upto(uint64_t v, uint32_t lane) {  // of this lane and those before it
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint64_t o = __shfl_up_sync(kFull, v, d);
    if (lane >= (uint32_t)d) v += o;
  }
  return v;
}
__device__ __forceinline__ uint32_t warp_upto(uint32_t v, uint32_t lane) {
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t o = __shfl_up_sync(kFull, v, d);
    if (lane >= (uint32_t)d) v += o;
  }
  return v;
}

// Two fp32 numbers whose sum is meant, the second small against the first.
struct Pair {
  float hi, lo;
};
__device__ __forceinline__ Pair exact_sum(float a, float b) {  // Knuth's sum without loss
  const float s = a + b, t = s - a;
  return Pair{s, (a - (s - t)) + (b - t)};
}
constexpr float kLn2 = 0.693147182464599609375f, kLn2Low = -1.904654323148236e-09f;      // ln 2
constexpr float kLog2e = 1.44269502162933349609375f, kLog2eLow = 1.92596303178237e-08f;  // 1 / ln 2

// log2(m 2^(k - 29)), 2^29 <= m < 2^30, to 2^-29: the table's entry below m, and a series for the rest.
__device__ __forceinline__ Pair log2_of(uint32_t m, int k, const uint32_t* powers) {
  int i = min(max((int)((__log2f((float)m) - 29.f) * 32.f), 0), 31);
  if (powers[i] > m && i > 0) --i;
  const float z = (float)(int32_t)(m - powers[i]) / (float)powers[i];  // 0 .. 0.022
  const float y = z * (1.f + z * (-0.5f + z * (0.33333334f + z * (-0.25f + z * (0.2f - z * 0.16666667f)))));
  return Pair{(float)k + (float)i * 0.03125f, fmaf(y, kLog2e, y * kLog2eLow)};
}
__device__ __forceinline__ Pair log2_of(uint64_t v, int one, const uint32_t* powers) {  // log2(v 2^-one)
  const int top = 63 - __clzll((long long)v);
  return log2_of(top >= 29 ? (uint32_t)(v >> (top - 29)) : (uint32_t)v << (29 - top), top - one, powers);
}

// W = value << max(0, 16 + octave) with a place = 32 t, rounded, in octave place >> 5.
struct Weights {
  float top;          // largest logit, finite
  float c, c_low;     // log2(e) / temperature
  float a, a_low;     // top * log2(e) / temperature: a multiple of 1/32, and the rest
  float to_small;     // what base() lacks to 45 + t
  bool plain;         // a is small enough for the short form
  const uint32_t* powers;

  __device__ __forceinline__ void set(float top_, float temperature, const uint32_t* powers_) {
    top = top_;
    powers = powers_;
    const float T = fminf(fmaxf(temperature, 7.52316385e-37f), 1.26765060e30f);  // 2^-120 .. 2^100: the quotient stays finite, and is not 0
    c = kLog2e / T;
    c_low = (fmaf(-c, T, kLog2e) + kLog2eLow) / T;
    const float full = top * c;
    plain = fabsf(full) < 65536.f;
    a = plain ? rintf(full * 32.f) * 0.03125f : 0.f;
    a_low = fmaf(top, c, -a) + top * c_low;
    to_small = (float)kOne - (plain ? a_low : 0.f);
  }
  // t in fp32, to a constant below 1/32; -inf where x is
  __device__ __forceinline__ float base(float x) const { return plain ? fmaf(x, c, -a) : (x - top) * c; }
  __device__ __forceinline__ Pair both(float x) const {
    const Pair d = exact_sum(x, -top);
    const float t = d.hi * c;
    return Pair{t, fmaf(d.lo, c, fmaf(d.hi, c_low, fmaf(d.hi, c, -t)))};
  }
  // A sum s of t with 1.5 * 2^18 is rounded to 1/32.  Below the histogram's octaves a weight is small, and that is told from s itself: below 0
  // (t < -393216: a mask of -65504 at a temperature of 0.2) its bits fall with t, and a place taken from them could be any.
  static constexpr float kRound = 393216.0f, kLeastSum = kRound - (float)kOctaves;
  __device__ __forceinline__ static bool is_small(float s) { return s < kLeastSum; }
  // 32 t rounded, of the sum of a weight that is not small.
  __device__ __forceinline__ static int place_in(float s) { return (int)(__float_as_uint(s) - 0x48C00000u); }
  // 2^t = 2^(place / 32) (1 + q 2^-26), of s = base(x) + kRound.
  static constexpr float kA2 = 0.24022651f, kA3 = 0.055504109f, kA4 = 0.0096181291f;  // (ln 2)^k / k!
  static constexpr float kQUnit = 67108864.0f, kQRound = 12582912.0f;                 // 2^26, 1.5 * 2^23
  static constexpr int kQBits = 0x4B400000;                                           // of kQRound
  __device__ __forceinline__ int fine(float x, float s) const {
    float r;
    if (plain) {
      const float k = kRound - a;
      r = fmaf(x, c, k - s) + fmaf(x, c_low, -a_low);
    } else {
      const Pair t = both(x);
      r = (t.hi - (s - kRound)) + t.lo;
    }
    const float q = r * fmaf(r, fmaf(r, fmaf(r, kA4, kA3), kA2), kLn2);
    return __float_as_int(fmaf(q, kQUnit, kQRound)) - kQBits;  // q to whole units of 2^-26, |q| < 0.031
  }
  // The value of a place and its q.
  __device__ __forceinline__ uint32_t value(int place, int q) const {
    const uint32_t base = powers[place & 31];
    const uint32_t v = base + (uint32_t)__mulhi((int)base, q * 64), down = (uint32_t)max(-16 - (place >> 5), 0);
    return (v + ((1u << down) >> 1)) >> down;
  }
  __device__ __forceinline__ static int shift(int place) { return max(0, 16 + (place >> 5)); }
  // Octaves below the histogram's; 0 for -inf.
  __device__ __forceinline__ uint32_t small(float base) const {
    float w;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(base + to_small));
    return __float_as_uint(w + 8388608.0f) - 0x4B000000u;  // rounded
  }
  __device__ __forceinline__ uint64_t operator()(float x) const {
    const float t = base(x), s = t + kRound;
    if (is_small(s)) return small(t);
    const int place = place_in(s);
    return (uint64_t)value(place, fine(x, s)) << shift(place);
  }
  // Four at once, for a whole warp: the chains of fine() side by side, or none of them where all weights are small.  use(j, is fine, place, q)
  // for each, or with its weight in q's place where that is small.
  template <class Use>
  __device__ __forceinline__ void four(const float (&x)[4], Use use) const {
    float t[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) t[j] = base(x[j]);
    if (!__any_sync(kFull, !is_small(fmaxf(fmaxf(t[0], t[1]), fmaxf(t[2], t[3])) + kRound))) {
#pragma unroll
      for (int j = 0; j < 4; ++j) use(j, false, 0, (int)small(t[j]));
      return;
    }
    int q[4];  // (of a small one it is not used)
    float sums[4];
    if (plain) {  // the operations of fine(), two weights to an instruction
      using namespace tq_attn;
      const float k = kRound - a;
      const uint64_t c2 = pair(c, c), l2 = pair(c_low, c_low), one = pair(-1.f, -1.f);
#pragma unroll
      for (int j = 0; j < 4; j += 2) {
        const uint64_t y = pair(x[j], x[j + 1]), s = add2(pair(t[j], t[j + 1]), pair(kRound, kRound));
        const uint64_t r = add2(fma2(y, c2, fma2(s, one, pair(k, k))), fma2(y, l2, pair(-a_low, -a_low)));
        const uint64_t h = fma2(r, fma2(r, fma2(r, pair(kA4, kA4), pair(kA3, kA3)), pair(kA2, kA2)), pair(kLn2, kLn2));
        float u, v;
        unpair(fma2(fma2(r, h, pair(-0.f, -0.f)), pair(kQUnit, kQUnit), pair(kQRound, kQRound)), u, v);
        q[j] = __float_as_int(u) - kQBits, q[j + 1] = __float_as_int(v) - kQBits;
        unpair(s, sums[j], sums[j + 1]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        sums[j] = t[j] + kRound;
        q[j] = fine(x[j], sums[j]);
      }
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool low = is_small(sums[j]);
      use(j, !low, place_in(sums[j]), low ? (int)small(t[j]) : q[j]);
    }
  }
};
// A weight in 32 bits, in the place of its logit: the place turned round, and q; or, with the last place, the weight itself where it is small.
constexpr uint32_t kSmallPlace = 1023u;
__device__ __forceinline__ uint32_t code_of(bool fine, int place, int q) { return (fine ? (uint32_t)(kTopPlace - place) : kSmallPlace) << 22 | ((uint32_t)q & 0x3FFFFFu); }

// floor(f * v) for 0 <= f < 1, v < 2^64, and whether there is a remainder.
__device__ __forceinline__ uint64_t times(float f, uint64_t v, bool& more) {
  const uint32_t b = __float_as_uint(f), e = b >> 23, m = e ? (b & 0x7FFFFFu) | 0x800000u : b & 0x7FFFFFu;
  const int s = 150 - (int)(e ? e : 1u);  // f = m 2^-s, s >= 24
  const uint64_t hi = __umul64hi(v, (uint64_t)m), lo = v * (uint64_t)m;
  if (s >= 64) {
    const int d = s - 64;
    more = lo != 0ull || (d < 64 ? (hi & ((1ull << d) - 1ull)) != 0ull : hi != 0ull);
    return d < 64 ? hi >> d : 0ull;
  }
  more = (lo & ((1ull << s) - 1ull)) != 0ull;
  return (hi << (64 - s)) | (lo >> s);
}
// The least integer not below f * v: a sum of weights is less than f * v exactly if it is less than this.
__device__ __forceinline__ uint64_t bound_of(float f, uint64_t v) {
  if (!(f > 0.f)) return 0ull;
  bool more;
  const uint64_t r = times(f, v, more);
  return r + (more ? 1ull : 0ull);
}

// Sorts list[0 .. n), n <= kList, from the largest down: by every entry's rank where there are few, else bitonic.
__device__ void sort_list(uint64_t* list, uint32_t n, uint32_t tid) {
  if (n <= kThreads / 2u) {
    const uint32_t each = n <= kThreads / 4u ? 4u : 2u, j = tid / each;  // threads to an entry
    const uint64_t mine = j < n ? list[j] : ~0ull;
    uint32_t rank = 0;
#pragma unroll 4
    for (uint32_t i = tid % each; i < n; i += each) rank += list[i] > mine ? 1u : 0u;
    rank += __shfl_xor_sync(kFull, rank, 1);
    if (each == 4u) rank += __shfl_xor_sync(kFull, rank, 2);
    __syncthreads();
    if (j < n && tid % each == 0u) list[rank] = mine;
    __syncthreads();
    return;
  }
  uint32_t size = 512;
  while (size < n) size *= 2u;
  for (uint32_t i = n + tid; i < size; i += kThreads) list[i] = 0ull;
  __syncthreads();
  for (uint32_t k = 2; k <= size; k *= 2u) {
    for (uint32_t j = k / 2u; j > 0; j /= 2u) {
      for (uint32_t i = tid; i < size / 2u; i += kThreads) {
        const uint32_t a = 2u * i - (i & (j - 1u)), b = a + j;
        const uint64_t x = list[a], y = list[b];
        if ((x < y) == ((a & k) == 0u)) {
          list[a] = y;
          list[b] = x;
        }
      }
      __syncthreads();
    }
  }
}

// What the drawn number asks for, below the total.
__device__ __forceinline__ uint64_t target(float u, uint64_t total) {
  if (!(u < 1.f)) return u >= 1.f ? total - 1u : 0ull;
  bool more;
  return u > 0.f ? times(u, total, more) : 0ull;
}
// Sums over the threads of a CTA, and what is of the threads before.
__device__ __forceinline__ uint64_t scan_cta(Shared& sh, uint64_t sum, uint64_t& total) {
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
  const uint64_t upto = warp_upto(sum, lane);
  __syncthreads();
  if (lane == 31) sh.warps[warp] = upto;
  __syncthreads();
  const uint64_t w = lane < kWarps ? sh.warps[lane] : 0ull;
  total = warp_sum(w);
  return warp_sum(lane < warp ? w : 0ull) + upto - sum;
}
// The token among the list's m entries: the last of top-k, the last of top-p, then the one that the drawn number asks for (by sorting twice, 1200
// entries take 20 us longer).  Each is the entry with which a sum reaches a bound, found by the sums of kParts parts and then each with each of the
// part that has it; ~0 where those are more than kNear.  What is summed: 0: numbers, from the largest logit down; 1: weights of those that
// are left, likewise; 2: these in the order of the vocabulary.  told[1] is the sum of what is kept.  (As a call it costs the other ways up to 8 %,
// inlined 2 to 4.)
__device__ __forceinline__ uint64_t token_of_list(Shared& sh, const Weights weight, uint32_t m, uint32_t k, float top_p, uint64_t keep, float u, float fall,
                                               uint32_t vocab) {
  const uint32_t tid = threadIdx.x;
  uint64_t edge = 0;
#pragma unroll 1
  for (uint32_t what = 0; what < 3u; ++what) {
    if (what == 0u ? k >= m : what == 1u && !(top_p < 1.f)) continue;
    if (what == 2u) edge = max(edge, keep);
    const float scale = what == 2u ? (float)kParts / (float)vocab : fall;
    auto measure = [&](uint64_t e) { return what == 0u ? 1ull : e >= edge ? weight(logit_of(e)) : 0ull; };
    auto part = [&](uint64_t e) { return (uint32_t)fminf((what == 2u ? (float)index_of(e) : weight.top - logit_of(e)) * scale, (float)(kParts - 1u)); };
    auto key = [&](uint64_t e) { return what == 2u ? e & kIndexMask : e; };  // falls along the order
    for (uint32_t i = tid; i < kParts; i += kThreads) sh.part[i] = 0ull;
    if (tid == 0) sh.near = 0u;
    __syncthreads();
    for (uint32_t i = tid; i < m; i += kThreads) {
      const uint64_t entry = sh.list[i], w = measure(entry);
      if (w != 0ull) atomicAdd(&sh.part[part(entry)], (unsigned long long)w);
    }
    __syncthreads();
    uint64_t mass[2], total;
#pragma unroll
    for (uint32_t z = 0; z < 2u; ++z) mass[z] = 2u * tid + z < kParts ? sh.part[2u * tid + z] : 0ull;
    uint64_t prev = scan_cta(sh, mass[0] + mass[1], total);
    const uint64_t bound = what == 0u ? (uint64_t)k : what == 1u ? bound_of(top_p, total) : target(u, total) + 1ull;
#pragma unroll
    for (uint32_t z = 0; z < 2u; ++z) {
      if (prev < bound && prev + mass[z] >= bound) {
        sh.told[0] = 2u * tid + z;
        sh.told[1] = prev;
      }
      prev += mass[z];
    }
    __syncthreads();
    const uint32_t chosen = (uint32_t)sh.told[0];
    const uint64_t ahead = sh.told[1];
    for (uint32_t i = tid; i < m; i += kThreads) {
      const uint64_t entry = sh.list[i];
      if (part(entry) != chosen) continue;
      const uint64_t w = measure(entry);
      if (w == 0ull) continue;
      const uint32_t at = atomicAdd(&sh.near, 1u);
      if (at >= kNear) continue;
      sh.close[at] = entry;
      sh.close_w[at] = w;
    }
    __syncthreads();
    const uint32_t near = sh.near, j = tid / 4u;
    if (near > kNear) return ~0ull;
    const uint64_t entry = j < near ? sh.close[j] : 0ull, mine = key(entry);
    uint64_t at = 0;
    for (uint32_t i = tid % 4u; i < near; i += 4u) at += key(sh.close[i]) > mine ? sh.close_w[i] : 0ull;
    at += __shfl_xor_sync(kFull, at, 1);
    at += __shfl_xor_sync(kFull, at, 2);
    at += ahead;
    if (j < near && tid % 4u == 0u && at < bound && at + sh.close_w[j] >= bound) sh.told[0] = entry;
    if (tid == 0) sh.told[1] = total;
    __syncthreads();
    edge = sh.told[0];
  }
  return edge;
}

template <int TYPE>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  float* const xs = reinterpret_cast<float*>(smem + kHead);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u, rank = cluster_rank(), ctas = cluster_size();
  const uint32_t row = blockIdx.x / ctas, from = min(rank * p.slice, p.vocab), n = min(p.slice, p.vocab - from);
  if (tid < 32) sh.powers[tid] = kPowers.v[tid];
  if (tid == 0) {
    sh.listed = sh.near = 0u;
    sh.told[0] = sh.found[0] = ~0ull;
  }
  cluster_arrive();
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const float temperature = p.temperature ? p.temperature[row] : 1.f;
  const int32_t k_given = p.top_k ? p.top_k[row] : 0;
  const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
  const float u = p.uniform[row];

  uint32_t turn = 0;
  // Tells what every warp has (the same in its lanes) to the whole cluster; a lane then has the entries of four warps, in the order of the vocabulary.
  auto tell = [&](uint64_t v, uint64_t (&e)[4]) {
    if (lane < ctas) store_remote(&sh.slots[turn][rank * kWarps + warp], lane, v);
    cluster_sync();
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) e[i] = lane * 4u + i < ctas * kWarps ? sh.slots[turn][lane * 4u + i] : 0ull;
    turn ^= 1u;
  };
  // The sum over the cluster, and what is of the warps before this one.
  auto all = [&](uint64_t mine, uint64_t& prev) {
    uint64_t e[4], b = 0;
    tell(warp_sum(mine), e);
    const uint32_t at = rank * kWarps + warp;
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) b += lane * 4u + i < at ? e[i] : 0ull;
    prev = warp_sum(b);
    return warp_sum(e[0] + e[1] + e[2] + e[3]);
  };

  // The sum over the cluster, and what is of the CTAs before this one and of this.
  auto all_of_ctas = [&](uint64_t mine, uint64_t& prev, uint64_t& own) {
    uint64_t e[4], b = 0, o = 0;
    tell(warp_sum(mine), e);
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) {
      const uint32_t of = (lane * 4u + i) / kWarps;
      b += of < rank ? e[i] : 0ull;
      o += of == rank ? e[i] : 0ull;
    }
    prev = warp_sum(b);
    own = warp_sum(o);
    return warp_sum(e[0] + e[1] + e[2] + e[3]);
  };
  // The sums over the cluster of two numbers, and what is of the warps before this one.  Both sets of slots at once: the cluster comes together before and after it.
  auto all_of_two = [&](uint64_t mine, uint64_t other, uint64_t& prev, uint64_t& sum_of_other) {
    const uint64_t a = warp_sum(mine), b = warp_sum(other);
    if (lane < ctas) {
      store_remote(&sh.slots[0][rank * kWarps + warp], lane, a);
      store_remote(&sh.slots[1][rank * kWarps + warp], lane, b);
    }
    cluster_sync();
    const uint32_t at = rank * kWarps + warp;
    uint64_t sum = 0, others = 0, ahead = 0;
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) {
      const uint32_t j = lane * 4u + i;
      const uint64_t e = j < ctas * kWarps ? sh.slots[0][j] : 0ull;
      others += j < ctas * kWarps ? sh.slots[1][j] : 0ull;
      sum += e;
      ahead += j < at ? e : 0ull;
    }
    prev = warp_sum(ahead);
    sum_of_other = warp_sum(others);
    return warp_sum(sum);
  };

  // ---- the row; its first token in falling order; the largest logit of every thread ------------------------
  float mine = -INFINITY;
  auto take = [&](float x) {
    x = fmaxf(x + 0.f, -INFINITY);  // -0 is 0, and what is not a number -inf
    mine = fmaxf(mine, x);
    return x;
  };
  const size_t row_at = (size_t)((int64_t)row * p.row_stride) + from;
  if (p.vectors) {
    constexpr uint32_t kPer = TYPE == TQ_TYPE_F32 ? 4 : 8;
    const uint32_t whole = n / kPer;
    const uint8_t* const src = (const uint8_t*)p.logits + row_at * (TYPE == TQ_TYPE_F32 ? 4 : 2);
#pragma unroll 1
    for (uint32_t i0 = tid; i0 < whole; i0 += 8u * kThreads) {
      uint4 v[8];
#pragma unroll
      for (uint32_t k = 0; k < 8u; ++k)
        if (i0 + k * kThreads < whole) v[k] = load_once(src + (size_t)(i0 + k * kThreads) * 16u);
#pragma unroll
      for (uint32_t k = 0; k < 8u; ++k) {
        const uint32_t i = i0 + k * kThreads;
        if (i >= whole) break;
        const uint32_t at = i * kPer;
        if constexpr (TYPE == TQ_TYPE_F32) {
          float4 y;
          y.x = take(__uint_as_float(v[k].x));
          y.y = take(__uint_as_float(v[k].y));
          y.z = take(__uint_as_float(v[k].z));
          y.w = take(__uint_as_float(v[k].w));
          *reinterpret_cast<float4*>(xs + at) = y;
        } else {
          float4 y, z;
          y.x = take(bf16_lo(v[k].x));
          y.y = take(bf16_hi(v[k].x));
          y.z = take(bf16_lo(v[k].y));
          y.w = take(bf16_hi(v[k].y));
          z.x = take(bf16_lo(v[k].z));
          z.y = take(bf16_hi(v[k].z));
          z.z = take(bf16_lo(v[k].w));
          z.w = take(bf16_hi(v[k].w));
          *reinterpret_cast<float4*>(xs + at) = y;
          *reinterpret_cast<float4*>(xs + at + 4u) = z;
        }
      }
    }
    for (uint32_t i = whole * kPer + tid; i < n; i += kThreads) xs[i] = take(load1<TYPE>(p.logits, row_at + i));
  } else {
    for (uint32_t i = tid; i < n; i += kThreads) xs[i] = take(load1<TYPE>(p.logits, row_at + i));
  }
  if (tid < 4u && n + tid < (n + 3u) / 4u * 4u) xs[n + tid] = -INFINITY;  // four are read together
  if (k_given > 0) {
    for (uint32_t i = tid; i < kKBins; i += kThreads) sh.k_bins[i] = 0u;
  }
  if (top_p < 1.f) {
    for (uint32_t i = tid; i < kBins; i += kThreads) sh.bins.hi[i] = sh.bins.lo[i] = 0u;
    if (tid < kSub) sh.sub.hi[tid] = sh.sub.lo[tid] = 0u;
  }
  cluster_wait();  // every CTA of the cluster runs: its shared memory can be written
  float top, least;  // the largest logit, and the least of the threads' own largest
  {
    const uint32_t bits = mine > -INFINITY ? rising(mine) : 0u, high = __reduce_max_sync(kFull, bits);
    const uint32_t low = ~__reduce_min_sync(kFull, bits ? bits : 0xFFFFFFFFu);  // turned round: 0 where there is none
    uint64_t e[4];
    tell((uint64_t)high << 32 | low, e);
    uint32_t h = 0, l = 0;
#pragma unroll
    for (uint32_t i = 0; i < 4u; ++i) {
      h = max(h, (uint32_t)(e[i] >> 32));
      l = max(l, (uint32_t)e[i]);
    }
    h = __reduce_max_sync(kFull, h);
    top = h ? from_rising(h) : -INFINITY;
    least = from_rising(~__reduce_max_sync(kFull, l));
  }
  // warps own consecutive pieces of the slice, a lane four consecutive logits of 128
  const uint32_t piece = (n + 4u * kThreads - 1u) / (4u * kThreads) * 128u, w0 = min(warp * piece, n), w1 = min(w0 + piece, n);
  auto read4 = [&](uint32_t i, uint32_t end, float (&x)[4]) {
    const float4 y = i < end ? *reinterpret_cast<const float4*>(xs + i) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;  // past the slice's end lies -inf
  };
  const bool p_on = top_p < 1.f;
  // the first token of the largest alone, or none
  if (top == -INFINITY || !(temperature > 0.f) || !(top_p > 0.f || top_p != top_p) || min_p > 1.f) {
    uint32_t at = kIndexMask + 1u;
    for (uint32_t i = w0 + 4u * lane; i < w1 && at > kIndexMask; i += 128u) {
      float x[4];
      read4(i, w1, x);
#pragma unroll
      for (int j = 3; j >= 0; --j)
        if (x[j] == top) at = from + i + j;
    }
    uint64_t e[4];
    tell(kIndexMask + 1u - __reduce_min_sync(kFull, at), e);
    const uint32_t first = __reduce_max_sync(kFull, (uint32_t)max(max(e[0], e[1]), max(e[2], e[3])));
    if (rank == 0 && tid == 0) {
      p.token[row] = top == -INFINITY ? -1 : (int32_t)(kIndexMask + 1u - first);
      if (p.logprob) p.logprob[row] = top == -INFINITY ? -INFINITY : 0.f;
    }
    return;
  }
  const bool infinite = top == INFINITY;
  if (infinite) {  // the infinite ones alone are kept, as equals: 0 takes their place, and -inf the others'
    for (uint32_t i = tid; i < (n + 3u) / 4u * 4u; i += kThreads) xs[i] = xs[i] == INFINITY ? 0.f : -INFINITY;
    mine = mine == INFINITY ? 0.f : -INFINITY;
    top = least = 0.f;
    __syncthreads();
  }
  Weights weight;
  weight.set(top, temperature, sh.powers);
  const uint64_t best = order_of(top, 0u);  // nothing is before this
  const uint32_t k = k_given > 0 && (uint32_t)k_given < p.vocab ? (uint32_t)k_given : 0u;

  uint64_t keep = 0;  // tokens at or after this are kept
  if (min_p > 0.f) {  // the least logit with t >= log2(min_p), by a search of one warp over the numbers' order
    if (warp == 0) {
      uint32_t lo = rising(-INFINITY), hi = rising(top);  // hi is kept
      if (min_p < 1.f) {
        const uint32_t b = __float_as_uint(min_p), e = b >> 23;
        const Pair edge = e ? log2_of(((b & 0x7FFFFFu) | 0x800000u) << 6, (int)e - 127, sh.powers) : log2_of((uint64_t)b, 149, sh.powers);
        while (lo < hi) {
          const uint32_t step = (hi - lo) / 33u + 1u, at = min(lo + (lane + 1u) * step - 1u, hi);  // rising over the lanes
          const float x = from_rising(at);
          const Pair t = weight.both(x);
          const bool in = at == hi || (x > -INFINITY && (t.hi - edge.hi) + (t.lo - edge.lo) >= 0.f);
          const uint32_t votes = __ballot_sync(kFull, in);
          const uint32_t first = votes ? __ffs(votes) - 1u : 32u;  // the first lane whose number is kept
          const uint32_t new_lo = min(lo + first * step, hi);
          hi = first < 32u ? min(lo + (first + 1u) * step - 1u, hi) : hi;
          lo = new_lo;
        }
      }
      if (lane == 0) sh.told[1] = hi;
    }
    __syncthreads();
    keep = sh.told[1] << kIndexBits;
    __syncthreads();
  }
  auto target_of = [&](uint64_t total) { return target(u, total); };
  auto answer = [&](uint64_t order, uint64_t total) {
    p.token[row] = (int32_t)index_of(order);
    if (p.logprob) {  // ln 2 (t - log2(total / 2^45))
      const float x = logit_of(order);
      const Pair sum = log2_of(total, kOne, sh.powers);
      const Pair t = x == top ? Pair{0.f, 0.f} : weight.both(x);
      const Pair d = exact_sum(t.hi, -sum.hi);
      const float low = d.lo + (t.lo - sum.lo), h = d.hi * kLn2;
      p.logprob[row] = h + fmaf(low, kLn2, fmaf(d.hi, kLn2Low, fmaf(d.hi, kLn2, -h)));
    }
  };
  // Tokens of a warp's piece into the first CTA's list, in no order: 4 bits of hits[] for each 128 logits of the piece.
  constexpr uint32_t kBlocks = TQ_SAMPLE_MAX_VOCAB / kMaxCluster / kWarps / 1024u;  // of 1024 logits of a piece
  auto place_of = [&](uint32_t block, uint32_t bit) { return w0 + block * 1024u + (bit >> 2) * 128u + 4u * lane + (bit & 3u); };
  auto list_hits = [&](const uint32_t (&hits)[kBlocks], auto logit) {
    uint32_t own = 0;
#pragma unroll
    for (uint32_t b = 0; b < kBlocks; ++b) own += __popc(hits[b]);
    if (!__any_sync(kFull, own != 0u)) return;
    const uint32_t upto = warp_upto(own, lane);
    uint32_t at = 0;
    if (lane == 31) at = add_remote(&sh.listed, 0u, upto);
    at = __shfl_sync(kFull, at, 31) + upto - own;
#pragma unroll
    for (uint32_t b = 0; b < kBlocks; ++b) {
      for (uint32_t left = hits[b]; left != 0u; left &= left - 1u, ++at) {
        const uint32_t i = place_of(b, __ffs(left) - 1u);
        if (at < kList) store_remote(&sh.list[at], 0u, order_of(logit(i), from + i));
      }
    }
    __syncwarp();
  };
  constexpr uint32_t kEach = kList / kThreads;  // consecutive entries of the list to a thread
  auto scan = [&](uint64_t sum, uint64_t& total) { return scan_cta(sh, sum, total); };

  // Bisection of the order: the last place before which less than `bound` (a weight, or a number) lies.
  auto before = [&](uint64_t order, bool count) {
    uint64_t v = 0, prev;
    for (uint32_t i = tid; i < n; i += kThreads)
      if (order_of(xs[i], from + i) > order) v += count ? 1ull : weight(xs[i]);
    return all(v, prev);
  };
  auto border = [&](uint64_t bound, bool count, uint64_t lo) {
    uint64_t hi = best;  // nothing is before it
    while (lo < hi) {
      const uint64_t mid = lo + (hi - lo) / 2u;
      if (before(mid, count) < bound)
        hi = mid;
      else
        lo = mid + 1u;
    }
    return hi;
  };
  // A logit of the slice from memory, as it was taken.
  auto logit_at = [&](uint32_t i) {
    const float x = load1<TYPE>(p.logits, row_at + i);
    return infinite ? (x == INFINITY ? 0.f : -INFINITY) : x != x ? -INFINITY : x + 0.f;
  };
  // A weight out of 32 bits.
  auto weight_of = [&](uint32_t code) {
    const uint32_t turned = code >> 22;
    if (turned == kSmallPlace) return (uint64_t)(code & 0x3FFFFFu);
    const int place = kTopPlace - (int)turned;
    return (uint64_t)weight.value(place, (int)(code << 10) >> 10) << Weights::shift(place);
  };
  // Of the m tokens of a bin in the list the one with which their sum, from the largest down, reaches `bound`: told to the cluster, by its first CTA.
  auto border_in_list = [&](uint32_t m, uint64_t bound, uint32_t bin) {
    const int place = kTopPlace - (int)bin, shift = Weights::shift(place);
    // Parts of the bin that fall with x; which token is in which decides nothing but the work.
    const float middle = weight.plain ? (weight.a + (float)place * 0.03125f) / weight.c : weight.top + (float)place * 0.03125f / weight.c;
    const float per = weight.c * 32.f * (float)kSub;
    auto part = [&](float x) { return (uint32_t)fminf(fmaxf((middle - x) * per + 0.5f * (float)kSub, 0.f), (float)(kSub - 1u)); };
    const bool parts = m > kNear;
    uint64_t ahead = 0;
    uint32_t chosen = 0;
    if (parts) {
      for (uint32_t i = tid; i < m; i += kThreads) {
        const float x = logit_of(sh.list[i]);
        const uint32_t v = (uint32_t)(weight(x) >> shift), b = part(x);
        atomicAdd(&sh.sub.hi[b], v >> 15);
        atomicAdd(&sh.sub.lo[b], v & 0x7FFFu);
      }
      __syncthreads();
      const uint64_t mass = tid < kSub ? (((uint64_t)sh.sub.hi[tid] << 15) + sh.sub.lo[tid]) << shift : 0ull;
      uint64_t sum;
      const uint64_t prev = scan(mass, sum);
      if (prev < bound && prev + mass >= bound) {
        sh.told[0] = tid;
        sh.told[1] = prev;
      }
      __syncthreads();
      chosen = (uint32_t)sh.told[0];
      ahead = sh.told[1];
    }
    for (uint32_t i = tid; i < m; i += kThreads) {
      const uint64_t order = sh.list[i];
      const float x = logit_of(order);
      if (parts && part(x) != chosen) continue;
      const uint32_t at = atomicAdd(&sh.near, 1u);
      if (at >= kNear) continue;
      sh.close[at] = order;
      sh.close_w[at] = weight(x);
    }
    __syncthreads();
    const uint32_t near = sh.near;
    if (near <= kNear) {  // each with each, four threads to a token
      const uint32_t j = tid / 4u;
      const uint64_t order = j < near ? sh.close[j] : ~0ull;
      uint64_t at = 0;
      for (uint32_t i = tid % 4u; i < near; i += 4u) at += sh.close[i] > order ? sh.close_w[i] : 0ull;
      at += __shfl_xor_sync(kFull, at, 1);
      at += __shfl_xor_sync(kFull, at, 2);
      at += ahead;
      if (j < near && at < bound && at + sh.close_w[j] >= bound) {
        for (uint32_t r = tid % 4u; r < ctas; r += 4u) store_remote(&sh.told[0], r, order);
      }
      return;
    }
    sort_list(sh.list, m, tid);
    uint64_t w[kEach], own = 0, sum;
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
      const uint32_t j = tid * kEach + i;
      w[i] = j < m ? weight(logit_of(sh.list[j])) : 0ull;
      own += w[i];
    }
    uint64_t at = scan(own, sum);
#pragma unroll
    for (uint32_t i = 0; i < kEach; ++i) {
      const uint32_t j = tid * kEach + i;
      if (j < m && at < bound && at + w[i] >= bound) {
        for (uint32_t r = 0; r < ctas; ++r) store_remote(&sh.told[0], r, sh.list[j]);
      }
      at += w[i];
    }
  };
  // The filters and the token of at most kNear listed ones by comparing each with each, four threads to a token: three steps of the CTA,
  // where sorting by order and by place takes some thirty (one row 10.1 us with that, 8.7 with this).
  auto few_in_list = [&](uint32_t m, uint32_t k, uint64_t keep) {
    const uint32_t j = tid / 4u, part = tid % 4u;
    const uint64_t order = j < m ? sh.list[j] : 0ull, own = j < m ? weight(logit_of(order)) : 0ull;
    if (part == 0u && j < m) sh.close_w[j] = own;
    __syncthreads();
    uint32_t ahead = 0;
    uint64_t before = 0;
    for (uint32_t i = part; i < m; i += 4u) {
      const bool larger = sh.list[i] > order;
      ahead += larger ? 1u : 0u;
      before += larger ? sh.close_w[i] : 0ull;
    }
#pragma unroll
    for (int d = 1; d < 4; d *= 2) {
      ahead += __shfl_xor_sync(kFull, ahead, d);
      before += __shfl_xor_sync(kFull, before, d);
    }
    bool in = j < m && ahead < k;
    if (p_on) {
      const uint64_t of_warp = warp_sum(in && part == 0u ? own : 0ull);
      if (lane == 0) sh.warps[warp] = of_warp;
      __syncthreads();
      const uint64_t bound = bound_of(top_p, warp_sum(lane < kWarps ? sh.warps[lane] : 0ull));  // (all lanes take part in the sum)
      in = in && before < bound;
    }
    in = in && order >= keep;
    __syncthreads();
    if (part == 0u && j < m) sh.close_w[j] = in ? own : 0ull;
    __syncthreads();
    const uint32_t at = index_of(order);
    uint64_t prev = 0, total = 0;
    for (uint32_t i = part; i < m; i += 4u) {
      const uint64_t w = sh.close_w[i];
      total += w;
      prev += index_of(sh.list[i]) < at ? w : 0ull;
    }
#pragma unroll
    for (int d = 1; d < 4; d *= 2) {
      total += __shfl_xor_sync(kFull, total, d);
      prev += __shfl_xor_sync(kFull, prev, d);
    }
    const uint64_t target = target_of(total);
    if (in && part == 0u && target >= prev && target < prev + own) answer(order, total);
  };
  bool coded = false;  // weights lie where the logits were
  bool summed = false;  // the bins have the sums of what is kept, hits[] the tokens in the border's
  bool whole_bin = false;  // and all of them are kept
  uint32_t hits[kBlocks] = {}, border_bin = 0;
  bool searched = !p_on && k == 0u;  // the border is known

  if (k != 0u && k <= kListK) {
    // ---- top-k: a bound from the threads' maxima, and a list -----------------------------------------------
    // bins that fall with x from the largest logit to the least of the maxima; what is below is in the last.  One bin where a bin's width would be
    // 0, infinite, or so small that bins to a unit are (a span below 7.5e-37).
    const float span = top - least, per = (float)(kKBins - 1u) / span, scale = span > 0.f && per < INFINITY ? per : 0.f;
    auto bin_at = [&](float x) { return min((uint32_t)((top - x) * scale), kKBins - 1u); };
    if (mine > -INFINITY) atomicAdd(&sh.k_bins[bin_at(mine)], 1u);
    cluster_sync();
    uint32_t in_bin = 0;
    if (tid < kKBins) {
      uint32_t c[kMaxCluster];
#pragma unroll
      for (uint32_t r = 0; r < kMaxCluster; ++r) c[r] = r < ctas ? load_remote(&sh.k_bins[tid], r) : 0u;
#pragma unroll
      for (uint32_t r = 0; r < kMaxCluster; ++r) in_bin += c[r];
    }
    uint64_t maxima;
    const uint32_t ahead = (uint32_t)scan(in_bin, maxima);
    if (tid == 0) sh.told[0] = kKBins - 1u;  // fewer maxima than k: nothing is left out
    __syncthreads();
    if (ahead < k && ahead + in_bin >= k) sh.told[0] = tid;
    cluster_sync();
    const uint32_t cut = (uint32_t)sh.told[0];
    // the products of bin_at, compared with the bin's end; where all are alike, or in the last bin, everything is listed: the products are then with 0,
    // which is not beyond the end even where the distance is infinite (a choice beside the comparison: one row 11.3 us, so 10.3, in a graph)
    const float end = cut == kKBins - 1u || scale == 0.f ? INFINITY : (float)(cut + 1u), by = end < INFINITY ? scale : 0.f;
#pragma unroll
    for (uint32_t b = 0; b < kBlocks; ++b) {
      for (uint32_t s = 0; s < 8u && w0 + b * 1024u + s * 128u < w1; ++s) {
        float x[4];
        read4(w0 + b * 1024u + s * 128u + 4u * lane, w1, x);
        uint32_t mask = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) mask |= x[j] > -INFINITY && !((top - x[j]) * by >= end) ? 1u << j : 0u;
        hits[b] |= mask << (4u * s);
      }
    }
    list_hits(hits, [&](uint32_t i) { return xs[i]; });
    cluster_sync();
    const uint32_t m = load_remote(&sh.listed, 0u);
    if (m <= kList) {
      cluster_arrive();  // the first CTA stays until all have read that
      if (rank != 0) return;
      if (m <= kNear) {
        few_in_list(m, k, keep);
        cluster_wait();
        return;
      }
      const uint64_t found = token_of_list(sh, weight, m, k, top_p, keep, u, scale * ((float)kParts / fminf(end, 2.f * (float)kKBins)), p.vocab);
      if (found != ~0ull) {
        if (tid == 0) answer(found, sh.told[1]);
        cluster_wait();
        return;
      }
      sort_list(sh.list, m, tid);
      uint32_t kept = min(k, m);
      uint64_t w[kEach], sum = 0, total, prev;
      if (p_on) {
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
          const uint32_t j = tid * kEach + i;
          w[i] = j < kept ? weight(logit_of(sh.list[j])) : 0ull;
          sum += w[i];
        }
        prev = scan(sum, total);
        const uint64_t bound = bound_of(top_p, total);
        uint32_t in = 0;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
          in += tid * kEach + i < kept && prev < bound ? 1u : 0u;
          prev += w[i];
        }
        scan(in, total);
        kept = max(1u, (uint32_t)total);
      }
      if (keep != 0ull) {  // min-p
        uint32_t in = 0;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) in += tid * kEach + i < kept && sh.list[tid * kEach + i] >= keep ? 1u : 0u;
        scan(in, total);
        kept = (uint32_t)total;
      }
      // those in the order of the vocabulary
      uint64_t own[kEach];
      __syncthreads();
#pragma unroll
      for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t j = tid * kEach + i;
        if (j < kept) sh.list[j] = (sh.list[j] & kIndexMask) << 32 | sh.list[j] >> kIndexBits;
      }
      __syncthreads();
      sort_list(sh.list, kept, tid);
      sum = 0;
#pragma unroll
      for (uint32_t i = 0; i < kEach; ++i) {
        const uint32_t j = tid * kEach + i;
        own[i] = j < kept ? sh.list[j] << kIndexBits & (0xFFFFFFFFull << kIndexBits) | sh.list[j] >> 32 : 0ull;
        w[i] = j < kept ? weight(logit_of(own[i])) : 0ull;
        sum += w[i];
      }
      prev = scan(sum, total);
      const uint64_t target = target_of(total);
      if (target >= prev && target < prev + sum) {
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
          if (target >= prev && target < prev + w[i]) answer(own[i], total);
          prev += w[i];
        }
      }
      cluster_wait();
      return;
    }
  }
  if (!searched && k == 0u) {
    // ---- top-p: a histogram of the weights, and a list of the bin with the border -----------------------------
    // (the logits of a bin's tokens are read again from memory, for their order)
    uint64_t rest = 0;  // of the octaves below
    for (uint32_t i0 = w0; i0 < w1; i0 += 128u) {
      float x[4];
      read4(i0 + 4u * lane, w1, x);
      uint32_t code[4];
      weight.four(x, [&](int j, bool fine, int place, int q) {
        code[j] = code_of(fine, place, q);
        if (fine) {
          const uint32_t v = weight.value(place, q);
          atomicAdd(&sh.bins.hi[kTopPlace - place], v >> 15);
          atomicAdd(&sh.bins.lo[kTopPlace - place], v & 0x7FFFu);
        } else {
          rest += (uint32_t)q;
        }
      });
      // from here on the weights lie where the logits were
      if (i0 + 4u * lane < w1) *reinterpret_cast<uint4*>(xs + i0 + 4u * lane) = make_uint4(code[0], code[1], code[2], code[3]);
    }
    coded = true;
    cluster_sync();
    // this CTA's bins of all CTAs: consecutive ones, up to two to a thread
    const uint32_t share = (kBins + ctas - 1u) / ctas, each = (share + kThreads - 1u) / kThreads;
    uint64_t mass[2] = {0, 0};
#pragma unroll
    for (uint32_t j = 0; j < 2u; ++j) {
      const uint32_t mine_of = tid * each + j, b = rank * share + mine_of;
      if (j >= each || mine_of >= share || b >= kBins) continue;
      uint32_t hi[kMaxCluster], lo[kMaxCluster];
#pragma unroll
      for (uint32_t r = 0; r < kMaxCluster; ++r) {
        hi[r] = r < ctas ? load_remote(&sh.bins.hi[b], r) : 0u;
        lo[r] = r < ctas ? load_remote(&sh.bins.lo[b], r) : 0u;
      }
      uint64_t sum_hi = 0, sum_lo = 0;
#pragma unroll
      for (uint32_t r = 0; r < kMaxCluster; ++r) sum_hi += hi[r], sum_lo += lo[r];
      mass[j] = ((sum_hi << 15) + sum_lo) << Weights::shift(kTopPlace - (int)b);
    }
    uint64_t ahead, below;
    const uint64_t sum = mass[0] + mass[1], upto = warp_upto(sum, lane), total = all_of_two(sum, rest, ahead, below) + below;
    const uint64_t bound = bound_of(top_p, total);
    uint64_t prev = ahead + upto - sum;
#pragma unroll
    for (uint32_t j = 0; j < 2u; ++j) {
      if (mass[j] != 0ull && prev < bound && prev + mass[j] >= bound) {
        // less than two of the bin's least weights (2^(-1/64) of the one in its middle) are one token
        const uint32_t b = rank * share + tid * each + j;
        const int place = kTopPlace - (int)b;
        const uint64_t one = (uint64_t)weight.value(place, 0) << Weights::shift(place), single = mass[j] < 2u * one - one / 16u ? 1ull << 32 : 0ull;
        for (uint32_t r = 0; r < ctas; ++r) {
          store_remote(&sh.told[0], r, single | b);
          store_remote(&sh.told[1], r, prev);
        }
      }
      prev += mass[j];
    }
    cluster_sync();
    const uint64_t bin = sh.told[0], up_to_bin = sh.told[1];
    if (bin != ~0ull) {
      border_bin = (uint32_t)bin;
      whole_bin = bin >> 32 != 0ull && keep == 0ull;
      if (!whole_bin) {
#pragma unroll
        for (uint32_t b = 0; b < kBlocks; ++b) {
          for (uint32_t s = 0; s < 8u && w0 + b * 1024u + s * 128u < w1; ++s) {
            float x[4];
            read4(w0 + b * 1024u + s * 128u + 4u * lane, w1, x);  // (past the end: a place that no bin has)
            uint32_t mask = 0;
#pragma unroll
            for (int j = 0; j < 4; ++j) mask |= __float_as_uint(x[j]) >> 22 == border_bin ? 1u << j : 0u;
            hits[b] |= mask << (4u * s);
          }
        }
      }
      summed = keep == 0ull && !whole_bin;
    }
    if (whole_bin) {
      searched = true;
    } else if (bin != ~0ull) {
      list_hits(hits, logit_at);
      cluster_sync();
      const uint32_t m = load_remote(&sh.listed, 0u);
      if (m <= kList) {
        if (rank == 0) border_in_list(m, bound - up_to_bin, border_bin);
        cluster_sync();
        keep = max(keep, sh.told[0]);
        searched = true;
      } else {
        summed = false;
      }
    }
  }
  if (!searched) {
    if (coded) {  // too many in one bin: the logits again
      for (uint32_t i = tid; i < n; i += kThreads) xs[i] = logit_at(i);
      if (tid < 4u && n + tid < (n + 3u) / 4u * 4u) xs[n + tid] = -INFINITY;
      __syncthreads();
      coded = false;
    }
    uint64_t edge = 0;
    if (k != 0u) edge = border(k, true, 0ull);
    if (p_on) {
      const uint64_t sum = before(edge ? edge - 1u : 0u, false);  // 0 is no token's place
      edge = border(bound_of(top_p, sum), false, edge);
    }
    keep = max(keep, edge);
  }

  // ---- the token up to which more than u of the kept sum lies ---------------------------------------
  const float keep_x = logit_of(keep);  // below it nothing is kept
  const uint32_t keep_at = index_of(keep);  // and of its equals the first ones
  // coded: places above this (weights below) are not kept; of the tokens of edge_place it goes by the logit, where their q is next to the border's:
  // q rises with x but for its roundings, together less than 2 units.
  int keep_place = 1, edge_place = -1, edge_q = 0, edge_near = 0;
  if (coded && whole_bin) {
    keep_place = (int)border_bin;
  } else if (coded) {
    const float s = weight.base(keep_x) + Weights::kRound;
    keep_place = (int)kSmallPlace;
    edge_near = 1 << 24;  // small ones: always by the logit
    if (keep_x > -INFINITY && !Weights::is_small(s)) {
      keep_place = kTopPlace - Weights::place_in(s);
      edge_q = weight.fine(keep_x, s);
      edge_near = 2;
    }
    edge_place = keep_place;
  }
  auto in_edge = [&](uint32_t i, uint32_t code) {
    const int d = ((int)(code << 10) >> 10) - edge_q;
    if (d > edge_near || d < -edge_near) return d > 0;
    const float y = i < n ? logit_at(i) : -INFINITY;
    return y > keep_x || (y == keep_x && from + i <= keep_at);
  };
  // weights of four logits, 0 where they are not kept
  const bool every = keep == 0ull, ties = keep_at != kIndexMask;
  auto kept = [&](uint32_t i, uint32_t end, uint64_t (&w)[4]) {
    float x[4];
    read4(i, end, x);
    if (coded) {
      int place[4];
      bool any = false;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        place[j] = i < end ? (int)(__float_as_uint(x[j]) >> 22) : (int)kSmallPlace + 1;
        any = any || place[j] <= keep_place;
        w[j] = 0ull;
      }
      if (!__any_sync(kFull, any)) return false;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        if (place[j] > keep_place) continue;
        const uint32_t code = __float_as_uint(x[j]);
        if (place[j] == edge_place && !in_edge(i + j, code)) continue;
        w[j] = weight_of(code);
      }
      return true;
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = 0ull;
    if (!every) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (x[j] < keep_x || (ties && x[j] == keep_x && from + i + j > keep_at)) x[j] = -INFINITY;
      if (!__any_sync(kFull, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) > -INFINITY)) return false;
    }
    weight.four(x, [&](int j, bool fine, int place, int q) { w[j] = fine ? (uint64_t)weight.value(place, q) << Weights::shift(place) : (uint64_t)(uint32_t)q; });
    return true;
  };
  uint64_t sum_mine = 0, sum, total, target;
  auto add_kept = [&] {
    for (uint32_t i0 = w0; i0 < w1; i0 += 128u) {
      uint64_t w[4];
      kept(i0 + 4u * lane, w1, w);
      sum_mine += (w[0] + w[1]) + (w[2] + w[3]);
    }
  };
  uint64_t of_warp;
  if (summed) {  // the CTAs' sums are in their bins: only the one that has the token adds up its tokens
    for (uint32_t b = tid; b < border_bin; b += kThreads) sum_mine += (((uint64_t)sh.bins.hi[b] << 15) + sh.bins.lo[b]) << Weights::shift(kTopPlace - (int)b);
#pragma unroll
    for (uint32_t b = 0; b < kBlocks; ++b) {
      for (uint32_t left = hits[b]; left != 0u; left &= left - 1u) {
        const uint32_t i = place_of(b, __ffs(left) - 1u), code = __float_as_uint(xs[i]);
        if (in_edge(i, code)) sum_mine += weight_of(code);
      }
    }
    __syncwarp();
    uint64_t ahead, own;
    total = all_of_ctas(sum_mine, ahead, own);
    target = target_of(total);
    if (target < ahead || target - ahead >= own) return;
    sum_mine = 0;
    add_kept();
    of_warp = warp_sum(sum_mine);
    if (lane == 0) sh.warps[warp] = of_warp;
    __syncthreads();
    sum = ahead + warp_sum(lane < warp ? sh.warps[lane] : 0ull);
  } else {
    add_kept();
    of_warp = warp_sum(sum_mine);
    total = all(sum_mine, sum);
    target = target_of(total);
  }
  if (lane == 0 && target >= sum && target < sum + of_warp) {
    sh.found[0] = warp;
    sh.found[1] = sum;
  }
  __syncthreads();
  if (sh.found[0] == ~0ull) return;  // another CTA has it
  // a warp of the CTA to each 128 logits of the piece that has it (there are no more of them than warps)
  static_assert(TQ_SAMPLE_MAX_VOCAB / kMaxCluster / kWarps <= 128u * kWarps, "a piece has a part for every warp at most");
  const uint32_t p0 = min((uint32_t)sh.found[0] * piece, n), p1 = min(p0 + piece, n), i = p0 + warp * 128u + 4u * lane;
  uint64_t w[4] = {0, 0, 0, 0};
  kept(i, p1, w);
  const uint64_t own = (w[0] + w[1]) + (w[2] + w[3]);
  uint64_t in_piece, at = sh.found[1] + scan(own, in_piece);
  if (target < at || target >= at + own) return;
  uint32_t j = 0;
#pragma unroll
  for (uint32_t x = 0; x < 3u; ++x) {
    if (j == x && at + w[x] <= target) {
      at += w[x];
      ++j;
    }
  }
  answer(order_of(coded ? logit_at(i + j) : xs[i + j], from + i + j), total);
}

template <int TYPE>
int launch(SampleParams& p, uint32_t rows, cudaStream_t st) {
  auto kern = sample_kernel<TYPE>;
  // eight CTAs to a row, fewer where a CTA would have less than 2048 logits
  uint32_t ctas = kMaxCluster;
  while (ctas > 1 && p.vocab < 2048u * ctas) ctas /= 2;
  if (rows > 0x7FFFFFFFu / ctas) return TQ_ERR_UNSUPPORTED_SHAPE;
  p.slice = ((p.vocab + ctas - 1u) / ctas + 7u) / 8u * 8u;
  p.vectors = ((uintptr_t)p.logits & 15u) == 0 && (rows == 1 || (p.row_stride * (TYPE == TQ_TYPE_F32 ? 4 : 2)) % 16 == 0);
  const char* what = "sample launch";
  if (int rc = tq_ensure_dynamic_smem((const void*)kern, kHead + TQ_SAMPLE_MAX_VOCAB / kMaxCluster * sizeof(float), what)) return rc;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(rows * ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = kHead + p.slice * sizeof(float);
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return tq_cuda_status((int)cudaLaunchKernelEx(&cfg, kern, p), what);
}

bool bad_ptr(const void* ptr, bool optional) { return (!optional && ptr == nullptr) || ((uintptr_t)ptr & 3u) != 0; }

}  // namespace

extern "C" int tq_sample(const void* d_logits, int x_type, int64_t row_stride, uint32_t rows, uint32_t vocab, const float* d_uniform,
                         const float* d_temperature, const int32_t* d_top_k, const float* d_top_p, const float* d_min_p,
                         int32_t* d_token, float* d_logprob, void* cuda_stream) {
  if ((x_type != TQ_TYPE_BF16 && x_type != TQ_TYPE_F32) || vocab == 0) return TQ_ERR_INVALID_ARG;
  if (vocab > TQ_SAMPLE_MAX_VOCAB) return TQ_ERR_UNSUPPORTED_SHAPE;
  if (rows == 0) return TQ_OK;
  if (!d_logits || ((uintptr_t)d_logits & (x_type == TQ_TYPE_F32 ? 3u : 1u))) return TQ_ERR_INVALID_ARG;
  if (bad_ptr(d_uniform, false) || bad_ptr(d_token, false) || bad_ptr(d_temperature, true) || bad_ptr(d_top_k, true) || bad_ptr(d_top_p, true) ||
      bad_ptr(d_min_p, true) || bad_ptr(d_logprob, true))
    return TQ_ERR_INVALID_ARG;
  SampleParams p{};
  p.logits = d_logits;
  p.row_stride = row_stride;
  p.uniform = d_uniform;
  p.temperature = d_temperature;
  p.top_k = d_top_k;
  p.top_p = d_top_p;
  p.min_p = d_min_p;
  p.token = d_token;
  p.logprob = d_logprob;
  p.vocab = vocab;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return x_type == TQ_TYPE_F32 ? launch<TQ_TYPE_F32>(p, rows, st) : launch<TQ_TYPE_BF16>(p, rows, st);
}
