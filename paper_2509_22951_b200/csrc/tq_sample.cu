// One token for each row of logits (tq_sample): temperature, top-k, top-p, min-p, and the inverse of the distribution
// function at a given uniform number.
//
// Exact sums.  Every decision is a comparison of sums of weights w = 2^t, t = (x - max) log2(e) / temperature, with a bound: a
// weight is therefore an integer W = round(2^45 w), and sums of up to 2^18 of them are exact in 64 bits whatever their
// order, so that neither the split of a row nor the order of atomics can change a token.  t is held in two fp32 numbers (difference and
// product with their errors, by the usual sums without loss of Dekker and Knuth); rounded to 1/256 it gives a place in a table of 2^(i/256) and an
// octave, and what is left a cubic, to 29 bits.  (fp64 would say it in fewer words, but its instructions take some 40 cycles of an SM's
// quarter each: a row of 128256 tokens 18.6 us that way, %%% this way.)  W below 2^21 (t < -24) is taken from the fp32 exponential, to a unit or two.
//
// Order.  Tokens fall by (x, lower index first): as one integer, the logit's bits made to rise with it above the index turned
// round.  What is kept is all that is not below a border in that order, so every filter is a search for its border.
//
// A row is read once: a cluster of up to eight CTAs holds it in shared memory and speaks through distributed shared memory.  Then
//   top-k (up to 1024): the k-th largest of the threads' own maxima is a bound of the k-th logit that few others pass: those go to one CTA in
//          the order of the vocabulary, which sorts them and does the rest;
//   top-p alone: a histogram of the weights over 64 bins an octave (exact: two integers a bin) finds the bin of the border, whose
//          tokens one CTA sorts; then every CTA adds up what it keeps;
//   neither, or min-p alone: the border is known; every CTA adds up what it keeps.
// Where so many logits are alike that a list does not hold them (2048), and for larger k, the border is found by bisection of the order.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "tq_internal.h"
#include "tq_ops_common.cuh"

namespace {

using namespace tq_ops;

constexpr uint32_t kThreads = 512, kWarps = kThreads / 32;
constexpr uint32_t kMaxCluster = 8;
constexpr uint32_t kIndexBits = 18;
static_assert((1u << kIndexBits) == TQ_SAMPLE_MAX_VOCAB, "a token's index fits its place in the order");
constexpr uint32_t kIndexMask = (1u << kIndexBits) - 1u;
constexpr int kOne = 45;     // W of the largest logit is 2^45
constexpr int kOctaves = 24; // of the histogram, and of the weights that are computed to 29 bits
constexpr uint32_t kBins = kOctaves * 64u;
constexpr uint32_t kList = 2048;   // tokens that one CTA sorts
constexpr uint32_t kListK = 1024;  // largest k of the list: the threads' maxima bound it well up to a quarter of their number
constexpr uint32_t kKBins = 256;   // of the threads' maxima

// 2^(i / 256) with 29 bits behind the point
struct Powers {
  uint32_t v[256];
};
constexpr Powers powers() {
  Powers p{};
  for (int i = 0; i < 256; ++i) {
    const double y = i * (0.69314718055994530942 / 256.0);
    double term = 1.0, sum = 1.0;
    for (int k = 1; k < 24; ++k) {
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
  uint64_t slots[2][kMaxCluster][2];  // what the cluster's CTAs tell one another; two sets, used in turn
  uint64_t warps[2][kWarps][2];
  uint64_t told[2];                   // by one CTA to all
  uint2 powers[256];                  // 2^(i / 256) with 29 bits behind the point, and as fp32
  uint32_t listed;                    // tokens in the list (of the first CTA)
  union {
    struct {
      uint32_t hi[kBins], lo[kBins];  // sums of the upper and lower 15 bits of the weights of a bin
    } bins;
    uint64_t list[kList];
    uint32_t k_bins[kKBins];
  };
};

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
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t at_rank(const void* ptr, uint32_t rank) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tq_sm100::smem_u32(ptr)), "r"(rank));
  return a;
}
__device__ __forceinline__ void store_remote(const uint64_t* ptr, uint32_t rank, uint64_t v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(at_rank(ptr, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ uint32_t load_remote(const uint32_t* ptr, uint32_t rank) {
  uint32_t v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at_rank(ptr, rank)) : "memory");
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

// Two fp32 numbers whose sum is meant, the second small against the first.
struct Pair {
  float hi, lo;
};
__device__ __forceinline__ Pair exact_sum(float a, float b) {
  const float s = a + b, t = s - a;
  return Pair{s, (a - (s - t)) + (b - t)};
}
constexpr float kLn2 = 0.693147182464599609375f, kLn2Low = -1.904654323148236e-09f;       // ln 2
constexpr float kLog2e = 1.44269502162933349609375f, kLog2eLow = 1.92596303178237e-08f;   // 1 / ln 2

// log2(m 2^(k - 29)), 2^29 <= m < 2^30, to 2^-30.
__device__ __forceinline__ Pair log2_of(uint32_t m, int k, const uint2* powers) {
  int i = min(max((int)(__log2f((float)m) * 256.f) - 29 * 256, 0), 255);
  if (powers[i].x > m && i > 0) --i;
  const float z = (float)(int32_t)(m - powers[i].x) / __uint_as_float(powers[i].y);  // 0 .. 0.0028
  return Pair{(float)k + (float)i * 0.00390625f, z * (1.f + z * (-0.5f + z * (0.33333334f - z * 0.25f))) * kLog2e};
}
__device__ __forceinline__ Pair log2_of(uint64_t v, int one, const uint2* powers) {  // log2(v 2^-one)
  const int top = 63 - __clzll((long long)v);
  return log2_of(top >= 29 ? (uint32_t)(v >> (top - 29)) : (uint32_t)v << (29 - top), top - one, powers);
}

struct Weights {
  float top, c, c_low;  // largest logit; log2(e) / temperature
  const uint2* powers;

  __device__ __forceinline__ void set(float top_, float temperature, const uint2* powers_) {
    top = top_;
    powers = powers_;
    c = c_low = 0.f;
    if (temperature < INFINITY) {
      const float T = fmaxf(temperature, 7.52316385e-37f);  // 2^-120: where the quotient stays finite
      c = kLog2e / T;
      c_low = (fmaf(-c, T, kLog2e) + kLog2eLow) / T;
    }
  }
  // t in fp32 (NaN where the distance overflows and the temperature is infinite: fine() takes that for 0)
  __device__ __forceinline__ float coarse(float x) const { return (x - top) * c; }
  __device__ __forceinline__ Pair both(float x) const {
    const Pair d = exact_sum(x, -top);
    const float t = d.hi * c;
    return Pair{t, fmaf(d.lo, c, fmaf(d.hi, c_low, fmaf(d.hi, c, -t)))};
  }
  __device__ __forceinline__ bool none(float x) const { return x == -INFINITY || (top == INFINITY && x != top); }
  // Place of t in 1/256 (octave n = place >> 8, at most -1) and the value of W = value << max(0, 16 + n): 29 bits of 2^fraction, or W itself below
  // octave -16.  For t down to some octaves below the histogram's.
  __device__ __forceinline__ uint32_t fine(float x, int& place) const {
    const Pair t = both(x);
    const float s = t.hi + 49152.0f;  // 1.5 * 2^15: rounded to 1/256
    place = __float_as_int(s) - 0x47400000;
    const float r = (t.hi - (s - 49152.0f)) + t.lo;  // -1/512 .. 1/512
    const bool whole = x == top || place > 0;  // (not a number: above every place)
    const uint2 base = powers[place & 255];
    constexpr float a1 = kLn2, a2 = 0.24022651f, a3 = 0.055504109f;  // (ln 2)^k / k!
    const float q = r * fmaf(r, fmaf(r, a3, a2), a1);
    // rounded to whole units of 2^-29
    uint32_t v = whole ? 1u << 29 : base.x + (__float_as_uint(fmaf(__uint_as_float(base.y), q, 12582912.0f)) - 0x4B400000u);
    if (whole || place == 0) {  // twice as much in octave -1, which then is the first
      place = -1;
      v *= 2u;
    }
    const int down = -16 - (place >> 8);
    return down > 0 ? (v + (1u << (down - 1))) >> down : v;
  }
  __device__ __forceinline__ static int shift(int place) { return max(0, 16 + (place >> 8)); }
  // Octaves below the histogram's.
  __device__ __forceinline__ uint32_t small(float t) const {
    float w;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(w) : "f"(t + (float)kOne));
    return t < -46.f ? 0u : __float2uint_rn(w);
  }
  __device__ __forceinline__ uint64_t operator()(float x) const {
    if (none(x)) return 0ull;
    const float t = coarse(x);
    if (t < -(float)kOctaves) return small(t);
    int place;
    const uint32_t v = fine(x, place);
    return (uint64_t)v << shift(place);
  }
  // Four at once, for a whole warp: the chains of fine() side by side, or none of them where all weights are small.  use(j, is fine, place,
  // value) for each; value is 0 where there is no weight.
  template <class Use>
  __device__ __forceinline__ void four(const float (&x)[4], Use use) const {
    float t[4];
    bool any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      t[j] = none(x[j]) ? -INFINITY : coarse(x[j]);
      any = any || !(t[j] < -(float)kOctaves);
    }
    if (!__any_sync(kFull, any)) {
#pragma unroll
      for (int j = 0; j < 4; ++j) use(j, false, -1, small(t[j]));
      return;
    }
    int place[4];
    uint32_t v[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = fine(t[j] < -(float)kOctaves ? top : x[j], place[j]);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool is_small = t[j] < -(float)kOctaves;
      use(j, !is_small, place[j], is_small ? small(t[j]) : v[j]);
    }
  }
};
// Four places to a bin; what lies below the histogram by a rounding is in its last.
__device__ __forceinline__ uint32_t bin_of(int place) { return min((uint32_t)(-1 - place) >> 2, kBins - 1u); }
// floor(f * v), f >= 0 an fp32 number below 1, and whether there is a remainder
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
// The least integer not below f * v: as many units and more are not less than f * v.
__device__ __forceinline__ uint64_t bound_of(float f, uint64_t v) {
  if (!(f > 0.f)) return 0ull;
  bool more;
  const uint64_t r = times(f, v, more);
  return r + (more ? 1ull : 0ull);
}

// Sorts list[0 .. n), n <= kList, from the largest down: by every entry's rank where there are few, else bitonic.
__device__ void sort_list(uint64_t* list, uint32_t n, uint32_t tid) {
  if (n <= 128u) {
    const uint64_t mine = tid < n ? list[tid] : 0ull;
    uint32_t rank = 0;
    if (tid < n)
      for (uint32_t i = 0; i < n; ++i) rank += list[i] > mine ? 1u : 0u;
    __syncthreads();
    if (tid < n) list[rank] = mine;
    __syncthreads();
    return;
  }
  uint32_t size = 256;
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

template <int TYPE>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const SampleParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  float* const xs = reinterpret_cast<float*>(smem + (sizeof(Shared) + 15u) / 16u * 16u);
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u, rank = cluster_rank(), ctas = cluster_size();
  const uint32_t row = blockIdx.x / ctas, from = min(rank * p.slice, p.vocab), n = min(p.slice, p.vocab - from);
  if (tid < 256) sh.powers[tid] = make_uint2(kPowers.v[tid], __float_as_uint((float)kPowers.v[tid]));
  if (tid == 0) sh.listed = 0u;
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  uint32_t turn = 0;
  // Two numbers of every thread added up (or the largest taken) over the CTA, then told to the whole cluster: of[r] is what CTA r had.
  // warps[turn] keeps what the warps had.
  auto all2 = [&](uint64_t& v0, uint64_t& v1, bool largest, uint64_t (&of0)[kMaxCluster]) {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const uint64_t a = __shfl_xor_sync(kFull, v0, d), b = __shfl_xor_sync(kFull, v1, d);
      v0 = largest ? (a > v0 ? a : v0) : v0 + a;
      v1 = largest ? (b > v1 ? b : v1) : v1 + b;
    }
    if (lane == 0) {
      sh.warps[turn][warp][0] = v0;
      sh.warps[turn][warp][1] = v1;
    }
    __syncthreads();
    if (warp == 0) {
      v0 = lane < kWarps ? sh.warps[turn][lane][0] : 0ull;
      v1 = lane < kWarps ? sh.warps[turn][lane][1] : 0ull;
#pragma unroll
      for (int d = 8; d > 0; d >>= 1) {
        const uint64_t a = __shfl_xor_sync(kFull, v0, d), b = __shfl_xor_sync(kFull, v1, d);
        v0 = largest ? (a > v0 ? a : v0) : v0 + a;
        v1 = largest ? (b > v1 ? b : v1) : v1 + b;
      }
      v0 = __shfl_sync(kFull, v0, 0);
      v1 = __shfl_sync(kFull, v1, 0);
      if (lane < ctas) {
        store_remote(&sh.slots[turn][rank][0], lane, v0);
        store_remote(&sh.slots[turn][rank][1], lane, v1);
      }
    }
    cluster_sync();
    v0 = v1 = 0;
#pragma unroll
    for (uint32_t i = 0; i < kMaxCluster; ++i) {
      of0[i] = i < ctas ? sh.slots[turn][i][0] : 0ull;
      const uint64_t b = i < ctas ? sh.slots[turn][i][1] : 0ull;
      v0 = largest ? (of0[i] > v0 ? of0[i] : v0) : v0 + of0[i];
      v1 = largest ? (b > v1 ? b : v1) : v1 + b;
    }
    turn ^= 1u;
  };
  uint64_t of[kMaxCluster];

  // ---- the row; its first token in falling order; the largest logit of every thread ------------------------
  float mine = -INFINITY;
  uint32_t mine_at = 0;
  auto take = [&](float x, uint32_t i) {
    x = x != x ? -INFINITY : x + 0.f;  // -0 is 0
    if (x > mine) {
      mine = x;
      mine_at = i;
    }
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
          y.x = take(__uint_as_float(v[k].x), at);
          y.y = take(__uint_as_float(v[k].y), at + 1u);
          y.z = take(__uint_as_float(v[k].z), at + 2u);
          y.w = take(__uint_as_float(v[k].w), at + 3u);
          *reinterpret_cast<float4*>(xs + at) = y;
        } else {
          float4 y, z;
          y.x = take(bf16_lo(v[k].x), at);
          y.y = take(bf16_hi(v[k].x), at + 1u);
          y.z = take(bf16_lo(v[k].y), at + 2u);
          y.w = take(bf16_hi(v[k].y), at + 3u);
          z.x = take(bf16_lo(v[k].z), at + 4u);
          z.y = take(bf16_hi(v[k].z), at + 5u);
          z.z = take(bf16_lo(v[k].w), at + 6u);
          z.w = take(bf16_hi(v[k].w), at + 7u);
          *reinterpret_cast<float4*>(xs + at) = y;
          *reinterpret_cast<float4*>(xs + at + 4u) = z;
        }
      }
    }
    for (uint32_t i = whole * kPer + tid; i < n; i += kThreads) xs[i] = take(load1<TYPE>(p.logits, row_at + i), i);
  } else {
    for (uint32_t i = tid; i < n; i += kThreads) xs[i] = take(load1<TYPE>(p.logits, row_at + i), i);
  }
  if (tid < 4u && n + tid < (n + 3u) / 4u * 4u) xs[n + tid] = -INFINITY;
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // every CTA of the cluster runs: its shared memory can be written
  uint64_t best = mine > -INFINITY ? order_of(mine, from + mine_at) : 0ull;
  uint64_t lowest = mine > -INFINITY ? (uint64_t)~rising(mine) : 0ull;  // the least of the threads' maxima, turned round
  all2(best, lowest, true, of);
  const float temperature = p.temperature ? p.temperature[row] : 1.f;
  if (best == 0ull || !(temperature > 0.f)) {
    if (rank == 0 && tid == 0) {
      p.token[row] = best == 0ull ? -1 : (int32_t)(kIndexMask - (uint32_t)(best & kIndexMask));
      if (p.logprob) p.logprob[row] = best == 0ull ? -INFINITY : 0.f;
    }
    return;
  }
  const float top = from_rising((uint32_t)(best >> kIndexBits));
  Weights weight;
  weight.set(top, temperature, sh.powers);

  const int32_t k_given = p.top_k ? p.top_k[row] : 0;
  const uint32_t k = k_given > 0 && (uint32_t)k_given < p.vocab ? (uint32_t)k_given : 0u;
  const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
  const float u = p.uniform[row];
  uint64_t keep = 0;  // tokens at or after this are kept
  if (min_p > 0.f) {  // the least logit with t >= log2(min_p), by a search of one warp over the numbers' order
    if (warp == 0) {
      uint32_t lo = rising(-INFINITY), hi = rising(top);  // hi is kept
      if (min_p < 1.f && top < INFINITY) {
        const uint32_t b = __float_as_uint(min_p), e = b >> 23;
        const Pair edge = e ? log2_of((b & 0x7FFFFFu | 0x800000u) << 6, (int)e - 127, sh.powers) : log2_of((uint64_t)b, 149, sh.powers);
        while (lo < hi) {
          const uint32_t step = (hi - lo) / 33u + 1u;
          const uint32_t at = min(lo + (lane + 1u) * step - 1u, hi);  // rising over the lanes
          const float x = from_rising(at);
          const Pair t = weight.both(x);
          const bool in = at == hi || x == top || (!weight.none(x) && (t.hi - edge.hi) + (t.lo - edge.lo) >= 0.f);
          const uint32_t votes = __ballot_sync(kFull, in);
          const uint32_t first = votes ? __ffs(votes) - 1u : 32u;  // the first lane whose number is kept
          const uint32_t new_lo = first ? min(lo + first * step, hi) : lo;
          hi = first < 32u ? min(lo + (first + 1u) * step - 1u, hi) : hi;
          lo = new_lo;
        }
      } else {
        lo = hi;
      }
      if (lane == 0) sh.told[1] = hi;
    }
    __syncthreads();
    keep = sh.told[1] << kIndexBits;
    __syncthreads();
  }
  auto target_of = [&](uint64_t total) {
    if (!(u < 1.f)) return u >= 1.f ? total - 1u : 0ull;
    bool more;
    return u > 0.f ? times(u, total, more) : 0ull;  // below the total
  };
  auto answer = [&](uint32_t index, float x, uint64_t total) {
    p.token[row] = (int32_t)index;
    if (p.logprob) {  // ln 2 (t - log2(total / 2^45))
      const Pair sum = log2_of(total, kOne, sh.powers);
      const Pair t = x == top ? Pair{0.f, 0.f} : weight.both(x);
      const Pair d = exact_sum(t.hi, -sum.hi);
      const float low = d.lo + (t.lo - sum.lo), h = d.hi * kLn2;
      p.logprob[row] = h + fmaf(low, kLn2, fmaf(d.hi, kLn2Low, fmaf(d.hi, kLn2, -h)));
    }
  };

  // Bisection of the order: the last place before which less than `bound` (a weight, or a number) lies.
  auto before = [&](uint64_t order, bool count) {
    uint64_t v = 0, zero = 0;
    for (uint32_t i = tid; i < n; i += kThreads)
      if (order_of(xs[i], from + i) > order) v += count ? 1ull : weight(xs[i]);
    all2(v, zero, false, of);
    return v;
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
  // warps own consecutive pieces of the slice, a lane four consecutive logits of 128
  const uint32_t piece = (n + 4u * kThreads - 1u) / (4u * kThreads) * 128u, w0 = min(warp * piece, n), w1 = min(w0 + piece, n);
  auto read4 = [&](uint32_t i, uint32_t end, float (&x)[4]) {
    const float4 y = i < end ? *reinterpret_cast<const float4*>(xs + i) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
    x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;  // past the slice's end lies -inf
  };
  const bool p_on = top_p < 1.f;
  bool searched = !p_on && k == 0u;  // the border is known

  if (!searched && k != 0u && k <= kListK) {
    // ---- top-k: a bound from the threads' maxima, and a list -----------------------------------------------
    for (uint32_t i = tid; i < kKBins; i += kThreads) sh.k_bins[i] = 0u;
    __syncthreads();
    const float low = from_rising(~(uint32_t)lowest), span = top - low;
    // bins fall with x; equal logits, and infinite ones, are all in the first
    const float scale = span > 0.f && span < INFINITY ? (float)(kKBins - 1u) / span : 0.f;
    auto k_bin = [&](float x) { return scale == 0.f ? (x == top || span < INFINITY ? 0u : kKBins - 1u) : min((uint32_t)((top - x) * scale), kKBins - 1u); };
    if (mine > -INFINITY) atomicAdd(&sh.k_bins[k_bin(mine)], 1u);
    cluster_sync();
    uint32_t in_bin = 0;
    if (tid < kKBins)
      for (uint32_t r = 0; r < ctas; ++r) in_bin += load_remote(&sh.k_bins[tid], r);
    uint32_t upto = in_bin;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t o = __shfl_up_sync(kFull, upto, d);
      if (lane >= (uint32_t)d) upto += o;
    }
    if (lane == 31) sh.warps[turn][warp][0] = upto;
    __syncthreads();
    uint32_t earlier = 0;
    for (uint32_t i = 0; i < min(warp, kKBins / 32u); ++i) earlier += (uint32_t)sh.warps[turn][i][0];
    upto += earlier;
    if (tid == 0) sh.told[0] = kKBins - 1u;  // fewer maxima than k: nothing is left out
    __syncthreads();
    if (tid < kKBins && upto >= k && upto - in_bin < k) sh.told[0] = tid;
    __syncthreads();
    const uint32_t cut = (uint32_t)sh.told[0];
    // the same products as in k_bin, compared with the bin's end
    const float last_bin = scale == 0.f ? 0.f : (float)(cut + 1u);
    const bool all_bins = cut == kKBins - 1u;
    auto listed = [&](float x) { return x > -INFINITY && (all_bins || (scale == 0.f ? k_bin(x) <= cut : (top - x) * scale < last_bin)); };
    uint32_t count = 0;
    for (uint32_t i = w0 + 4u * lane; i < w1; i += 128u) {
      float x[4];
      read4(i, w1, x);
#pragma unroll
      for (int j = 0; j < 4; ++j) count += listed(x[j]) ? 1u : 0u;
    }
    uint64_t v = count, zero = 0;
    const uint32_t last = turn;
    all2(v, zero, false, of);  // (also: every CTA has read the bins, the list may lie over them)
    if (v <= kList) {
      // the list in the order of the vocabulary, in the first CTA
      uint32_t at = 0;
      for (uint32_t i = 0; i < rank; ++i) at += (uint32_t)of[i];
      for (uint32_t i = 0; i < warp; ++i) at += (uint32_t)sh.warps[last][i][0];
      for (uint32_t i0 = w0; i0 < w1; i0 += 128u) {
        const uint32_t i = i0 + 4u * lane;
        float x[4];
        read4(i, w1, x);
        uint32_t mask = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) mask |= listed(x[j]) ? 1u << j : 0u;
        if (!__any_sync(kFull, mask != 0u)) continue;
        const uint32_t own = __popc(mask);
        uint32_t upto = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const uint32_t o = __shfl_up_sync(kFull, upto, d);
          if (lane >= (uint32_t)d) upto += o;
        }
        uint32_t to = at + upto - own;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if ((mask >> j) & 1u) store_remote(&sh.list[to++], 0u, order_of(x[j], from + i + j));
        at += __shfl_sync(kFull, upto, 31);
      }
      cluster_sync();
      if (rank != 0) return;
      const uint32_t m = (uint32_t)v;
      constexpr uint32_t kEach = kList / kThreads;  // consecutive entries of a thread
      uint64_t own[kEach];                          // in the order of the vocabulary
#pragma unroll
      for (uint32_t i = 0; i < kEach; ++i) own[i] = tid * kEach + i < m ? sh.list[tid * kEach + i] : 0ull;
      __syncthreads();
      sort_list(sh.list, m, tid);
      // sums of weights over the threads' entries, and what is before them
      auto scan = [&](uint64_t sum, uint64_t& total) {
        uint64_t incl = sum;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const uint64_t o = __shfl_up_sync(kFull, incl, d);
          if (lane >= (uint32_t)d) incl += o;
        }
        __syncthreads();
        if (lane == 31) sh.warps[0][warp][0] = incl;
        __syncthreads();
        total = 0;
        uint64_t prev = 0;
        for (uint32_t i = 0; i < kWarps; ++i) {
          const uint64_t o = sh.warps[0][i][0];
          prev += i < warp ? o : 0ull;
          total += o;
        }
        return prev + incl - sum;
      };
      uint32_t kept = min(k, m);
      if (p_on) {
        uint64_t w[kEach], sum = 0, total;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
          const uint32_t j = tid * kEach + i;
          w[i] = j < kept ? weight(from_rising((uint32_t)(sh.list[j] >> kIndexBits))) : 0ull;
          sum += w[i];
        }
        uint64_t prev = scan(sum, total);
        const uint64_t bound = bound_of(top_p, total);
        uint32_t in = 0;
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
          in += tid * kEach + i < kept && prev < bound ? 1u : 0u;
          prev += w[i];
        }
        uint64_t sum_in;
        scan(in, sum_in);
        kept = max(1u, (uint32_t)sum_in);
      }
      const uint64_t edge = sh.list[kept - 1u];
      keep = min(max(keep, edge), best);
      uint64_t w[kEach], sum = 0, total;
#pragma unroll
      for (uint32_t i = 0; i < kEach; ++i) {
        w[i] = own[i] != 0ull && own[i] >= keep ? weight(from_rising((uint32_t)(own[i] >> kIndexBits))) : 0ull;
        sum += w[i];
      }
      uint64_t prev = scan(sum, total);
      const uint64_t target = target_of(total);
      if (target >= prev && target < prev + sum) {
#pragma unroll
        for (uint32_t i = 0; i < kEach; ++i) {
          if (target >= prev && target < prev + w[i])
            answer(kIndexMask - (uint32_t)(own[i] & kIndexMask), from_rising((uint32_t)(own[i] >> kIndexBits)), total);
          prev += w[i];
        }
      }
      return;
    }
  }
  if (!searched && k == 0u) {
    // ---- top-p: a histogram of the weights, and a list of the bin with the border -----------------------------
    for (uint32_t i = tid; i < kBins; i += kThreads) sh.bins.hi[i] = sh.bins.lo[i] = 0u;
    __syncthreads();
    uint64_t rest = 0;  // of the octaves below
    for (uint32_t i0 = w0; i0 < w1; i0 += 128u) {
      float x[4];
      read4(i0 + 4u * lane, w1, x);
      weight.four(x, [&](int, bool fine, int place, uint32_t v) {
        if (fine) {
          const uint32_t b = bin_of(place);
          atomicAdd(&sh.bins.hi[b], v >> 15);
          atomicAdd(&sh.bins.lo[b], v & 0x7FFFu);
        } else {
          rest += v;
        }
      });
    }
    cluster_sync();
    // this CTA's bins of all CTAs: kBins / ctas consecutive ones, up to three to a thread
    const uint32_t share = kBins / ctas, each = (share + kThreads - 1u) / kThreads, first = rank * share + tid * each;
    uint64_t mass[3] = {0, 0, 0}, sum = 0;
    for (uint32_t j = 0; j < each; ++j) {
      if (tid * each + j >= share) break;
      uint64_t hi = 0, lo = 0;
      for (uint32_t r = 0; r < ctas; ++r) {
        hi += load_remote(&sh.bins.hi[first + j], r);
        lo += load_remote(&sh.bins.lo[first + j], r);
      }
      const uint64_t m = ((hi << 15) + lo) << Weights::shift(-1 - 4 * (int)(first + j));
      if (j == 0) mass[0] = m;
      if (j == 1) mass[1] = m;
      if (j == 2) mass[2] = m;
      sum += m;
    }
    uint64_t total = sum, all_rest = rest;
    const uint32_t last = turn;
    uint64_t incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint64_t o = __shfl_up_sync(kFull, incl, d);
      if (lane >= (uint32_t)d) incl += o;
    }
    if (tid == 0) sh.told[0] = ~0ull;
    all2(total, all_rest, false, of);
    const uint64_t bound = bound_of(top_p, total + all_rest);
    uint64_t prev = incl - sum;
    for (uint32_t i = 0; i < rank; ++i) prev += of[i];
    for (uint32_t i = 0; i < warp; ++i) prev += sh.warps[last][i][0];
    if (bound != 0ull) {
#pragma unroll
      for (uint32_t j = 0; j < 3u; ++j) {
        if (j < each && mass[j] != 0ull && prev < bound && prev + mass[j] >= bound) {
          for (uint32_t r = 0; r < ctas; ++r) {
            store_remote(&sh.told[0], r, first + j);
            store_remote(&sh.told[1], r, prev);
          }
        }
        prev += mass[j];
      }
    }
    cluster_sync();  // (also: every CTA has read the bins, the list may lie over them)
    const uint64_t bin = sh.told[0], ahead = sh.told[1];
    if (bound == 0ull) {
      keep = best;
      searched = true;
    } else if (bin != ~0ull) {
      // the bin's logits lie between these, give or take the roundings of fp32: only there is the bin looked at
      const float t_hi = (float)bin * -0.015625f, t_lo = t_hi - 0.015625f;
      for (uint32_t i0 = w0; i0 < w1; i0 += 128u) {
        const uint32_t i = i0 + 4u * lane;
        float x[4];
        read4(i, w1, x);
        uint32_t mask = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (weight.none(x[j])) continue;
          const float t = weight.coarse(x[j]);
          if (t < t_lo - 0.01f || t > t_hi + 0.01f || t < -(float)kOctaves) continue;  // (a place is rounded to 1/256)
          int place;
          weight.fine(x[j], place);
          if (bin_of(place) == (uint32_t)bin) mask |= 1u << j;
        }
        if (!__any_sync(kFull, mask != 0u)) continue;
        const uint32_t own = __popc(mask);
        uint32_t upto = own;
#pragma unroll
        for (int d = 1; d < 32; d <<= 1) {
          const uint32_t o = __shfl_up_sync(kFull, upto, d);
          if (lane >= (uint32_t)d) upto += o;
        }
        uint32_t at = 0;
        if (lane == 31) at = add_remote(&sh.listed, 0u, upto);
        at = __shfl_sync(kFull, at, 31) + upto - own;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (!((mask >> j) & 1u)) continue;
          if (at < kList) store_remote(&sh.list[at], 0u, order_of(x[j], from + i + j));
          ++at;
        }
      }
      cluster_sync();
      const uint32_t m = load_remote(&sh.listed, 0u);
      if (m <= kList) {
        if (rank == 0) {
          sort_list(sh.list, m, tid);
          // the last entry before which less than the bound lies
          constexpr uint32_t kEach = kList / kThreads;
          uint64_t w[kEach], sum = 0, incl;
#pragma unroll
          for (uint32_t i = 0; i < kEach; ++i) {
            const uint32_t j = tid * kEach + i;
            w[i] = j < m ? weight(from_rising((uint32_t)(sh.list[j] >> kIndexBits))) : 0ull;
            sum += w[i];
          }
          incl = sum;
#pragma unroll
          for (int d = 1; d < 32; d <<= 1) {
            const uint64_t o = __shfl_up_sync(kFull, incl, d);
            if (lane >= (uint32_t)d) incl += o;
          }
          if (lane == 31) sh.warps[turn][warp][0] = incl;
          __syncthreads();
          uint64_t prev = ahead + incl - sum;
          for (uint32_t i = 0; i < warp; ++i) prev += sh.warps[turn][i][0];
#pragma unroll
          for (uint32_t i = 0; i < kEach; ++i) {
            const uint32_t j = tid * kEach + i;
            if (j < m && prev < bound && (j + 1u == m || prev + w[i] >= bound)) {
              for (uint32_t r = 0; r < ctas; ++r) store_remote(&sh.told[0], r, sh.list[j]);
            }
            prev += w[i];
          }
          __syncthreads();
        }
        cluster_sync();
        keep = min(max(keep, sh.told[0]), best);
        searched = true;
      }
    }
  }
  if (!searched) {
    uint64_t edge = 0;
    if (k != 0u) edge = border(k, true, 0ull);
    if (p_on) {
      const uint64_t sum = before(edge ? edge - 1u : 0u, false);  // 0 is no token's place
      edge = border(bound_of(top_p, sum), false, edge);
    }
    keep = max(keep, edge);
  }
  keep = min(keep, best);

  // ---- the token up to which more than u of the kept sum lies ---------------------------------------
  const float keep_x = from_rising((uint32_t)(keep >> kIndexBits));  // below it nothing is kept
  // weights of four logits, 0 where they are not kept
  auto kept = [&](uint32_t i, uint64_t (&w)[4]) {
    float x[4];
    read4(i, w1, x);
    bool any = false;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (x[j] < keep_x || order_of(x[j], from + i + j) < keep) x[j] = -INFINITY;
      any = any || x[j] > -INFINITY;
      w[j] = 0ull;
    }
    if (!__any_sync(kFull, any)) return;
    weight.four(x, [&](int j, bool fine, int place, uint32_t v) { w[j] = fine ? (uint64_t)v << Weights::shift(place) : v; });
  };
  uint64_t sum_mine = 0, zero = 0;
  for (uint32_t i0 = w0; i0 < w1; i0 += 128u) {
    uint64_t w[4];
    kept(i0 + 4u * lane, w);
    sum_mine += w[0] + w[1] + w[2] + w[3];
  }
  const uint32_t last = turn;
  all2(sum_mine, zero, false, of);
  const uint64_t total = sum_mine, target = target_of(total);
  uint64_t sum = 0;
  for (uint32_t i = 0; i < rank; ++i) sum += of[i];
  for (uint32_t i = 0; i < warp; ++i) sum += sh.warps[last][i][0];
  if (target < sum || target >= sum + sh.warps[last][warp][0]) return;  // another warp has it
  for (uint32_t i0 = w0; i0 < w1; i0 += 128u) {
    const uint32_t i = i0 + 4u * lane;
    uint64_t w[4];
    kept(i, w);
    const uint64_t own = w[0] + w[1] + w[2] + w[3];
    uint64_t upto = own;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint64_t o = __shfl_up_sync(kFull, upto, d);
      if (lane >= (uint32_t)d) upto += o;
    }
    const uint32_t past = __ballot_sync(kFull, sum + upto > target);
    if (past) {
      if (lane == __ffs(past) - 1u) {
        sum += upto - own;
        uint32_t j = 0;
        while (j < 3u && sum + w[j] <= target) sum += w[j++];
        answer(from + i + j, xs[i + j], total);
      }
      return;
    }
    sum += __shfl_sync(kFull, upto, 31);
  }
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
  constexpr size_t kHead = (sizeof(Shared) + 15u) / 16u * 16u;
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
