// One token for each row of logits (tq_sample): temperature, top-k, top-p, min-p, and the inverse of the distribution
// function at a given uniform number.
//
// Exact sums.  Every decision is a comparison of sums of weights w = 2^t, t = (x - max) log2(e) / temperature, with a bound: a
// weight is therefore an integer W = round(2^40 w), and sums of up to 2^18 of them are exact in 64 bits whatever their
// order.  t comes from one fp64 fused multiply-add onto 1.5 * 2^20, whose last bit is 2^-32: the low word of the result
// is the fraction of t and the high word its integer part.  2^fraction = table[upper 8 bits] * (1 + q), q a cubic in the lower 24.
//
// Order.  Tokens fall by (x, lower index first): as one integer, the logit's bits made to rise with it above the index turned
// round.  What is kept is all that is not below a border in that order, so every filter is a search for its border.
//
// A row is read once: a cluster of up to eight CTAs holds it in shared memory.
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
constexpr int kOne = 40;  // W of the largest logit is 2^40

// 2^(i / 256) with 30 bits behind the point
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
    p.v[i] = (uint32_t)(sum * 1073741824.0 + 0.5);
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
};

struct Shared {
  uint64_t slots[2][kMaxCluster];  // what the cluster's CTAs tell one another; two sets, used in turn
  uint64_t warps[2][kWarps];
  uint32_t powers[256];
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
__device__ __forceinline__ void store_remote(uint64_t* at, uint32_t rank, uint64_t v) {
  uint32_t a;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(tq_sm100::smem_u32(at)), "r"(rank));
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}

// Bits that rise with the number (no NaN, no -0).
__device__ __forceinline__ uint32_t rising(float x) {
  const uint32_t b = __float_as_uint(x);
  return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ uint64_t order_of(float x, uint32_t index) { return ((uint64_t)rising(x) << kIndexBits) | (kIndexMask - index); }

struct Weights {
  float top, c32;  // largest logit; log2(e) / temperature
  double c;
  const uint32_t* powers;

  __device__ __forceinline__ uint64_t operator()(float x) const {
    if (x == top) return 1ull << kOne;
    if (x == -INFINITY || top == INFINITY || (x - top) * c32 < -42.f) return 0ull;  // below half a unit
    const double z = fma((double)x - (double)top, c, 1572864.0);  // 1.5 * 2^20
    const int n = min(0, __double2hiint(z) - 0x41380000);         // t = n + fraction
    const uint32_t f = (uint32_t)__double2loint(z);
    const uint32_t base = powers[f >> 24];
    const float r = __uint_as_float(0x3F800000u | ((f & 0xFFFFFFu) >> 1)) - 1.0f;  // the lower 24 bits, 0 .. 1
    constexpr float a1 = 2.7076061740622863e-3f, a2 = 3.6655656e-6f, a3 = 3.3082868e-9f;  // (ln 2 / 256)^k / k!
    const float q = r * fmaf(r, fmaf(r, a3, a2), a1);
    const uint32_t add = __float_as_uint(fmaf((float)base, q, 8388608.0f)) - 0x4B000000u;  // rounded to whole units of 2^-30
    const uint64_t v = (uint64_t)(base + add);
    const int up = kOne - 30 + n;
    const uint64_t w = up >= 0 ? v << up : (v + (1ull << (-up - 1))) >> -up;
    return n == 0 ? 1ull << kOne : w;  // t rounded to 0
  }
};

template <int TYPE>
__global__ void __launch_bounds__(kThreads) sample_kernel(const SampleParams p) {
  extern __shared__ __align__(16) uint8_t smem[];
  Shared& sh = *reinterpret_cast<Shared*>(smem);
  float* const xs = reinterpret_cast<float*>(smem + sizeof(Shared));
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u, rank = cluster_rank(), ctas = cluster_size();
  const uint32_t row = blockIdx.x / ctas, from = min(rank * p.slice, p.vocab), n = min(p.slice, p.vocab - from);
  if (tid < 256) sh.powers[tid] = kPowers.v[tid];
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");

  uint32_t turn = 0;
  // Adds (or takes the largest of) every thread's value over the cluster; of[r]: what CTA r had.
  auto all = [&](uint64_t v, bool largest, uint64_t (&of)[kMaxCluster]) -> uint64_t {
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      const uint64_t o = __shfl_xor_sync(kFull, v, d);
      v = largest ? (o > v ? o : v) : v + o;
    }
    if (lane == 0) sh.warps[turn][warp] = v;
    __syncthreads();
    if (warp == 0) {
      v = lane < kWarps ? sh.warps[turn][lane] : 0ull;
#pragma unroll
      for (int d = 16; d > 0; d >>= 1) {
        const uint64_t o = __shfl_xor_sync(kFull, v, d);
        v = largest ? (o > v ? o : v) : v + o;
      }
      if (lane < ctas) store_remote(&sh.slots[turn][rank], lane, v);
    }
    cluster_sync();
    uint64_t r = 0;
    for (uint32_t i = 0; i < kMaxCluster; ++i) {
      of[i] = i < ctas ? sh.slots[turn][i] : 0ull;
      r = largest ? (of[i] > r ? of[i] : r) : r + of[i];
    }
    turn ^= 1u;
    return r;
  };
  uint64_t of[kMaxCluster];

  // ---- the row, and its first token in falling order -----------------------------------------------
  uint64_t best = 0;
  for (uint32_t i = tid; i < n; i += kThreads) {
    float x = load1<TYPE>(p.logits, (size_t)((int64_t)row * p.row_stride) + from + i);
    x = x != x ? -INFINITY : x + 0.f;  // -0 is 0
    xs[i] = x;
    const uint64_t o = order_of(x, from + i);
    best = o > best ? o : best;
  }
  asm volatile("barrier.cluster.wait.aligned;" ::: "memory");  // every CTA of the cluster runs: its shared memory can be written
  best = all(best, true, of);
  const uint32_t first = kIndexMask - (uint32_t)(best & kIndexMask);
  const uint32_t bits = (uint32_t)(best >> kIndexBits);
  const float top = __uint_as_float(bits ^ (bits >> 31 ? 0x80000000u : 0xFFFFFFFFu));
  const float temperature = p.temperature ? p.temperature[row] : 1.f;
  if (top == -INFINITY || !(temperature > 0.f)) {
    if (rank == 0 && tid == 0) {
      p.token[row] = top == -INFINITY ? -1 : (int32_t)first;
      if (p.logprob) p.logprob[row] = top == -INFINITY ? -INFINITY : 0.f;
    }
    return;
  }
  Weights weight;
  weight.top = top;
  weight.c = 1.4426950408889634074 / (double)temperature;
  weight.c32 = (float)weight.c;
  weight.powers = sh.powers;

  // Weight (or number) of the tokens that stand before `order`.
  auto before = [&](uint64_t order, bool count) {
    uint64_t v = 0;
    for (uint32_t i = tid; i < n; i += kThreads)
      if (order_of(xs[i], from + i) > order) v += count ? 1ull : weight(xs[i]);
    return all(v, false, of);
  };
  // The last place in the order before which less than `bound` lies.
  auto border = [&](double bound, bool count, uint64_t lo) {
    uint64_t hi = best;  // nothing is before it
    while (lo < hi) {
      const uint64_t mid = lo + (hi - lo) / 2u;
      if ((double)before(mid, count) < bound)
        hi = mid;
      else
        lo = mid + 1u;
    }
    return hi;
  };

  uint64_t keep = 0;  // tokens at or after this are kept
  const int32_t k = p.top_k ? p.top_k[row] : 0;
  if (k > 0 && (uint32_t)k < p.vocab) keep = border((double)k, true, keep);
  const float top_p = p.top_p ? p.top_p[row] : 1.f;
  if (top_p < 1.f) {
    const uint64_t sum = before(keep ? keep - 1u : 0u, false);  // 0 is no token's place
    keep = border((double)top_p * (double)sum, false, keep);
  }
  const float min_p = p.min_p ? p.min_p[row] : 0.f;
  if (min_p > 0.f) {
    const double edge = (double)top + (double)temperature * log((double)min_p);
    const float x = min_p >= 1.f || top == INFINITY ? top : fminf(__double2float_ru(edge), top);
    const uint64_t o = (uint64_t)rising(x + 0.f) << kIndexBits;
    keep = o > keep ? o : keep;
    keep = keep > best ? best : keep;
  }

  // ---- the token up to which more than u of the kept sum lies ---------------------------------------
  // warps own consecutive pieces of the slice
  const uint32_t piece = (n + kThreads - 1u) / kThreads * 32u, w0 = min(warp * piece, n), w1 = min(w0 + piece, n);
  auto kept = [&](uint32_t i) { return order_of(xs[i], from + i) >= keep ? weight(xs[i]) : 0ull; };
  uint64_t mine = 0;
  for (uint32_t i = w0 + lane; i < w1; i += 32u) mine += kept(i);
  const uint32_t last = turn;
  const uint64_t total = all(mine, false, of);
  const float u = p.uniform[row];
  uint64_t target = (uint64_t)((u > 0.f ? (double)u : 0.0) * (double)total);
  target = target < total ? target : total - 1u;
  uint64_t sum = 0;
  for (uint32_t i = 0; i < rank; ++i) sum += of[i];
  for (uint32_t i = 0; i < warp; ++i) sum += sh.warps[last][i];
  if (target < sum || target >= sum + sh.warps[last][warp]) return;  // another warp has it
  for (uint32_t i0 = w0; i0 < w1; i0 += 32u) {
    const uint32_t i = i0 + lane;
    const uint64_t w = i < w1 ? kept(i) : 0ull;
    uint64_t upto = w;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint64_t o = __shfl_up_sync(kFull, upto, d);
      if (lane >= (uint32_t)d) upto += o;
    }
    const uint32_t past = __ballot_sync(kFull, sum + upto > target);
    if (past) {
      if (lane == __ffs(past) - 1u) {
        p.token[row] = (int32_t)(from + i);
        if (p.logprob) {
          const double t = top == INFINITY ? 0.0 : ((double)xs[i] - (double)top) / (double)temperature;
          p.logprob[row] = (float)(t - (log((double)total) - kOne * 0.69314718055994530942));
        }
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
  p.slice = ((p.vocab + ctas - 1u) / ctas + 3u) / 4u * 4u;
  const char* what = "sample launch";
  if (int rc = tq_ensure_dynamic_smem((const void*)kern, sizeof(Shared) + TQ_SAMPLE_MAX_VOCAB / kMaxCluster * sizeof(float), what)) return rc;
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = dim3(rows * ctas);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = sizeof(Shared) + p.slice * sizeof(float);
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
