// Rotary positions of new tokens and the write of their keys and values to the cache (tq_rope_append), with the norm of every
// query and key head before it (tq_qk_norm_rope_append).
//
// Pair i of a head, (a, b) -> (a cos - b sin, a sin + b cos), with the cosine and sine of table row p,
// p the position on the pair's axis.  The pairs of a head are independent of one another: a thread owns
// four pairs (eight elements) of the heads it visits, loads their eight cosines and sines once per token
// and reuses them over the token's query and key heads.  8 to 16 bytes move per two or three operations:
// memory bound for prompts, latency for a decode step.
//
// Norm: the D / 8 lanes that have a head add its squares up by shuffles, and a thread keeps the eight weights of its elements,
// from its first key on those of keys (both sets at once, and a choice for every element: 23.2 us).  Eight multiplications and four shuffles
// an element group more on a path that waits for memory: 2047 tokens of 64 + 8 heads of 128 in bf16 take 20.8 us (their bytes: 12.8), 32 tokens of 24 + 8 in fp32 2.2 us.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "tq_internal.h"
#include "tq_ops_common.cuh"

namespace {

using namespace tq_ops;

constexpr uint32_t kRopeThreads = 256;

struct RopeParams {
  const void* q;
  const void* k;
  const void* v;
  int64_t q_stride, k_stride, v_stride;
  const float* table;
  const int32_t* positions;
  const int32_t* slots;
  __nv_bfloat16* q_out;
  tq_kv_cache cache;
  uint32_t n_tokens, n_q_heads, n_positions, rot_dim;
  uint32_t axis_end[TQ_ROPE_MAX_AXES];  // first pair past each axis' section
  uint32_t n_axes;
  const float* q_weight;  // norm of the heads
  const float* k_weight;
  float eps;
  bool weights_16;  // they may be read 16 bytes at a time
};

// Eight elements of a head as two runs of four, so that neighbouring lanes read neighbouring runs whatever the type and the
// order of the pairs (eight consecutive fp32 to a lane in two accesses would touch every sector twice).
template <int TYPE>
struct Raw4x2 {
  uint4 a, b;
  __device__ __forceinline__ void load(const void* base, size_t i, size_t j) {
    if constexpr (TYPE == TQ_TYPE_F32) {
      a = load_once((const float*)base + i);
      b = load_once((const float*)base + j);
    } else {
      const uint2 x = *reinterpret_cast<const uint2*>((const __nv_bfloat16*)base + i);
      const uint2 y = *reinterpret_cast<const uint2*>((const __nv_bfloat16*)base + j);
      a = make_uint4(x.x, x.y, 0, 0);
      b = make_uint4(y.x, y.y, 0, 0);
    }
  }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    if constexpr (TYPE == TQ_TYPE_F32) {
      f[0] = __uint_as_float(a.x), f[1] = __uint_as_float(a.y), f[2] = __uint_as_float(a.z), f[3] = __uint_as_float(a.w);
      f[4] = __uint_as_float(b.x), f[5] = __uint_as_float(b.y), f[6] = __uint_as_float(b.z), f[7] = __uint_as_float(b.w);
    } else {
      f[0] = bf16_lo(a.x), f[1] = bf16_hi(a.x), f[2] = bf16_lo(a.y), f[3] = bf16_hi(a.y);
      f[4] = bf16_lo(b.x), f[5] = bf16_hi(b.x), f[6] = bf16_lo(b.y), f[7] = bf16_hi(b.y);
    }
  }
};

// grid (tokens, parts of the heads); the 256 threads are 256 / (D / 8) heads side by side.
template <int TYPE, bool INTERLEAVED, int D, bool NORM>
__global__ void __launch_bounds__(kRopeThreads) rope_append_kernel(const RopeParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr uint32_t kPerHead = D / 8, kSide = kRopeThreads / kPerHead;
  const uint32_t j = threadIdx.x % kPerHead, t = blockIdx.x;
  const uint32_t pairs = p.rot_dim / 2u;
  // where this thread's two runs lie, the first pair of each two of its four, and whether the runs turn
  uint32_t e0, e1, pair_a, pair_b;
  bool turn_a, turn_b;
  if (INTERLEAVED) {  // two pairs to a run
    e0 = 4u * j;
    e1 = D / 2u + 4u * j;
    pair_a = e0 / 2u;
    pair_b = e1 / 2u;
    turn_a = e0 < p.rot_dim;
    turn_b = e1 < p.rot_dim;
  } else {  // first and second members of four pairs, or eight elements past the pairs
    turn_a = turn_b = 4u * j < pairs;
    e0 = turn_a ? 4u * j : 8u * j;
    e1 = turn_a ? pairs + 4u * j : e0 + 4u;
    pair_a = 4u * j;
    pair_b = pair_a + 2u;
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");

  const int32_t slot = p.slots[t];
  uint32_t pos[TQ_ROPE_MAX_AXES];
  bool known = true;
#pragma unroll
  for (uint32_t a = 0; a < TQ_ROPE_MAX_AXES; ++a) {
    pos[a] = a < p.n_axes ? (uint32_t)p.positions[(size_t)a * p.n_tokens + t] : 0u;
    known = known && pos[a] < p.n_positions;
  }

  // With the norm, whose reduction takes its time, the next head is under way during it, and of bf16 the one after that too (2047 tokens of 64 / 8
  // heads of 128, us, one | two under way: bf16 21.6 | 20.8, 32 / 8 heads 16.3 | 15.2; fp32, whose second one costs a block an SM, 22.2 | 26.9).
  constexpr bool kAhead = NORM && TYPE == TQ_TYPE_BF16;
  // Heads in order: queries, keys, values.  The first head is asked for before the cosines and sines, which wait for the
  // positions, and whether the token has a slot is not waited for either.  (Two or three heads of a thread under way: 15.5 and 14.1 us for 2047 tokens of 32 / 8 fp32 heads of 128, one:
  // 13.9.)
  const uint32_t H = p.n_q_heads, K = p.cache.n_kv_heads, heads = H + 2u * K, step = gridDim.y * kSide;
  const size_t tq = (size_t)t * p.q_stride + e0, tk = (size_t)t * p.k_stride + e0, tv = (size_t)t * p.v_stride + e0;
  const uint32_t gap = e1 - e0;
  Raw4x2<TYPE> raw, next;
  auto load = [&](uint32_t n, Raw4x2<TYPE>& to) {
    if (n >= heads) return;
    const void* src = n < H ? p.q : (n < H + K ? p.k : p.v);
    const size_t at = (n < H ? tq : (n < H + K ? tk : tv)) + (n < H ? n : (n < H + K ? n - H : n - H - K)) * D;
    to.load(src, at, at + gap);
  };
  uint32_t n = blockIdx.y * kSide + threadIdx.x / kPerHead;
  load(n, raw);
  if (kAhead) load(n + step, next);

  const uint32_t page = (uint32_t)slot / p.cache.page_size;  // -1: no slot; other negative ones are out of range like those past the pool
  const bool in_pool = slot >= 0 && page < p.cache.n_pages, keep = in_pool && known;
  if (threadIdx.x == 0 && blockIdx.y == 0 && p.cache.d_status != nullptr) {
    const uint32_t bad = (known ? 0u : TQ_STATUS_BAD_POSITION) | (slot != -1 && !in_pool ? TQ_STATUS_BAD_PAGE : 0u);
    if (bad) atomicOr(p.cache.d_status, bad);
  }
  const size_t slot_at = keep ? (size_t)page * p.cache.page_stride + (size_t)((uint32_t)slot - page * p.cache.page_size) * p.cache.slot_stride + e0 : 0;

  float w[NORM ? 8 : 1];  // of the queries, from the first key on of the keys
  bool keys = n >= H;
  auto weights = [&](const float* from) {
    if (p.weights_16) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(from + e0)), b = __ldg(reinterpret_cast<const float4*>(from + e1));
      w[0] = a.x, w[1] = a.y, w[2] = a.z, w[3] = a.w, w[4] = b.x, w[5] = b.y, w[6] = b.z, w[7] = b.w;
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) w[i] = __ldg(from + (i < 4 ? e0 : e1 - 4u) + i);
    }
  };
  if constexpr (NORM) weights(keys ? p.k_weight : p.q_weight);

  float cs[4], sn[4];
#pragma unroll
  for (uint32_t i = 0; i < 4; ++i) {
    cs[i] = known ? 1.f : __int_as_float(0x7FC00000);
    sn[i] = 0.f;
    if (!known || !(i < 2 ? turn_a : turn_b)) continue;
    const uint32_t pair = i < 2 ? pair_a + i : pair_b + i - 2u;
    const uint32_t at = pair < p.axis_end[0] ? pos[0] : (pair < p.axis_end[1] ? pos[1] : pos[2]);
    const float* row = p.table + (size_t)at * p.rot_dim + pair;
    cs[i] = __ldg(row);
    sn[i] = __ldg(row + pairs);
  }

  for (; n < heads && (n < H || keep); n += step) {
    float f[8];
    raw.get(f);
    if (kAhead) {
      raw = next;
      load(n + 2u * step, next);
    } else if (NORM) {
      load(n + step, raw);
    }
    if constexpr (NORM) {
      if (n >= H && !keys) {
        weights(p.k_weight);
        keys = true;
      }
      if (n < H + K) {
        float sum = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) sum += f[i] * f[i];
        // the lanes of one head take the same way through this loop, those of the warp's other heads need not
        const uint32_t mine = ((1u << kPerHead) - 1u) << (threadIdx.x % 32u / kPerHead * kPerHead);
#pragma unroll
        for (uint32_t d = kPerHead / 2u; d > 0; d >>= 1) sum += __shfl_xor_sync(mine, sum, d);
        const float r = rsqrtf(sum * (1.f / D) + p.eps);
#pragma unroll
        for (int i = 0; i < 8; ++i) f[i] = f[i] * r * w[i];
      }
    }
    if (n < H + K && (turn_a || turn_b || !known)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!(i < 2 ? turn_a : turn_b) && known) continue;
        float& x = INTERLEAVED ? f[2 * i] : f[i];
        float& y = INTERLEAVED ? f[2 * i + 1] : f[4 + i];
        const float a = x * cs[i] - y * sn[i], b = x * sn[i] + y * cs[i];
        x = a;
        y = b;
      }
    }
    __nv_bfloat16* dst = n < H ? p.q_out + ((size_t)t * H + n) * D + e0
                               : (n < H + K ? (__nv_bfloat16*)p.cache.d_k + slot_at + (size_t)(n - H) * p.cache.head_stride
                                            : (__nv_bfloat16*)p.cache.d_v + slot_at + (size_t)(n - H - K) * p.cache.head_stride);
    const uint4 o = pack8(f);
    *reinterpret_cast<uint2*>(dst) = make_uint2(o.x, o.y);
    *reinterpret_cast<uint2*>(dst + gap) = make_uint2(o.z, o.w);
    if (!NORM) load(n + step, raw);
  }
}

template <int TYPE, bool INTERLEAVED, bool NORM>
int launch(const RopeParams& p, cudaStream_t st) {
  const uint32_t side = kRopeThreads / (p.cache.head_dim / 8u), heads = p.n_q_heads + 2u * p.cache.n_kv_heads;
  // few tokens: a block for every set of heads; many: one block walks all heads of its token and keeps
  // the cosines and sines
  const uint32_t parts = p.n_tokens < 2u * (uint32_t)sm_count() ? (heads + side - 1u) / side : 1u;
  const dim3 grid(p.n_tokens, parts);
  const char* what = NORM ? "qk_norm_rope_append launch" : "rope_append launch";
  return p.cache.head_dim == 64 ? launch_pdl(rope_append_kernel<TYPE, INTERLEAVED, 64, NORM>, grid, kRopeThreads, 0, st, what, p)
                                : launch_pdl(rope_append_kernel<TYPE, INTERLEAVED, 128, NORM>, grid, kRopeThreads, 0, st, what, p);
}

template <bool NORM>
int rope(const void* d_q, const void* d_k, const void* d_v, int x_type, int64_t q_stride, int64_t k_stride, int64_t v_stride,
         uint32_t n_tokens, uint32_t n_q_heads, const float* d_q_weight, const float* d_k_weight, float eps, const float* d_table,
         uint32_t n_positions, uint32_t rot_dim, const int32_t* d_positions, const uint32_t* sections, uint32_t n_axes,
         int interleaved, const int32_t* d_slots, const tq_kv_cache* cache, void* d_q_out, void* cuda_stream) {
  if (int rc = tq_check_cache(cache)) return rc;
  if (x_type != TQ_TYPE_BF16 && x_type != TQ_TYPE_F32) return TQ_ERR_INVALID_ARG;
  if (!sections || n_axes == 0 || n_axes > TQ_ROPE_MAX_AXES || rot_dim == 0 || rot_dim % 8u || rot_dim > cache->head_dim) return TQ_ERR_INVALID_ARG;
  RopeParams p{};
  uint64_t end = 0;
  for (uint32_t a = 0; a < n_axes; ++a) {
    end += sections[a];
    if (end > rot_dim / 2u) return TQ_ERR_INVALID_ARG;
    p.axis_end[a] = (uint32_t)end;
  }
  for (uint32_t a = n_axes; a < TQ_ROPE_MAX_AXES; ++a) p.axis_end[a] = p.axis_end[n_axes - 1];
  if (end != rot_dim / 2u) return TQ_ERR_INVALID_ARG;
  if (NORM && !(eps >= 0.f)) return TQ_ERR_INVALID_ARG;
  if (n_tokens > 0x7FFFFFFFu || n_q_heads > 65536u) return TQ_ERR_UNSUPPORTED_SHAPE;
  if (n_tokens == 0) return TQ_OK;
  auto bad = [](const void* ptr, uintptr_t align) { return ptr == nullptr || ((uintptr_t)ptr & (align - 1u)) != 0; };
  if (bad(d_q, 16) || bad(d_k, 16) || bad(d_v, 16) || bad(d_table, 4) || bad(d_positions, 4) || bad(d_slots, 4) || bad(d_q_out, 16)) return TQ_ERR_INVALID_ARG;
  if (NORM && (bad(d_q_weight, 4) || bad(d_k_weight, 4))) return TQ_ERR_INVALID_ARG;
  if (n_q_heads == 0 || n_positions == 0 || q_stride % 8 || k_stride % 8 || v_stride % 8) return TQ_ERR_INVALID_ARG;
  p.q = d_q;
  p.k = d_k;
  p.v = d_v;
  p.q_stride = q_stride;
  p.k_stride = k_stride;
  p.v_stride = v_stride;
  p.table = d_table;
  p.positions = d_positions;
  p.slots = d_slots;
  p.q_out = (__nv_bfloat16*)d_q_out;
  p.cache = *cache;
  p.n_tokens = n_tokens;
  p.n_q_heads = n_q_heads;
  p.n_positions = n_positions;
  p.rot_dim = rot_dim;
  p.n_axes = n_axes;
  p.q_weight = d_q_weight;
  p.k_weight = d_k_weight;
  p.eps = eps;
  p.weights_16 = (((uintptr_t)d_q_weight | (uintptr_t)d_k_weight) & 15u) == 0;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (x_type == TQ_TYPE_F32) return interleaved ? launch<TQ_TYPE_F32, true, NORM>(p, st) : launch<TQ_TYPE_F32, false, NORM>(p, st);
  return interleaved ? launch<TQ_TYPE_BF16, true, NORM>(p, st) : launch<TQ_TYPE_BF16, false, NORM>(p, st);
}

}  // namespace

extern "C" {

int tq_rope_append(const void* d_q, const void* d_k, const void* d_v, int x_type, int64_t q_stride, int64_t k_stride,
                   int64_t v_stride, uint32_t n_tokens, uint32_t n_q_heads, const float* d_table, uint32_t n_positions,
                   uint32_t rot_dim, const int32_t* d_positions, const uint32_t* sections, uint32_t n_axes,
                   int interleaved, const int32_t* d_slots, const tq_kv_cache* cache, void* d_q_out,
                   void* cuda_stream) {
  return rope<false>(d_q, d_k, d_v, x_type, q_stride, k_stride, v_stride, n_tokens, n_q_heads, nullptr, nullptr, 0.f, d_table,
                     n_positions, rot_dim, d_positions, sections, n_axes, interleaved, d_slots, cache, d_q_out, cuda_stream);
}

int tq_qk_norm_rope_append(const void* d_q, const void* d_k, const void* d_v, int x_type, int64_t q_stride, int64_t k_stride,
                           int64_t v_stride, uint32_t n_tokens, uint32_t n_q_heads, const float* d_q_weight,
                           const float* d_k_weight, float eps, const float* d_table, uint32_t n_positions, uint32_t rot_dim,
                           const int32_t* d_positions, const uint32_t* sections, uint32_t n_axes, int interleaved,
                           const int32_t* d_slots, const tq_kv_cache* cache, void* d_q_out, void* cuda_stream) {
  return rope<true>(d_q, d_k, d_v, x_type, q_stride, k_stride, v_stride, n_tokens, n_q_heads, d_q_weight, d_k_weight, eps, d_table,
                    n_positions, rot_dim, d_positions, sections, n_axes, interleaved, d_slots, cache, d_q_out, cuda_stream);
}

}  // extern "C"
