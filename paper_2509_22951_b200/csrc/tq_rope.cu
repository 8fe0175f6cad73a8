// Rotary positions of new tokens and the write of their keys and values to the cache (tq_rope_append).
//
// Pair i of a head, (a, b) -> (a cos - b sin, a sin + b cos), with the cosine and sine of table row p,
// p the position on the pair's axis.  The pairs of a head are independent of one another: a thread owns
// four pairs (eight elements) of the heads it visits, loads their eight cosines and sines once per token
// and reuses them over the token's query and key heads.  8 to 16 bytes move per two or three operations:
// memory bound for prompts, latency for a decode step.
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
template <int TYPE, bool INTERLEAVED, int D>
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

  // Heads in order: queries, keys, values.  The first head is asked for before the cosines and sines, which wait for the
  // positions, and whether the token has a slot is not waited for either.  (Two or three heads of a thread under way: 15.5 and 14.1 us for 2047 tokens of 32 / 8 fp32 heads of 128, one:
  // 13.9.)
  const uint32_t H = p.n_q_heads, K = p.cache.n_kv_heads, heads = H + 2u * K, step = gridDim.y * kSide;
  const size_t tq = (size_t)t * p.q_stride + e0, tk = (size_t)t * p.k_stride + e0, tv = (size_t)t * p.v_stride + e0;
  const uint32_t gap = e1 - e0;
  Raw4x2<TYPE> raw;
  auto load = [&](uint32_t n) {
    if (n >= heads) return;
    const void* src = n < H ? p.q : (n < H + K ? p.k : p.v);
    const size_t at = (n < H ? tq : (n < H + K ? tk : tv)) + (n < H ? n : (n < H + K ? n - H : n - H - K)) * D;
    raw.load(src, at, at + gap);
  };
  uint32_t n = blockIdx.y * kSide + threadIdx.x / kPerHead;
  load(n);

  const uint32_t page = (uint32_t)slot / p.cache.page_size;  // -1: no slot; other negative ones are out of range like those past the pool
  const bool in_pool = slot >= 0 && page < p.cache.n_pages, keep = in_pool && known;
  if (threadIdx.x == 0 && blockIdx.y == 0 && p.cache.d_status != nullptr) {
    const uint32_t bad = (known ? 0u : TQ_STATUS_BAD_POSITION) | (slot != -1 && !in_pool ? TQ_STATUS_BAD_PAGE : 0u);
    if (bad) atomicOr(p.cache.d_status, bad);
  }
  const size_t slot_at = keep ? (size_t)page * p.cache.page_stride + (size_t)((uint32_t)slot - page * p.cache.page_size) * p.cache.slot_stride + e0 : 0;

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

  for (; n < heads && (n < H || keep); n += step, load(n)) {
    float f[8];
    raw.get(f);
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
  }
}

template <int TYPE, bool INTERLEAVED>
int launch(const RopeParams& p, cudaStream_t st) {
  const uint32_t side = kRopeThreads / (p.cache.head_dim / 8u), heads = p.n_q_heads + 2u * p.cache.n_kv_heads;
  // few tokens: a block for every set of heads; many: one block walks all heads of its token and keeps
  // the cosines and sines
  const uint32_t parts = p.n_tokens < 2u * (uint32_t)sm_count() ? (heads + side - 1u) / side : 1u;
  const dim3 grid(p.n_tokens, parts);
  const char* what = "rope_append launch";
  return p.cache.head_dim == 64 ? launch_pdl(rope_append_kernel<TYPE, INTERLEAVED, 64>, grid, kRopeThreads, 0, st, what, p)
                                : launch_pdl(rope_append_kernel<TYPE, INTERLEAVED, 128>, grid, kRopeThreads, 0, st, what, p);
}

}  // namespace

extern "C" int tq_rope_append(const void* d_q, const void* d_k, const void* d_v, int x_type, int64_t q_stride, int64_t k_stride,
                              int64_t v_stride, uint32_t n_tokens, uint32_t n_q_heads, const float* d_table, uint32_t n_positions,
                              uint32_t rot_dim, const int32_t* d_positions, const uint32_t* sections, uint32_t n_axes,
                              int interleaved, const int32_t* d_slots, const tq_kv_cache* cache, void* d_q_out,
                              void* cuda_stream) {
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
  if (n_tokens > 0x7FFFFFFFu || n_q_heads > 65536u) return TQ_ERR_UNSUPPORTED_SHAPE;
  if (n_tokens == 0) return TQ_OK;
  auto bad = [](const void* ptr, uintptr_t align) { return ptr == nullptr || ((uintptr_t)ptr & (align - 1u)) != 0; };
  if (bad(d_q, 16) || bad(d_k, 16) || bad(d_v, 16) || bad(d_table, 4) || bad(d_positions, 4) || bad(d_slots, 4) || bad(d_q_out, 16)) return TQ_ERR_INVALID_ARG;
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
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (x_type == TQ_TYPE_F32) return interleaved ? launch<TQ_TYPE_F32, true>(p, st) : launch<TQ_TYPE_F32, false>(p, st);
  return interleaved ? launch<TQ_TYPE_BF16, true>(p, st) : launch<TQ_TYPE_BF16, false>(p, st);
}
