// Attention of several new tokens of each sequence over its paged cache (tq_tree_attention).
//
//   out = sum_s p_s v_s / sum_s p_s,   p_s = exp(scale q.k_s - m),   m a running maximum
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "tq_internal.h"
#include "tq_ops_common.cuh"

namespace {

using namespace tq_ops;

struct TreeParams {
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  int64_t page_stride, head_stride, slot_stride;
  const __nv_bfloat16* q;
  int64_t q_stride;
  __nv_bfloat16* out;
  float* lse;
  const int32_t* first;
  const int32_t* lens;
  const int32_t* page_table;
  const uint32_t* mask;
  uint32_t mask_words, max_pages, page_size, n_pages;
  uint32_t n_tokens, n_seqs, n_q_heads, group;
  float scale_log2;
  uint32_t* status;
};

// A warp for a token and a query head.
template <int D>
__global__ void __launch_bounds__(128) tree_attention_kernel(const TreeParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint64_t job = (uint64_t)blockIdx.x * 4u + threadIdx.x / 32u;
  const uint32_t lane = threadIdx.x % 32u;
  if (job >= (uint64_t)p.n_tokens * p.n_q_heads) return;
  const int32_t row = (int32_t)(job / p.n_q_heads), h = (int32_t)(job % p.n_q_heads);
  uint32_t b = 0, end = p.n_seqs;  // the last sequence that begins at or before the row
  while (end - b > 1u) {
    const uint32_t mid = b + (end - b) / 2u;
    if (p.first[mid] <= row)
      b = mid;
    else
      end = mid;
  }
  const int32_t most = (int32_t)p.n_tokens, lo = max(0, min(p.first[b], most)), hi = max(lo, min(p.first[b + 1], most));
  if (row < lo || row >= hi) return;
  const int64_t cap = (int64_t)p.max_pages * p.page_size, given = p.lens[b], len = max((int64_t)0, min(given, cap));
  bool bad = given > cap;
  const int64_t before = given - (hi - lo);
  const int32_t i = row - lo;
  constexpr int kPer = D / 32;
  float q[kPer], o[kPer], m = -INFINITY, l = 0.f;
#pragma unroll
  for (int x = 0; x < kPer; ++x) {
    q[x] = __bfloat162float(p.q[(int64_t)row * p.q_stride + (int64_t)h * D + lane * kPer + x]);
    o[x] = 0.f;
  }
  for (int64_t s = 0; s < len; ++s) {
    if (s >= before) {
      const int64_t j = s - before;
      if (p.mask ? j >= (int64_t)p.mask_words * 32 || !((p.mask[(size_t)row * p.mask_words + j / 32] >> (j % 32)) & 1u) : j > i) continue;
    }
    const int32_t page = p.page_table[(size_t)b * p.max_pages + s / p.page_size];
    if ((uint32_t)page >= p.n_pages) {
      bad = true;
      continue;
    }
    const int64_t at = (int64_t)page * p.page_stride + (int64_t)(h / p.group) * p.head_stride + (s % p.page_size) * p.slot_stride + lane * kPer;
    float x = 0.f;
#pragma unroll
    for (int c = 0; c < kPer; ++c) x += q[c] * __bfloat162float(p.k[at + c]);
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(kFull, x, d);
    x *= p.scale_log2;
    const float mn = fmaxf(m, x), ref = mn == -INFINITY ? 0.f : mn, f = mn == -INFINITY ? 1.f : exp2f(m - mn), e = exp2f(x - ref);
    m = mn;
    l = l * f + e;
#pragma unroll
    for (int c = 0; c < kPer; ++c) o[c] = o[c] * f + e * __bfloat162float(p.v[at + c]);
  }
  const size_t at = ((size_t)row * p.n_q_heads + h);
#pragma unroll
  for (int c = 0; c < kPer; ++c) p.out[at * D + lane * kPer + c] = __float2bfloat16_rn(l == 0.f ? 0.f : o[c] / l);
  if (lane == 0 && p.lse) p.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
  if (bad && lane == 0 && p.status) atomicOr(p.status, TQ_STATUS_BAD_PAGE);
}

bool misaligned(const void* ptr, uintptr_t align) { return ptr == nullptr || ((uintptr_t)ptr & (align - 1u)) != 0; }

}  // namespace

extern "C" int tq_tree_attention(const tq_kv_cache* cache, const void* d_q, int64_t q_stride, uint32_t n_tokens, uint32_t n_seqs,
                                 uint32_t n_q_heads, const int32_t* d_first, const int32_t* d_page_table, uint32_t max_pages,
                                 const int32_t* d_lens, const uint32_t* d_mask, uint32_t mask_words, float scale, void* d_out,
                                 float* d_lse, void* d_ws, uint64_t ws_bytes, void* cuda_stream) {
  if (int rc = tq_check_cache(cache)) return rc;
  if (n_q_heads == 0 || n_q_heads % cache->n_kv_heads || q_stride % 8 || max_pages == 0 || !(scale > 0.f && scale < INFINITY) || (d_mask && mask_words == 0)) return TQ_ERR_INVALID_ARG;
  if (n_q_heads > 65536u || n_tokens > 0x7FFFFFFFu || n_seqs > 0x7FFFFFFEu || (uint64_t)n_tokens * n_q_heads > 0x7FFFFFFFull) return TQ_ERR_UNSUPPORTED_SHAPE;
  const uint64_t group = n_q_heads / cache->n_kv_heads, states = (uint64_t)max_pages * cache->page_size;
  const uint64_t tiles = (states < 0x7FFFFFFFull ? states : 0x7FFFFFFFull) / 128u + 1u, row_tiles = ((uint64_t)n_tokens * group + 127u) / 128u + n_seqs;
  if (row_tiles > 0xFFFFFFFFull / cache->n_kv_heads / tiles) return TQ_ERR_UNSUPPORTED_SHAPE;
  if (n_seqs == 0 || n_tokens == 0) return TQ_OK;
  if (misaligned(d_q, 16) || misaligned(d_first, 4) || misaligned(d_page_table, 4) || misaligned(d_lens, 4) || ((uintptr_t)d_mask & 3u) || misaligned(d_out, 16) ||
      ((uintptr_t)d_lse & 3u) || misaligned(d_ws, 256))
    return TQ_ERR_INVALID_ARG;
  const tq_attn_ws ws = tq_attn_ws_plan(d_ws, ws_bytes);
  if (!ws.counters) return TQ_ERR_BUFFER_TOO_SMALL;
  TreeParams p{};
  p.k = (const __nv_bfloat16*)cache->d_k;
  p.v = (const __nv_bfloat16*)cache->d_v;
  p.page_stride = cache->page_stride;
  p.head_stride = cache->head_stride;
  p.slot_stride = cache->slot_stride;
  p.q = (const __nv_bfloat16*)d_q;
  p.q_stride = q_stride;
  p.out = (__nv_bfloat16*)d_out;
  p.lse = d_lse;
  p.first = d_first;
  p.lens = d_lens;
  p.page_table = d_page_table;
  p.mask = d_mask;
  p.mask_words = mask_words;
  p.max_pages = max_pages;
  p.page_size = cache->page_size;
  p.n_pages = cache->n_pages;
  p.n_tokens = n_tokens;
  p.n_seqs = n_seqs;
  p.n_q_heads = n_q_heads;
  p.group = n_q_heads / cache->n_kv_heads;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.status = cache->d_status;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const uint32_t blocks = (uint32_t)(((uint64_t)n_tokens * n_q_heads + 3u) / 4u);
  const char* what = "tree attention launch";
  return cache->head_dim == 64 ? launch_pdl(tree_attention_kernel<64>, dim3(blocks), 128, 0, st, what, p)
                               : launch_pdl(tree_attention_kernel<128>, dim3(blocks), 128, 0, st, what, p);
}
