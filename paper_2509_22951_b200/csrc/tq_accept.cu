// Drafted tokens that the samples agree with (tq_tree_accept): the walk through a sequence's tree, and the copies of the
// accepted tokens' keys and values, in every layer's cache, to the places that follow the certain ones.
//
// The walk is a chain of dependent looks at a few hundred integers and the copies are a few kilobytes a layer: all latency.  So one
// launch does both: every block walks its sequence for itself (the integers come into shared memory in one round trip, a step
// is a compare and a ballot over 32 rows) and then copies its share of the layers, 16 bytes a thread.  One B200, calls in a graph: one sequence of
// 32 tokens and 16 caches 2.4 us, 64 sequences of 48 tokens 5.8 us (their bytes: 0.65).
//
// Order of the copies.  A row follows its parent, so the path rises and path[d] >= d: state d is written where no later entry's
// source lies, and an entry's source has been read before a later one can be written over it.  A thread owns the same
// 16 bytes of every state and goes along the path, up to four loads ahead of their stores: nothing else orders the copies.
#include <cuda_runtime.h>

#include <cstdint>

#include "tq_internal.h"
#include "tq_ops_common.cuh"

namespace {

using namespace tq_ops;

constexpr uint32_t kAcceptThreads = 256;
constexpr uint32_t kStaged = 512;  // rows of a sequence that are looked at in shared memory

struct AcceptParams {
  const int32_t* first;
  const int32_t* lens;
  const int32_t* tokens;
  const int32_t* parents;
  const int32_t* sampled;
  const int32_t* page_table;
  int32_t* out_tokens;
  int32_t* path;
  int32_t* count;
  int32_t* lens_out;
  uint32_t n_tokens, max_path, max_pages, n_caches;
  uint32_t n_pages, page_size, n_kv_heads, chunks;  // chunks: 16 bytes of a head
  int64_t page_stride, head_stride, slot_stride;
  uint32_t n_pools;
  uint4* pools[2 * TQ_MAX_CACHES];  // keys and values of the caches, each once
  uint32_t* status[TQ_MAX_CACHES];
};

// grid (sequences, shares of the caches)
__global__ void __launch_bounds__(kAcceptThreads) tree_accept_kernel(const __grid_constant__ AcceptParams p) {
  __shared__ int32_t s_parent[kStaged], s_token[kStaged], s_sampled[kStaged];
  __shared__ int32_t s_path[TQ_TREE_MAX_PATH];
  __shared__ int64_t s_from[TQ_TREE_MAX_PATH], s_to[TQ_TREE_MAX_PATH];
  __shared__ uint32_t s_count, s_moves;
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint32_t b = blockIdx.x, tid = threadIdx.x, lane = tid & 31u;
  const int32_t most = (int32_t)p.n_tokens;
  const int32_t lo = max(0, min(p.first[b], most)), hi = max(lo, min(p.first[b + 1], most)), n = hi - lo;
  const int32_t len = p.lens[b];
  for (uint32_t i = tid; i < kStaged && (int32_t)i < n; i += kAcceptThreads) {
    s_parent[i] = p.parents[lo + i];
    s_token[i] = p.tokens[lo + i];
    s_sampled[i] = p.sampled[lo + i];
  }
  if (tid == 0) s_moves = 0u;
  __syncthreads();
  if (tid < 32u) {
    uint32_t d = 0;
    int32_t cur = n > 0 ? 0 : -1;
    while (cur >= 0) {
      const int32_t drawn = cur < (int32_t)kStaged ? s_sampled[cur] : p.sampled[lo + cur];
      if (lane == 0) {
        s_path[d] = cur;
        if (blockIdx.y == 0) {
          p.path[(size_t)b * p.max_path + d] = cur;
          p.out_tokens[(size_t)b * p.max_path + d] = drawn;
        }
      }
      if (++d == p.max_path) break;
      int32_t next = -1;
      for (int64_t base = cur + 1; base < n && next < 0; base += 32) {
        const int64_t j = base + lane;
        bool follows = false;
        if (j < n) follows = j < (int64_t)kStaged ? s_parent[j] == cur && s_token[j] == drawn : p.parents[lo + j] == cur && p.tokens[lo + j] == drawn;
        const uint32_t any = __ballot_sync(kFull, follows);
        if (any) next = (int32_t)(base + __ffs(any) - 1);
      }
      cur = next;
    }
    if (lane == 0) s_count = d;
    if (blockIdx.y == 0) {
      for (uint32_t i = d + lane; i < p.max_path; i += 32u) p.path[(size_t)b * p.max_path + i] = p.out_tokens[(size_t)b * p.max_path + i] = -1;
      if (lane == 0) {
        p.count[b] = (int32_t)d;
        p.lens_out[b] = len - n + (int32_t)d;
      }
    }
  }
  __syncthreads();
  const uint32_t count = s_count;
  // where the states of the path lie and go to, in elements; 0 entries that stay or cannot be moved
  bool bad = false;
  for (uint32_t d = tid; d < count; d += kAcceptThreads) {
    const int64_t before = (int64_t)len - n;
    int64_t at[2] = {-1, -1};
    const bool moves = s_path[d] != (int32_t)d;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int64_t pos = before + (i ? (int64_t)d : (int64_t)s_path[d]);
      if (!moves || p.n_caches == 0u) continue;
      if (pos < 0 || pos >= (int64_t)p.max_pages * p.page_size) {
        bad = true;
        continue;
      }
      const uint32_t pg = (uint32_t)((uint64_t)pos / p.page_size), slot = (uint32_t)((uint64_t)pos - (uint64_t)pg * p.page_size);
      const int32_t page = p.page_table[(size_t)b * p.max_pages + pg];
      if ((uint32_t)page >= p.n_pages) {
        bad = true;
        continue;
      }
      at[i] = (int64_t)page * p.page_stride + (int64_t)slot * p.slot_stride;
    }
    const bool go = at[0] >= 0 && at[1] >= 0;
    s_from[d] = go ? at[0] : -1;
    s_to[d] = at[1];
    if (go) s_moves = 1u;
  }
  if (bad && blockIdx.y == 0)
    for (uint32_t c = 0; c < p.n_caches; ++c)
      if (p.status[c]) atomicOr(p.status[c], TQ_STATUS_BAD_PAGE);
  __syncthreads();
  if (s_moves == 0u) return;
  const uint32_t per_head = p.chunks, per_side = p.n_kv_heads * per_head, columns = p.n_pools * per_side;
  for (uint32_t col = blockIdx.y * kAcceptThreads + tid; col < columns; col += gridDim.y * kAcceptThreads) {
    const uint32_t pool = col / per_side, rest = col - pool * per_side, head = rest / per_head, x = rest - head * per_head;
    uint4* const base = p.pools[pool] + ((int64_t)head * p.head_stride) / 8 + x;
    for (uint32_t d0 = 1; d0 < count; d0 += 4u) {
      uint4 v[4];
#pragma unroll
      for (uint32_t i = 0; i < 4u; ++i)
        if (d0 + i < count && s_from[d0 + i] >= 0) v[i] = base[s_from[d0 + i] / 8];
#pragma unroll
      for (uint32_t i = 0; i < 4u; ++i)
        if (d0 + i < count && s_from[d0 + i] >= 0) base[s_to[d0 + i] / 8] = v[i];
    }
  }
}

bool bad_ptr(const void* ptr) { return ptr == nullptr || ((uintptr_t)ptr & 3u) != 0; }

}  // namespace

extern "C" int tq_tree_accept(const tq_kv_cache* caches, uint32_t n_caches, const int32_t* d_page_table, uint32_t max_pages,
                              uint32_t n_seqs, uint32_t n_tokens, const int32_t* d_first, const int32_t* d_lens,
                              const int32_t* d_tokens, const int32_t* d_parents, const int32_t* d_sampled, uint32_t max_path,
                              int32_t* d_out_tokens, int32_t* d_path, int32_t* d_count, int32_t* d_lens_out,
                              void* cuda_stream) {
  if ((n_caches && !caches) || max_path == 0 || (n_caches && max_pages == 0)) return TQ_ERR_INVALID_ARG;
  if (n_caches > TQ_MAX_CACHES || max_path > TQ_TREE_MAX_PATH || n_seqs > 0x7FFFFFFFu || n_tokens > 0x7FFFFFFFu) return TQ_ERR_UNSUPPORTED_SHAPE;
  AcceptParams p{};
  constexpr uint32_t kKnown = 512;  // places of a table of the pools, twice as many as there can be
  static_assert(kKnown >= 4 * TQ_MAX_CACHES && kKnown == 1u << (32 - 23), "the table does not fill up");
  const void* known[kKnown] = {};
  for (uint32_t i = 0; i < n_caches; ++i) {
    const tq_kv_cache &c = caches[i], &c0 = caches[0];
    if (int rc = tq_check_cache(&c)) return rc;
    if (c.n_pages != c0.n_pages || c.page_size != c0.page_size || c.n_kv_heads != c0.n_kv_heads || c.head_dim != c0.head_dim ||
        c.page_stride != c0.page_stride || c.head_stride != c0.head_stride || c.slot_stride != c0.slot_stride)
      return TQ_ERR_INVALID_ARG;
    for (void* pool : {c.d_k, c.d_v}) {  // moved twice at once, a pool's states would be read after they have been written over
      uint32_t at = (uint32_t)((uintptr_t)pool >> 4) * 2654435769u >> 23;
      while (known[at] != nullptr && known[at] != pool) at = (at + 1u) % kKnown;
      if (known[at] == nullptr) known[at] = p.pools[p.n_pools++] = static_cast<uint4*>(pool);
    }
    p.status[i] = c.d_status;
  }
  if (n_seqs == 0) return TQ_OK;
  if (bad_ptr(d_first) || bad_ptr(d_lens) || bad_ptr(d_out_tokens) || bad_ptr(d_path) || bad_ptr(d_count) || bad_ptr(d_lens_out)) return TQ_ERR_INVALID_ARG;
  if (n_tokens && (bad_ptr(d_tokens) || bad_ptr(d_parents) || bad_ptr(d_sampled))) return TQ_ERR_INVALID_ARG;
  if ((n_caches && bad_ptr(d_page_table)) || d_lens_out == d_lens) return TQ_ERR_INVALID_ARG;
  p.first = d_first;
  p.lens = d_lens;
  p.tokens = d_tokens;
  p.parents = d_parents;
  p.sampled = d_sampled;
  p.page_table = d_page_table;
  p.out_tokens = d_out_tokens;
  p.path = d_path;
  p.count = d_count;
  p.lens_out = d_lens_out;
  p.n_tokens = n_tokens;
  p.max_path = max_path;
  p.max_pages = max_pages;
  p.n_caches = n_caches;
  if (n_caches) {
    p.n_pages = caches[0].n_pages;
    p.page_size = caches[0].page_size;
    p.n_kv_heads = caches[0].n_kv_heads;
    p.chunks = caches[0].head_dim / 8u;
    p.page_stride = caches[0].page_stride;
    p.head_stride = caches[0].head_stride;
    p.slot_stride = caches[0].slot_stride;
  }
  // a block for every 256 pieces of 16 bytes of a state, but no more than eight blocks an SM in all: each walks the tree again
  const uint64_t columns = (uint64_t)p.n_pools * p.n_kv_heads * p.chunks, room = 8ull * (uint64_t)sm_count() / n_seqs;
  const uint64_t shares = (columns + kAcceptThreads - 1u) / kAcceptThreads;
  const uint32_t y = (uint32_t)(shares < room ? shares : room);
  return launch_pdl(tree_accept_kernel, dim3(n_seqs, y ? y : 1u), kAcceptThreads, 0, (cudaStream_t)cuda_stream, "tree_accept launch", p);
}
