// Attention of few queries over a long run of keys: one new token of each sequence over its paged cache
// (tq_paged_attention), one or a few tokens over an encoder's states (tq_cross_attention; each token is a query of its own).
//
//   out = sum_s p_s v_s / sum_s p_s,   p_s = exp(scale q.k_s - m),   m a running maximum
//
// Every key and value is used by the G = n_q_heads / n_kv_heads query heads that share it, at 2 G
// operations a byte: memory bound by a factor of 20 and more, so the kernel is built around the loads.
//
// Split.  The work is a flat list of units of 128 states, all sequences' and heads' one after the other;
// each CTA takes an equal share of consecutive units, whatever the lengths are (they are known on the
// device only).  A group (sequence, key-value head) that lies in several shares leaves its parts
// (maximum, sum, unnormalised output) in the workspace and the CTA that finishes last joins them in the
// order of the CTAs, so the result does not depend on timing.
//
// CTA.  Eight warps, one CTA to an SM.  A warp works on its own 16 states of each unit with its own ring of two
// stages filled by 16-byte cp.async, so nothing in the loop waits for another warp, and 64 KB and more are under way
// on every SM (6.5 TB/s x 1 us of latency / 148 SMs = 44 KB are the least).  The page ids of a step are loaded one
// step before its copies are issued.  Measured for 8 sequences of up to 8191 tokens with 24 / 8 heads | one of
// 131071, 32 / 8 | 64 of up to 16384, 64 / 8 | 4 over 6404 encoder states, 32 / 8 (us), before the last steps
// (now 33.4 | 91.1 | 391 | 24.8 on another GPU): 34.7 | 90.1 | 392 | 24.6;
// three stages 35.6 | 93.0 | 414 | 25.4; two CTAs of four warps, which leave twice the parts to join,
// 35.6 | 90.3 | 392 | 28.1; ten warps 34.4 | 93.7 | 402 | 25.5, six 37.8 | 95.4 | 418 | 26.4.
//
// Arithmetic.  mma.sync m16n8k16, bf16 in, fp32 out, with the states as the rows: S^T = K Q^T (16 states x
// 8 heads), then O^T = V^T P^T (head_dim x 8 heads), so that a group of up to 8 heads wastes nothing but
// the columns it lacks; the accumulators of S^T become the operand P^T by one 8x8 transpose in registers
// (movmatrix).  tcgen05 would have to run with 120 of 128 rows empty and gains nothing on a kernel that
// waits for memory.  p goes into the product with V as two bf16 parts, which hold 16 of its bits between them: in one part, the
// error against 64 bits is 1.9e-3 of the result's norm, in two 1.7e-3, which is the rounding of the result (8 sequences 32.8 us in one
// part, 33.4 in two; 64: 388 and 391; encoder states 24.4 and 24.8).  The lower parts' products are summed apart: where a value of V
// is infinite they are 0 x Inf, and the upper parts' sum is the answer.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>
#include <cstdio>

#include "tq_internal.h"
#include "tq_ops_common.cuh"

namespace {

using namespace tq_ops;

constexpr int kWarps = 8, kThreads = kWarps * 32;
constexpr int kStages = 2;
constexpr uint32_t kStepStates = 16;                     // states of a warp's step
constexpr uint32_t kUnitStates = kWarps * kStepStates;   // states of a CTA's unit
constexpr uint32_t kHeads = 8;                           // query heads of a group: the columns of the products

struct AttnParams {
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  int64_t outer_stride, head_stride, inner_stride;  // page or sequence, head, slot or state
  const __nv_bfloat16* q;
  int64_t q_batch_stride, q_token_stride;
  __nv_bfloat16* out;
  float* lse;
  const int32_t* lens;        // paged: lengths; cross: kv_len or nullptr
  const int32_t* page_table;  // paged
  const uint8_t* mask;        // cross: or nullptr
  uint32_t max_pages, page_size, n_pages;
  uint32_t n_states, block_len, n_blocks;
  uint32_t compact;           // cross: the units are those of the visible blocks alone (one token, at most 32 blocks)
  uint32_t n_seqs, n_tokens, n_q_heads, n_kv_heads, group, head_parts;  // head_parts: groups of 8 heads that share a key-value head
  float scale_log2;
  uint32_t* status;
  tq_attn_ws ws;
};

template <int D>
struct Smem {
  static constexpr uint32_t kRow = D * 2;                        // bytes of a state's keys or values
  static constexpr uint32_t kTile = kStepStates * kRow;          // keys or values of a step
  static constexpr uint32_t kRing = kStages * 2 * kTile;         // of one warp
  static constexpr uint32_t kORow = D + 4;                       // floats: the four heads of a store land in different banks
  static constexpr uint32_t kOffO = kWarps * kRing;
  static constexpr uint32_t kOffM = kOffO + kWarps * kHeads * kORow * 4;
  static constexpr uint32_t kOffL = kOffM + kWarps * kHeads * 4;
  static constexpr uint32_t kOffFlag = kOffL + kWarps * kHeads * 4;
  static constexpr uint32_t kTotal = kOffFlag + 16;
};
// floats of one part of a split group in the workspace
constexpr uint32_t kPartFloats = kHeads * 128 + 2 * kHeads;

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void ldsm4(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4_t(uint32_t (&r)[4], uint32_t addr) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t a) {
  uint32_t d;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(d) : "r"(a));
  return d;
}
__device__ __forceinline__ void mma_bf16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

// States of sequence b that a call may look at.
template <bool PAGED>
__device__ __forceinline__ uint32_t length_of(const AttnParams& p, uint32_t b) {
  if (PAGED) {
    const int32_t n = __ldg(p.lens + b);
    const uint64_t cap = (uint64_t)p.max_pages * p.page_size;
    return n <= 0 ? 0u : (uint32_t)((uint64_t)n > cap ? cap : (uint64_t)n);
  }
  uint32_t len = p.n_states;
  if (p.lens != nullptr) {
    const int32_t n = __ldg(p.lens + b);
    len = n <= 0 ? 0u : min((uint32_t)n, p.n_states);
  }
  if (!p.compact) return len;
  // the visible blocks' states, one block after the other; only the last one of them can be cut by the length
  const uint8_t* m = p.mask + (size_t)b * p.n_blocks;
  uint32_t sum = 0;
#pragma unroll 8
  for (uint32_t k = 0; k < p.n_blocks; ++k) sum += __ldg(m + k) != 0 && k * p.block_len < len ? min(p.block_len, len - k * p.block_len) : 0u;
  return sum;
}
// Units of a group of sequence b; a group without states keeps one, whose CTA writes its zeros.
__device__ __forceinline__ uint32_t units_of(uint32_t len) { return len == 0u ? 1u : (len + kUnitStates - 1u) / kUnitStates; }

// A position in the flat list of units: unit `tile` of group m of sequence b.
struct Walk {
  uint32_t b, m, tile, len, tiles;
  template <bool PAGED>
  __device__ __forceinline__ void enter(const AttnParams& p) {
    len = length_of<PAGED>(p, b);
    tiles = units_of(len);
  }
  template <bool PAGED>
  __device__ __forceinline__ void next(const AttnParams& p, uint32_t groups) {
    if (++tile < tiles) return;
    tile = 0;
    if (++m < groups) return;
    m = 0;
    if (++b < p.n_seqs) enter<PAGED>(p);
  }
};

template <int D, bool PAGED>
__global__ void __launch_bounds__(kThreads, 1) split_attention_kernel(const AttnParams p) {
  using L = Smem<D>;
  extern __shared__ __align__(128) uint8_t smem[];
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t tid = threadIdx.x, warp = tid >> 5, lane = tid & 31u;
  const uint32_t groups = p.n_tokens * p.n_kv_heads * p.head_parts;  // of one sequence
  float* const so = reinterpret_cast<float*>(smem + L::kOffO);
  float* const sm = reinterpret_cast<float*>(smem + L::kOffM);
  float* const sl = reinterpret_cast<float*>(smem + L::kOffL);
  uint32_t* const flag = reinterpret_cast<uint32_t*>(smem + L::kOffFlag);
  asm volatile("griddepcontrol.wait;" ::: "memory");

  // ---- this CTA's share of the units: every warp finds it for itself -------------------------------
  // (32-bit arithmetic, the launch has seen to it that the units fit: this code runs once and cold, so it is kept short)
  uint32_t u0, n_units, mean, over;  // CTA i has the units i * mean + min(i, over) and on
  Walk at;
  {
    const uint32_t per = (p.n_seqs + 31u) / 32u, begin = min(lane * per, p.n_seqs), end = min(begin + per, p.n_seqs);
    uint32_t sum = 0;
    for (uint32_t b = begin; b < end; ++b) sum += units_of(length_of<PAGED>(p, b));
    uint32_t incl = sum;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) {
      const uint32_t o = __shfl_up_sync(kFull, incl, d);
      if (lane >= (uint32_t)d) incl += o;
    }
    const uint32_t total = __shfl_sync(kFull, incl, 31) * groups, ctas = min(gridDim.x, total);
    if (blockIdx.x >= ctas) return;  // nothing waits for this CTA
    mean = total / ctas;
    over = total - mean * ctas;
    u0 = blockIdx.x * mean + min(blockIdx.x, over);
    n_units = mean + (blockIdx.x < over ? 1u : 0u);
    const uint32_t owner = __ffs(__ballot_sync(kFull, u0 < incl * groups)) - 1u;
    uint32_t before = incl - sum, b = begin;  // before: units of one group of each earlier sequence
    if (lane == owner) {
      for (; b + 1u < end; ++b) {
        const uint32_t n = units_of(length_of<PAGED>(p, b));
        if (u0 < (before + n) * groups) break;
        before += n;
      }
    }
    at.b = __shfl_sync(kFull, b, owner);
    before = __shfl_sync(kFull, before, owner);
    at.enter<PAGED>(p);
    const uint32_t rest = u0 - before * groups;
    at.m = rest / at.tiles;
    at.tile = rest - at.m * at.tiles;
  }
  auto cta_of = [&](uint32_t u) { return u < over * (mean + 1u) ? u / (mean + 1u) : over + (u - over * (mean + 1u)) / mean; };

  // ---- loads: page ids (or mask bytes) one step ahead of the copies ---------------------------------
  const uint32_t ring = tq_sm100::smem_u32(smem) + warp * L::kRing;
  Walk fw = at;            // the step whose ids are loaded next
  uint32_t f_left = n_units;
  int32_t f_id = 0;        // lane 0..15: page of the lane's state, or its mask byte
  uint32_t f_inner = 0;    // its slot in the page, or its state
  uint32_t f_head = 0, f_b = 0;
  bool f_live = false;
  bool bad_page = false;
  uint32_t list = 0, list_b = 0xFFFFFFFFu;  // compact: lane k has the k-th visible block of sequence list_b
  auto fetch = [&]() {
    f_live = false;
    if (f_left == 0) return;
    const uint32_t s = fw.tile * kUnitStates + warp * kStepStates + lane;
    f_head = (fw.m / p.head_parts) % p.n_kv_heads;
    f_b = fw.b;
    f_live = lane < kStepStates && s < fw.len;
    if (PAGED) {
      const uint32_t pg = s / p.page_size;
      f_inner = s - pg * p.page_size;
      if (f_live) f_id = __ldg(p.page_table + (size_t)fw.b * p.max_pages + pg);
      if (fw.tile == 0 && __ldg(p.lens + fw.b) > 0 && (uint32_t)__ldg(p.lens + fw.b) > fw.len) bad_page = true;
    } else if (p.compact) {
      if (fw.b != list_b) {
        list_b = fw.b;
        const bool seen = lane < p.n_blocks && __ldg(p.mask + (size_t)fw.b * p.n_blocks + lane) != 0;
        list = __fns(__ballot_sync(kFull, seen), 0, (int)lane + 1);
      }
      const uint32_t k = f_live ? s / p.block_len : 0u;
      f_inner = __shfl_sync(kFull, list, k) * p.block_len + (s - k * p.block_len);
      f_id = 1;
    } else {
      f_inner = s;
      f_id = 1;
      if (f_live && p.mask != nullptr) {
        const uint32_t t = fw.m / (p.head_parts * p.n_kv_heads);
        f_id = __ldg(p.mask + ((size_t)fw.b * p.n_tokens + t) * p.n_blocks + s / p.block_len);
      }
    }
    --f_left;
    if (f_left) fw.next<PAGED>(p, groups);
  };
  // copies of the fetched step into a stage; returns which of its 16 states are there
  auto issue = [&](uint32_t stage) -> uint32_t {
    bool live = f_live;
    int64_t off = (int64_t)f_head * p.head_stride + (int64_t)f_inner * p.inner_stride;
    if (PAGED) {
      if (live && (uint32_t)f_id >= p.n_pages) {
        live = false;
        bad_page = true;
      }
      off += (int64_t)f_id * p.outer_stride;
    } else {
      live = live && f_id != 0;
      off += (int64_t)f_b * p.outer_stride;
    }
    if (!live) off = 0;
    const uint32_t there = __ballot_sync(kFull, live);
    if (there != 0) {
      constexpr uint32_t kChunks = L::kRow / 16, kRows = 32 / kChunks;  // chunks of a row, rows of a warp-wide copy
      const uint32_t c = lane % kChunks, dst0 = ring + stage * 2 * L::kTile;
#pragma unroll
      for (uint32_t r0 = 0; r0 < kStepStates; r0 += kRows) {
        const uint32_t r = r0 + lane / kChunks;
        const int64_t o = __shfl_sync(kFull, off, r) + c * 8;
        const uint32_t dst = dst0 + r * L::kRow + ((c ^ (r & 7u)) << 4);
        const uint32_t bytes = (there >> r) & 1u ? 16u : 0u;  // 0: zeros, nothing is read
        cp_async16(dst, p.k + o, bytes);
        cp_async16(dst + L::kTile, p.v + o, bytes);
      }
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
    return there;
  };

  // groups of which this CTA has a part: [0] one that began in an earlier CTA's share, [1] one that goes on in the next
  struct Part {
    uint32_t parts, c0, n_heads;
    size_t out0;
  };
  Part open_parts[2] = {};

  // a thread's place where outputs are summed: four columns of a head
  const uint32_t mine_h = tid / (D / 4), quad = tid % (D / 4);
  static_assert(kThreads >= kHeads * D / 4, "four columns of each head to a thread");
  auto finish = [&](size_t row, const float4& o, float M, float Ls) {
    const float inv = 1.0f / Ls;
    const bool none = Ls == 0.f;
    *reinterpret_cast<uint2*>(p.out + row * D + 4u * quad) =
        none ? make_uint2(0u, 0u) : make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
    if (quad == 0u && p.lse) p.lse[row] = none ? -INFINITY : (M + log2f(Ls)) * 0.6931471805599453f;
  };

  uint32_t there[kStages];
  fetch();
#pragma unroll
  for (int s = 0; s < kStages - 1; ++s) {
    there[s] = issue(s);
    fetch();
  }

  uint32_t qb[D / 16][2];
  float o[D / 16][4], o_low[D / 16][4], m[2], l[2];  // o: by p's upper parts; o_low: by its lower ones
  bool fresh = true;
  uint32_t group_first = u0 - at.tile;  // first unit of the current group
  uint32_t stage = 0;
  for (uint32_t i = 0; i < n_units; ++i) {
    const uint32_t part = at.m % p.head_parts, kvh = (at.m / p.head_parts) % p.n_kv_heads;
    const uint32_t t = at.m / (p.head_parts * p.n_kv_heads);
    const uint32_t n_heads = min(kHeads, p.group - part * kHeads), h0 = kvh * p.group + part * kHeads;
    if (fresh) {
      fresh = false;
      const uint32_t n = lane >> 2;
      const __nv_bfloat16* q = p.q + (int64_t)at.b * p.q_batch_stride + (int64_t)t * p.q_token_stride + (size_t)(h0 + n) * D + 2u * (lane & 3u);
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        qb[kk][0] = n < n_heads ? __ldg(reinterpret_cast<const uint32_t*>(q + kk * 16)) : 0u;
        qb[kk][1] = n < n_heads ? __ldg(reinterpret_cast<const uint32_t*>(q + kk * 16 + 8)) : 0u;
      }
#pragma unroll
      for (int d = 0; d < D / 16; ++d)
#pragma unroll
        for (int c = 0; c < 4; ++c) o[d][c] = o_low[d][c] = 0.f;
      m[0] = m[1] = -INFINITY;
      l[0] = l[1] = 0.f;
    }
    __syncwarp();  // the stage that is refilled now was read by every lane
    there[kStages - 1] = issue(stage == 0 ? kStages - 1 : stage - 1);
    fetch();
    asm volatile("cp.async.wait_group %0;" ::"n"(kStages - 1) : "memory");
    __syncwarp();

    const uint32_t live = there[0];
    if (live != 0) {
      const uint32_t kt = ring + stage * 2 * L::kTile, vt = kt + L::kTile;
      const uint32_t mi = lane >> 3, r8 = lane & 7u;
      float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int kk = 0; kk < D / 16; ++kk) {
        uint32_t a[4];
        const uint32_t r = (mi & 1u) * 8u + r8;
        ldsm4(a, kt + r * L::kRow + (((kk * 2u + (mi >> 1)) ^ r8) << 4));
        mma_bf16(s, a, qb[kk][0], qb[kk][1]);
      }
      // rows lane/4 and lane/4 + 8, columns (heads) 2 (lane % 4) and + 1
      const bool lo = (live >> (lane >> 2)) & 1u, hi = (live >> ((lane >> 2) + 8u)) & 1u;
      float x[4];
      x[0] = lo ? s[0] * p.scale_log2 : -INFINITY;
      x[1] = lo ? s[1] * p.scale_log2 : -INFINITY;
      x[2] = hi ? s[2] * p.scale_log2 : -INFINITY;
      x[3] = hi ? s[3] * p.scale_log2 : -INFINITY;
      float mx[2] = {fmaxf(x[0], x[2]), fmaxf(x[1], x[3])};
#pragma unroll
      for (int d = 4; d < 32; d <<= 1) {
        mx[0] = fmaxf(mx[0], __shfl_xor_sync(kFull, mx[0], d));
        mx[1] = fmaxf(mx[1], __shfl_xor_sync(kFull, mx[1], d));
      }
      const bool grows = mx[0] > m[0] || mx[1] > m[1];
      if (__any_sync(kFull, grows)) {
#pragma unroll
        for (int c = 0; c < 2; ++c) {
          const float mn = fmaxf(m[c], mx[c]);
          const float f = mn == -INFINITY ? 1.f : exp2_fast(m[c] - mn);  // 0 when there was nothing before
          m[c] = mn;
          l[c] *= f;
#pragma unroll
          for (int d = 0; d < D / 16; ++d) {
            o[d][c] *= f;
            o[d][c + 2] *= f;
            o_low[d][c] *= f;
            o_low[d][c + 2] *= f;
          }
        }
      }
      const float r0 = m[0] == -INFINITY ? 0.f : m[0], r1 = m[1] == -INFINITY ? 0.f : m[1];
      const float e0 = exp2_fast(x[0] - r0), e1 = exp2_fast(x[1] - r1), e2 = exp2_fast(x[2] - r0), e3 = exp2_fast(x[3] - r1);
      l[0] += e0 + e2;
      l[1] += e1 + e3;
      const uint32_t h0 = pack_bf16(e0, e1), h1 = pack_bf16(e2, e3);
      const uint32_t b0 = transpose8x8(h0), b1 = transpose8x8(h1);
      const uint32_t c0 = transpose8x8(pack_bf16(e0 - bf16_lo(h0), e1 - bf16_hi(h0))), c1 = transpose8x8(pack_bf16(e2 - bf16_lo(h1), e3 - bf16_hi(h1)));
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
        uint32_t a[4];
        const uint32_t r = (mi >> 1) * 8u + r8;
        ldsm4_t(a, vt + r * L::kRow + (((d * 2u + (mi & 1u)) ^ r8) << 4));
        mma_bf16(o[d], a, b0, b1);
        mma_bf16(o_low[d], a, c0, c1);
      }
    }
#pragma unroll
    for (int s = 0; s < kStages - 1; ++s) there[s] = there[s + 1];
    if (++stage == kStages) stage = 0;

    if (at.tile + 1u != at.tiles && i + 1u != n_units) {
      ++at.tile;
      continue;
    }
    // ---- end of the group, or of this CTA's part of it: the warps' results become one ------------
    fresh = true;
#pragma unroll
    for (int d = 4; d < 32; d <<= 1) {
      l[0] += __shfl_xor_sync(kFull, l[0], d);
      l[1] += __shfl_xor_sync(kFull, l[1], d);
    }
    if (lane < 4) {
      sm[warp * kHeads + 2 * lane] = m[0];
      sm[warp * kHeads + 2 * lane + 1] = m[1];
      sl[warp * kHeads + 2 * lane] = l[0];
      sl[warp * kHeads + 2 * lane + 1] = l[1];
    }
    {
      float* w = so + (warp * kHeads + 2u * (lane & 3u)) * L::kORow + (lane >> 2);
#pragma unroll
      for (int d = 0; d < D / 16; ++d) {
#pragma unroll
        for (int c = 0; c < 4; ++c) o[d][c] += fabsf(o_low[d][c]) < INFINITY ? o_low[d][c] : 0.f;
        w[d * 16] = o[d][0];
        w[d * 16 + L::kORow] = o[d][1];
        w[d * 16 + 8] = o[d][2];
        w[d * 16 + 8 + L::kORow] = o[d][3];
      }
    }
    __syncthreads();
    const uint32_t first = group_first, end = first + at.tiles;  // units of the whole group
    const bool whole = first >= u0 && end - u0 <= n_units;
    const uint32_t c0 = whole ? blockIdx.x : cta_of(first);
    const size_t out0 = ((size_t)at.b * p.n_tokens + t) * p.n_q_heads + h0;
    if (mine_h < n_heads) {  // four columns of a head to a thread
      const float* const ow = so + mine_h * L::kORow + 4u * quad;
      float M = sm[mine_h];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) M = fmaxf(M, sm[w * kHeads + mine_h]);
      const float ref = M == -INFINITY ? 0.f : M;
      float Ls = 0.f;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2_fast(sm[w * kHeads + mine_h] - ref);
        const float4 y = *reinterpret_cast<const float4*>(ow + w * kHeads * L::kORow);
        Ls += f * sl[w * kHeads + mine_h];
        sum.x += f * y.x, sum.y += f * y.y, sum.z += f * y.z, sum.w += f * y.w;
      }
      if (whole) {
        finish(out0 + mine_h, sum, M, Ls);
      } else {
        float* const mine = p.ws.parts + (size_t)(2u * blockIdx.x + (blockIdx.x == c0 ? 1u : 0u)) * kPartFloats;
        reinterpret_cast<float4*>(mine)[mine_h * (D / 4) + quad] = sum;
        if (quad == 0u) {
          mine[kHeads * D + mine_h] = M;
          mine[kHeads * D + kHeads + mine_h] = Ls;
        }
      }
    }
    if (!whole) {  // published when the share is done: a fence and an atomic here would hold up the loads
      const Part g{cta_of(end - 1u) - c0 + 1u, c0, n_heads, out0};
      if (blockIdx.x == c0)
        open_parts[1] = g;
      else
        open_parts[0] = g;
    }
    __syncthreads();  // the merge area is free again
    group_first = end;
    if (i + 1u != n_units) at.next<PAGED>(p, groups);
  }
  asm volatile("cp.async.wait_all;" ::: "memory");
  if (PAGED && bad_page && p.status != nullptr) atomicOr(p.status, TQ_STATUS_BAD_PAGE);

  // ---- the at most two groups that other CTAs have parts of as well ---------------------------------------
  if (open_parts[0].parts == 0u && open_parts[1].parts == 0u) return;
  if (tid == 0) {
    // what the CTA wrote before the last barrier is published with this thread's fence; atomicInc wraps to 0 with the
    // last part, which is the state the next call needs
    __threadfence();
#pragma unroll
    for (int k = 0; k < 2; ++k)
      flag[k] = open_parts[k].parts != 0u && atomicInc(p.ws.counters + open_parts[k].c0, open_parts[k].parts - 1u) == open_parts[k].parts - 1u;
    __threadfence();
  }
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    if (!flag[k]) continue;
    const Part g = k ? open_parts[1] : open_parts[0];
    if (mine_h >= g.n_heads) continue;
    float M = -INFINITY, Ls = 0.f;
    float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (uint32_t i = 0; i < g.parts; ++i) {  // in the order of the parts
      const float* src = p.ws.parts + (size_t)(2u * (g.c0 + i) + (i == 0 ? 1u : 0u)) * kPartFloats;
      const float mi = __ldcg(src + kHeads * D + mine_h), li = __ldcg(src + kHeads * D + kHeads + mine_h);
      const float4 y = __ldcg(reinterpret_cast<const float4*>(src) + mine_h * (D / 4) + quad);
      const float mn = fmaxf(M, mi), ref = mn == -INFINITY ? 0.f : mn, f = exp2_fast(M - ref), h = exp2_fast(mi - ref);
      M = mn;
      Ls = Ls * f + li * h;
      o.x = o.x * f + y.x * h;
      o.y = o.y * f + y.y * h;
      o.z = o.z * f + y.z * h;
      o.w = o.w * f + y.w * h;
    }
    finish(g.out0 + mine_h, o, M, Ls);
  }
}

template <int D, bool PAGED>
int launch(AttnParams& p, cudaStream_t st) {
  const uint64_t states = PAGED ? (uint64_t)p.max_pages * p.page_size : p.n_states;
  const uint64_t tiles = (states < 0x7FFFFFFFull ? states : 0x7FFFFFFFull) / kUnitStates + 1u, groups = (uint64_t)p.n_tokens * p.n_kv_heads * p.head_parts;
  if (groups > 0xFFFFFFFFull / tiles || groups * tiles > 0xFFFFFFFFull / p.n_seqs) return TQ_ERR_UNSUPPORTED_SHAPE;
  auto kern = split_attention_kernel<D, PAGED>;
  constexpr size_t smem = Smem<D>::kTotal;
  const char* what = PAGED ? "paged attention launch" : "cross attention launch";
  if (int rc = tq_ensure_dynamic_smem((const void*)kern, smem, what)) return rc;
  const uint32_t grid = min((uint32_t)sm_count(), kAttnMaxCtas);
  return launch_pdl(kern, dim3(grid), kThreads, smem, st, what, p);
}

bool scale_ok(float scale) { return scale > 0.f && scale < INFINITY; }
bool misaligned(const void* ptr, uintptr_t align) { return ptr == nullptr || ((uintptr_t)ptr & (align - 1u)) != 0; }

}  // namespace

int tq_check_cache(const tq_kv_cache* c) {
  if (!c || misaligned(c->d_k, 16) || misaligned(c->d_v, 16) || ((uintptr_t)c->d_status & 3u)) return TQ_ERR_INVALID_ARG;
  if (c->n_pages == 0 || c->page_size == 0 || c->n_kv_heads == 0) return TQ_ERR_INVALID_ARG;
  if (c->page_stride % 8 || c->head_stride % 8 || c->slot_stride % 8 || c->page_stride < 0 || c->head_stride < 0 || c->slot_stride < 0) return TQ_ERR_INVALID_ARG;
  if ((c->head_dim != 64 && c->head_dim != 128) || c->n_pages > 0x7FFFFFFFu || c->n_kv_heads > 65536u) return TQ_ERR_UNSUPPORTED_SHAPE;
  return TQ_OK;
}

tq_attn_ws tq_attn_ws_plan(void* d_ws, uint64_t ws_bytes) {
  tq_attn_ws w{};
  uint64_t need = 0;
  if (misaligned(d_ws, 256) || tq_attn_workspace_size(&need) != TQ_OK || ws_bytes < need) return w;
  w.counters = static_cast<uint32_t*>(d_ws);
  w.status = w.counters + kAttnMaxCtas;
  w.open = reinterpret_cast<uint4*>(static_cast<uint8_t*>(d_ws) + kAttnWsOpen);
  w.parts = reinterpret_cast<float*>(static_cast<uint8_t*>(d_ws) + kAttnWsHeader);
  return w;
}

extern "C" {

int tq_attn_workspace_size(uint64_t* device_bytes) {
  if (!device_bytes) return TQ_ERR_INVALID_ARG;
  const uint64_t ctas = min((uint32_t)sm_count(), kAttnMaxCtas);
  const uint64_t split = ctas * 2u * kPartFloats * sizeof(float), cross = tq_cross_workspace_bytes(), tree = tq_tree_workspace_bytes();
  *device_bytes = kAttnWsHeader + max(max(split, cross), tree);
  return TQ_OK;
}

int tq_attn_workspace_init(void* d_ws, uint64_t ws_bytes, void* cuda_stream) {
  uint64_t need = 0;
  if (int rc = tq_attn_workspace_size(&need)) return rc;
  if (misaligned(d_ws, 256)) return TQ_ERR_INVALID_ARG;
  if (ws_bytes < need) return TQ_ERR_BUFFER_TOO_SMALL;
  return tq_cuda_status((int)cudaMemsetAsync(d_ws, 0, kAttnWsHeader, (cudaStream_t)cuda_stream), "attention workspace");
}

int tq_attn_status(void* d_ws, void* cuda_stream, uint32_t* status) {
  if (misaligned(d_ws, 256) || !status) return TQ_ERR_INVALID_ARG;
  uint32_t* word = static_cast<uint32_t*>(d_ws) + kAttnMaxCtas;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (int rc = tq_cuda_status((int)cudaMemcpyAsync(status, word, 4, cudaMemcpyDeviceToHost, st), "attention status")) return rc;
  if (int rc = tq_cuda_status((int)cudaMemsetAsync(word, 0, 4, st), "attention status")) return rc;
  return tq_cuda_status((int)cudaStreamSynchronize(st), "attention status");
}

int tq_paged_attention(const tq_kv_cache* cache, const void* d_q, int64_t q_stride, uint32_t n_seqs, uint32_t n_q_heads,
                       const int32_t* d_page_table, uint32_t max_pages, const int32_t* d_lens, float scale, void* d_out,
                       float* d_lse, void* d_ws, uint64_t ws_bytes, void* cuda_stream) {
  if (int rc = tq_check_cache(cache)) return rc;
  if (n_q_heads == 0 || n_q_heads % cache->n_kv_heads || q_stride % 8 || max_pages == 0 || !scale_ok(scale)) return TQ_ERR_INVALID_ARG;
  if (n_q_heads > 65536u || n_seqs > 0x7FFFFFFFu) return TQ_ERR_UNSUPPORTED_SHAPE;
  if (n_seqs == 0) return TQ_OK;
  if (misaligned(d_q, 16) || misaligned(d_page_table, 4) || misaligned(d_lens, 4) || misaligned(d_out, 16) || ((uintptr_t)d_lse & 3u)) return TQ_ERR_INVALID_ARG;
  if (misaligned(d_ws, 256)) return TQ_ERR_INVALID_ARG;
  AttnParams p{};
  p.ws = tq_attn_ws_plan(d_ws, ws_bytes);
  if (!p.ws.counters) return TQ_ERR_BUFFER_TOO_SMALL;
  p.k = (const __nv_bfloat16*)cache->d_k;
  p.v = (const __nv_bfloat16*)cache->d_v;
  p.outer_stride = cache->page_stride;
  p.head_stride = cache->head_stride;
  p.inner_stride = cache->slot_stride;
  p.q = (const __nv_bfloat16*)d_q;
  p.q_batch_stride = q_stride;
  p.out = (__nv_bfloat16*)d_out;
  p.lse = d_lse;
  p.lens = d_lens;
  p.page_table = d_page_table;
  p.max_pages = max_pages;
  p.page_size = cache->page_size;
  p.n_pages = cache->n_pages;
  p.n_seqs = n_seqs;
  p.n_tokens = 1;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = cache->n_kv_heads;
  p.group = n_q_heads / cache->n_kv_heads;
  p.head_parts = (p.group + kHeads - 1u) / kHeads;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.status = cache->d_status;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return cache->head_dim == 64 ? launch<64, true>(p, st) : launch<128, true>(p, st);
}

int tq_cross_attention(const tq_encoder_kv* kv, const void* d_q, int64_t q_batch_stride, int64_t q_token_stride,
                       uint32_t n_tokens, uint32_t n_q_heads, const int32_t* d_kv_len, const uint8_t* d_mask,
                       uint32_t block_len, float scale, void* d_out, float* d_lse, void* d_ws, uint64_t ws_bytes,
                       void* cuda_stream) {
  if (!kv || kv->n_kv_heads == 0 || (kv->n_states && (misaligned(kv->d_k, 16) || misaligned(kv->d_v, 16)))) return TQ_ERR_INVALID_ARG;
  if (kv->batch_stride % 8 || kv->state_stride % 8 || kv->head_stride % 8 || kv->batch_stride < 0 || kv->state_stride < 0 || kv->head_stride < 0) return TQ_ERR_INVALID_ARG;
  if (n_q_heads == 0 || n_q_heads % kv->n_kv_heads || q_batch_stride % 8 || q_token_stride % 8 || (d_mask && block_len == 0) || !scale_ok(scale)) return TQ_ERR_INVALID_ARG;
  if ((kv->head_dim != 64 && kv->head_dim != 128) || n_q_heads > 65536u || kv->n_states > 0x7FFFFFFFu || n_tokens > 0x7FFFFFFFu ||
      kv->n_seqs > 0x7FFFFFFFu || (uint64_t)n_tokens * n_q_heads > 0x7FFFFFFFull)
    return TQ_ERR_UNSUPPORTED_SHAPE;
  if (kv->n_seqs == 0 || n_tokens == 0) return TQ_OK;
  if (misaligned(d_q, 16) || ((uintptr_t)d_kv_len & 3u) || misaligned(d_out, 16) || ((uintptr_t)d_lse & 3u)) return TQ_ERR_INVALID_ARG;
  if (misaligned(d_ws, 256)) return TQ_ERR_INVALID_ARG;
  AttnParams p{};
  p.ws = tq_attn_ws_plan(d_ws, ws_bytes);
  if (!p.ws.counters) return TQ_ERR_BUFFER_TOO_SMALL;
  p.k = (const __nv_bfloat16*)kv->d_k;
  p.v = (const __nv_bfloat16*)kv->d_v;
  p.outer_stride = kv->batch_stride;
  p.head_stride = kv->head_stride;
  p.inner_stride = kv->state_stride;
  p.q = (const __nv_bfloat16*)d_q;
  p.q_batch_stride = q_batch_stride;
  p.q_token_stride = q_token_stride;
  p.out = (__nv_bfloat16*)d_out;
  p.lse = d_lse;
  p.lens = d_kv_len;
  p.mask = d_mask;
  p.n_states = kv->n_states;
  p.block_len = d_mask ? block_len : 1u;
  p.n_blocks = d_mask ? (uint32_t)(((uint64_t)kv->n_states + block_len - 1u) / block_len) : 0u;
  p.compact = d_mask != nullptr && n_tokens == 1 && p.n_blocks <= 32u;
  p.n_seqs = kv->n_seqs;
  p.n_tokens = n_tokens;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = kv->n_kv_heads;
  p.group = n_q_heads / kv->n_kv_heads;
  p.head_parts = (p.group + kHeads - 1u) / kHeads;
  p.scale_log2 = scale * 1.4426950408889634f;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  // Few tokens over few states: this kernel, which reads the states again (from L2) for every token and every 8 heads of a group,
  // against the tensor-core kernel, which reads them once but starts slowly and, where groups are few, leaves many parts of
  // 256 rows to be joined.  One side's cost goes by its visits of (token, key-value head, 8 heads, state), the other's by the
  // parts of a group and their size.  Measured (us, this | the other), at head_dim 128 but for the last two:
  //   1 x 6404 states, 64 / 8 heads: 4 tokens 21.4 | 30.0, 6: 25.8 | 31.0, 8: 32.6 | 31.4, 16: 54.3 | 33.2
  //   4 x 6404, 32 / 8: 2 tokens 37.0 | 37.1, 4: 57.0 | 37.8
  //   4 x 1601, 64 / 8: 2 tokens 17.0 | 22.5, 4: 23.3 | 23.6, 8: 36.7 | 24.5
  //   4 x 1601, 64 / 2: 2 tokens 15.8 | 20.4, 4: 21.7 | 21.6, 8: 34.5 | 25.2, 16: 59.7 | 31.1
  //   1 x 6404, 64 / 2: 4 tokens 21.4 | 43.6, 8: 32.7 | 49.6, 12: 43.5 | 47.3, 16: 54.3 | 50.9
  //   1 x 20000, 64 / 2: 4 tokens 44.9 | 68.1, 8: 78.0 | 74.3, 16: 143 | 55
  //   2 x 3000, 32 / 2 x 64: 4 tokens 12.4 | 20.0, 12: 21.0 | 21.4, 16: 25.2 | 22.2
  //   1 x 500, 32 / 8 x 64: 4 tokens 6.6 | 12.6, 16: 10.4 | 12.9
  constexpr uint64_t kFewTokens = 16, kFewVisits = 120000, kPartVisits = 84;  // of a column of a part
  auto few = [&] {
    const uint64_t tokens = (uint64_t)kv->n_seqs * n_tokens, tiles = ((uint64_t)kv->n_states + 127u) / 128u;
    const uint64_t groups = (uint64_t)kv->n_seqs * kv->n_kv_heads * (((uint64_t)n_tokens * p.group + 255u) / 256u);
    const uint64_t ctas = (uint64_t)sm_count(), parts = min(tiles, groups < ctas ? ctas / groups : 1u);
    const uint64_t visits = tokens * kv->n_kv_heads * p.head_parts;  // of a state
    return kv->n_states == 0 || visits <= (kFewVisits + kPartVisits * kv->head_dim * parts) / kv->n_states;
  };
  if (n_tokens > 1 && (n_tokens > kFewTokens || !few())) {
    bool served = false;
    const int rc = tq_cross_launch(kv, d_q, q_batch_stride, q_token_stride, n_tokens, n_q_heads, d_kv_len, d_mask, p.block_len, p.n_blocks,
                                   p.scale_log2, d_out, d_lse, p.ws, cuda_stream, &served);
    if (served) return rc;
  }
  return kv->head_dim == 64 ? launch<64, false>(p, st) : launch<128, false>(p, st);
}

}  // extern "C"
