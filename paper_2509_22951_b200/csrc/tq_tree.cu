// Attention of several new tokens of each sequence over its paged cache (tq_tree_attention): drafted tokens, or a piece of a prompt.
//
//   out = sum_s p_s v_s / sum_s p_s,   p_s = exp(scale q.k_s - m),   m a running maximum
//
// The G query heads that share a key-value head and the sequence's new tokens are R = G n rows over the same states: 4 R D operations
// and 4 D bytes a state and key-value head.  For R up to about 200 the bytes bound it, above that the tensor cores and the exponentials; so
// everything is built to keep the loads going while tiles of 128 rows x 128 states go through the 5th-generation tensor cores.
//
// Work.  The units are (sequence, key-value head, tile of rows, tile of 128 states); of a chain, only the tiles that a tile's last row sees.  Each
// CTA takes an equal share of consecutive units, whatever the lengths are (they are known on the device only).  A group (sequence, key-value
// head, tile of rows) that lies in several shares leaves its parts in the workspace, and a second kernel joins them in the order of the
// CTAs: the result does not depend on timing.  (Joined by the last CTA of a group instead, without a second kernel: 31 tokens over 131071 states
// 148 us instead of 104, 8 ragged sequences 39.1 instead of 34.6; one SM reads the parts more slowly than all of them.)
//
// CTA, one to an SM, 16 warps:
//   8-11   bring K and V, two warps each, a ring of tiles for each: tensor copies of boxes of a page's slots, the largest power of two that divides
//          pages and tiles, in the layout that the tensor core reads (128-byte swizzle).  Pages that no box of 8 slots fits, or that a tensor
//          map cannot describe, are copied row by row with cp.async, by the four warps in teams, a tile to a team.
//   13-15  copy the queries of the next group.
//   12     issues the products, of scores and with V, whichever has its operands.
//   0-7    softmax, a thread a row, in fp32; p goes back to tensor memory as bf16 over its scores, where it is the A operand of the product
//          with V.  The two forms of the kernel differ in what the two sets of four warps take:
//     128 rows a tile: the first four take the states 0-63 of a tile, the others 64-127, each with a running maximum and sum and an output in
//          tensor memory of its own, so that neither waits for the other but at a group's end, where the two become one.  Scores have two buffers.
//     256 rows a tile: the first four take the rows 0-127, the others 128-255.  K and V are read once for twice the rows, and one half's products
//          run during the other's softmax; the product with V begins when the first 64 states have their p.
//   256 rows are taken where the sequences have more than 128 on average.  us, 256 rows | 128 rows, 32 heads on 8 of 128: 4096 tokens of a prompt
//   194 | 246, 40 tokens over 131071 states 139 | 173, 64 sequences of up to 64 tokens and 4096 states 180 | 204; where it does not matter:
//   512 tokens 28.0 | 27.5, 33 tokens over 1000 states 18.2 | 16.9.  The average says little of a mix: a piece of 1024 tokens of 9001 with 63 sequences of one
//   token and 4096 states goes by tiles of 128, 321 us, where the two by themselves take 161 and 178.
//   Of 256 rows x 128 states some 3200 cycles are left beside the 2048 of the tensor core at its full rate: a half's softmax takes 2100 (exponentials
//   1450, 1024 at the special function unit's rate; maxima 450), its next scores come some 1300 after its p.
// Bits of p: rounded to one bf16 number for the product with V (the sum of p is fp32 and takes it unrounded).  The error against 64 bits is then 2.1 -
// 2.3e-3 of the result's norm, where the rounding of the result alone makes 1.64 - 1.67e-3.  Two numbers, which hold 16 of p's bits, as in tq_paged_attention
// for one token, leave the result's rounding alone, but want a second product: the kernel is not bound by the tensor core, but a tile's chain
// gets longer by it, and at the power limit the clock lower.  One | two (us, in a graph): 8 ragged 37.3 | 39.1, 131071 states 110.5 | 117.8, 64 chains 398 -
// 403 | 441 - 494, pieces of prompts 191 - 213 | 249 - 265; only calls of a few tiles lose nothing (197 states 12.36 | 12.36).  (The lower parts in lanes 64 - 127 of
// tiles with up to 64 rows, beside a copy of the queries, without a second product: twice the exponentials, 8 ragged 49.)  So it is one.
//
// The output is rescaled only when a row's maximum has grown by more than 2^8 since the last rescaling (online softmax with the rescaling
// delayed up to a threshold, as in the kernel of cross attention): p stays below 2^8, which costs no precision in bf16 or the fp32 sum.
//
// Measured (one B200, 6545 GB/s copied, us): 197 states x 8 tokens, 32 heads of 64 9.7; 8 sequences of up to 16 tokens and 8191 states, 24 heads 35 (its
// bytes: 19); 31 tokens over 131071 states, 32 heads 104 (82); 64 chains of 5 tokens over up to 16384 states, 64 heads 392 (386), 453 under the
// power limit; pieces of 1024 tokens of two prompts up to 9001 long, 32 heads 184, 207 under the limit (operations at the rate of a library product: 106).
//
// States that are not there (past the end, on a page outside the pool) are hidden from all rows, and their values zeros in shared memory.  A state that only
// some rows see enters the others' sums with p = 0; if its value is Inf or NaN that product is NaN, so a row whose sum of p is finite but whose
// output has a NaN is computed again from the states it sees (slow).
//
// Every wait is bounded; one that runs out raises TQ_STATUS_WAIT_EXPIRED, all roles leave their loops and tensor memory is released on
// every path.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "tq_attn_sm100.cuh"
#include "tq_internal.h"
#include "tq_ops_common.cuh"

namespace {

using namespace tq_ops;
using namespace tq_sm100;
using namespace tq_attn;

constexpr uint32_t kRows = 128;    // rows of a product: the lanes of tensor memory
constexpr uint32_t kStates = 128;  // states of a tile
constexpr uint32_t kSide = 64;     // states of a tile that one half of the softmax warps takes
constexpr int kSoftWarps = 8, kLoadWarp = 8, kLoadWarps = 4, kMmaWarp = 12, kQueryWarp = 13, kQueryWarps = 3;
constexpr int kTreeThreads = 512;
// registers a thread: 128 at launch (16 warps of an SM's 65536); the softmax warps hold a row of 64 scores and two of output.  The launch
// checks the kernel's own count: a split above it would wait for ever.
constexpr int kSoftRegs = 192, kOtherRegs = 64;
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kMlSets = 2;    // sets of the rows' maxima and sums that the two halves exchange at a group's end, used in turn
constexpr uint32_t kThere = 16;    // tiles whose words of present states are kept: more than loads run ahead of the softmax
constexpr uint32_t kWideRows = 129;  // rows of a sequence, on average, from which on tiles have 256
constexpr float kRescale = 8.0f;   // log2 of how far p may exceed 1

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
  uint32_t n_tokens, n_seqs, n_q_heads, n_kv_heads, group;
  uint32_t row_bits;  // log2 of a tile's rows: 7 or 8
  bool whole;         // no group is cut
  float scale_log2;
  uint32_t box, boxes;  // slots of a page that one tensor copy brings, copies to a tile of 128 states
  uint32_t* status;
  tq_attn_ws ws;
};

template <int D, bool WIDE>
struct TreeSmem {
  static constexpr uint32_t kSlabs = D / 64;                       // 64 columns = 128 bytes of a swizzled row
  static constexpr uint32_t kTileBytes = kSlabs * kStates * 128;   // queries, keys or values of a tile
  // Buffers of queries, keys and values.  Keys and values have a ring each: values are wanted a softmax later than keys, and in one ring they
  // would wait in slots that keys could use.  More is not better: 128 KB under way on every SM are three times what the memory's latency asks for,
  // and what is beyond that waits in the memory system and lets other accesses (parts, page tables) wait with it.  Measured at head_dim 128 (us, two
  // keys and values | three of each): 64 chains 387 | 423, 131071 states 103.5 | 117.6, 8 ragged 35.0 | 39.2.
  static constexpr uint32_t kQueries = D == 128 ? 1 : 2, kKeys = D == 128 ? 2 : 4, kValues = D == 128 ? 2 : 4;
  // The loading warps of the other path work in teams, a tile to a team in turn: a team waits for its copies and announces them, the others' are
  // under way.
  static constexpr uint32_t kTeams = D == 128 ? 2 : 4;
  static constexpr uint32_t kQueryBytes = (WIDE ? 2 : 1) * kTileBytes;
  static constexpr uint32_t kOffK = kQueries * kQueryBytes, kOffV = kOffK + kKeys * kTileBytes;
  static constexpr uint32_t kOffMisc = kOffV + kValues * kTileBytes;
  // misc: [0] dead flag, [4] tensor-memory base, barriers from 16 on
  static constexpr uint32_t kBarKFull = 16, kBarKEmpty = kBarKFull + 8 * kKeys, kBarVFull = kBarKEmpty + 8 * kKeys, kBarVEmpty = kBarVFull + 8 * kValues;
  static constexpr uint32_t kBarQFull = kBarVEmpty + 8 * kValues, kBarQEmpty = kBarQFull + 8 * kQueries;
  static constexpr uint32_t kBarSFull = kBarQEmpty + 8 * kQueries, kBarPFull = kBarSFull + 16, kBarODone = kBarPFull + 32, kBarMl = kBarODone + 16;
  static constexpr uint32_t kOffPlan = (kBarMl + 8 + 15) / 16 * 16;
  static constexpr uint32_t kOffThere = kOffPlan + 96;
  static constexpr uint32_t kOffMl = kOffThere + kThere * 16;
  static constexpr uint32_t kTotal = kOffMisc + kOffMl + (WIDE ? 0 : kMlSets * 2 * kRows * 8);
  static_assert(kTotal <= 232448, "shared memory of one CTA");
};
// a part of a cut group: [D / 4][128] float4 of output, then the rows' maxima and sums; two of them in a row where tiles have 256 rows
constexpr uint64_t kTreePartFloats = kRows * (128 + 2);

__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, uint32_t bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
               : "memory");
}
// Between a wait for copies by cp.async and an instruction that reads what they have written through the asynchronous proxy.
__device__ __forceinline__ void copies_fence() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// Units that a group counts beside its tiles of states: what its end and the next one's beginning cost the softmax warps.
// (us, 1 | 3 | 5 units: pieces of prompts 193 | 185 | 185, 64 sequences of up to 20 tokens and 4000 states 185 | 155 | 153, 8 chains of 333 tokens 84 | 76 | 77)
constexpr uint32_t kGroupUnits = 3;

// A group of the list of work: tile rt of the rows of sequence b over key-value head kvh.
struct Walk {
  uint32_t b, kvh, rt, row_tiles;
  int32_t lo;       // first row of the sequence
  uint32_t n, len;  // its new tokens and states
  int64_t before;   // states before its new tokens (negative: the first ones have none)
  uint32_t end;     // states that the tile's rows may look at
  uint32_t tiles, unit;  // of states; first unit (kGroupUnits of them, then a unit for each tile)

  __device__ __forceinline__ void enter(const TreeParams& p) {
    const int32_t most = (int32_t)p.n_tokens;
    lo = max(0, min(__ldg(p.first + b), most));
    n = (uint32_t)(max(lo, min(__ldg(p.first + b + 1), most)) - lo);
    const int32_t given = __ldg(p.lens + b);
    const uint64_t cap = min((uint64_t)p.max_pages * p.page_size, (uint64_t)0x7FFFFFFF);
    len = given <= 0 ? 0u : (uint32_t)min((uint64_t)given, cap);
    before = (int64_t)given - n;
    row_tiles = (uint32_t)(((uint64_t)n * p.group + (1u << p.row_bits) - 1u) >> p.row_bits);
  }
  __device__ __forceinline__ void tile(const TreeParams& p) {
    end = len;
    if (p.mask == nullptr) {
      const uint32_t last = (uint32_t)min((uint64_t)n - 1u, ((((uint64_t)rt + 1u) << p.row_bits) - 1u) / p.group);
      end = (uint32_t)max((int64_t)0, min((int64_t)len, before + last + 1));
    }
    tiles = max(1u, (end + kStates - 1u) / kStates);
  }
  // the next sequence with rows, from b on
  __device__ __forceinline__ void settle(const TreeParams& p) {
    for (; b < p.n_seqs; ++b) {
      enter(p);
      if (n != 0u) {
        tile(p);
        return;
      }
    }
  }
  __device__ __forceinline__ void next(const TreeParams& p) {
    unit += tiles + kGroupUnits;
    if (++rt == row_tiles) {
      rt = 0;
      if (++kvh == p.n_kv_heads) {
        kvh = 0;
        ++b;
        settle(p);
        return;
      }
    }
    if (p.mask == nullptr) tile(p);
  }
};

// This CTA's share of the units, found by one warp.
struct Plan {
  uint32_t u0, u1, cut;             // units; whether groups are cut (else the groups that begin in the share are the share)
  uint32_t mean, over;              // CTA i has the units i * mean + min(i, over) and on
  Walk at;                          // first group; at.b = n_seqs: none
  __device__ __forceinline__ uint32_t cta_of(uint32_t u) const { return u < over * (mean + 1u) ? u / (mean + 1u) : over + (u - over * (mean + 1u)) / mean; }
};
static_assert(sizeof(Plan) <= 96 && alignof(Plan) <= 16, "room for the plan");

// Groups are left whole where the longest share is then no more than kWholeTiles tiles above the mean of the shares.
constexpr uint32_t kWholeTiles = 3;
// Where the page table has no room for longer sequences than this, none is cut and the joining kernel is not launched.  us, never cut | cut as the
// lengths have it, 32 / 8 heads of 128, 8 new tokens: 1 sequence of 100 states 9.2 | 10.8, 16 of 500 15.5 | 18.7, 64 of 250 31.6 | 34.5; 512 tokens
// of a prompt 24 | 28; but 1 sequence of 1000 states 17.2 | 14.7, of 760 14.9 | 13.8.  (The lengths are known on the device only: a table wider than its
// sequences, as a program that serves has it, is on the right-hand side of these.)
constexpr uint32_t kNeverCutTiles = 4;

__device__ __forceinline__ Plan make_plan(const TreeParams& p, uint32_t lane) {
  Plan r{};
  Walk w{};
  const uint32_t per = (p.n_seqs + 31u) / 32u, begin = min(lane * per, p.n_seqs), end = min(begin + per, p.n_seqs);
  uint32_t sum = 0, most = 0, least = 0xFFFFFFFFu, groups = 0;  // units and groups of one key-value head
  auto units = [&](uint32_t b) {
    w.b = b;
    w.enter(p);
    uint32_t u = 0;
    for (w.rt = 0; w.rt < w.row_tiles; ++w.rt) {
      w.tile(p);
      u += w.tiles + kGroupUnits;
      most = max(most, w.tiles + kGroupUnits);
      least = min(least, w.tiles + kGroupUnits);
    }
    return u;
  };
  for (uint32_t b = begin; b < end; ++b) {
    sum += units(b);
    groups += w.row_tiles;
  }
  uint32_t incl = sum;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const uint32_t o = __shfl_up_sync(kFull, incl, d);
    if (lane >= (uint32_t)d) incl += o;
  }
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) {
    most = max(most, __shfl_xor_sync(kFull, most, d));
    least = min(least, __shfl_xor_sync(kFull, least, d));
    groups += __shfl_xor_sync(kFull, groups, d);
  }
  const uint32_t total = __shfl_sync(kFull, incl, 31) * p.n_kv_heads;
  r.at.b = p.n_seqs;
  if (total == 0u) return r;
  const uint32_t ctas = min(gridDim.x, total);
  r.mean = total / ctas;
  r.over = total - r.mean * ctas;
  // the longest share without cuts: whole groups of one size, or up to one group over the mean
  const uint32_t longest = most == least ? ((groups * p.n_kv_heads - 1u) / ctas + 1u) * most : r.mean + most;
  r.cut = !p.whole && longest > r.mean + (r.over != 0u ? 1u : 0u) + kWholeTiles;
  if (blockIdx.x >= ctas) return r;
  r.u0 = r.mean * blockIdx.x + min(blockIdx.x, r.over);
  r.u1 = r.u0 + r.mean + (blockIdx.x < r.over ? 1u : 0u);
  const uint32_t owner = __ffs(__ballot_sync(kFull, r.u0 < incl * p.n_kv_heads)) - 1u;
  uint32_t at = (incl - sum) * p.n_kv_heads, b = begin, u = 0;
  if (lane == owner) {
    for (; b < end; ++b) {
      u = units(b);
      if (r.u0 < at + u * p.n_kv_heads) break;
      at += u * p.n_kv_heads;
    }
  }
  w.b = __shfl_sync(kFull, b, owner);
  at = __shfl_sync(kFull, at, owner);
  u = __shfl_sync(kFull, u, owner);
  if (u == 0u || w.b >= p.n_seqs) return r;  // only rows that overlap (first not rising) get here
  w.kvh = (r.u0 - at) / u;
  if (w.kvh >= p.n_kv_heads) return r;  // likewise: their units may have passed 32 bits
  w.unit = at + w.kvh * u;
  w.rt = 0;
  w.enter(p);
  w.tile(p);
  while (w.b < p.n_seqs && (r.u0 >= w.unit + kGroupUnits + w.tiles || (!r.cut && w.unit < r.u0))) w.next(p);
  r.at = w;
  return r;
}

// TMA: K and V come by tensor copies of p.box slots of a page, else by cp.async, row by row.
template <int D, bool TMA, bool WIDE>
__global__ void __launch_bounds__(kTreeThreads, 1)
    tree_attention_kernel(const TreeParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using L = TreeSmem<D, WIDE>;
  extern __shared__ __align__(1024) uint8_t smem[];  // swizzled tiles start on 1024 bytes
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t smem0 = smem_u32(smem), misc = smem0 + L::kOffMisc;
  volatile uint32_t* const dead = reinterpret_cast<uint32_t*>(smem + L::kOffMisc);
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kOffMisc + 4);
  Plan* const s_plan = reinterpret_cast<Plan*>(smem + L::kOffMisc + L::kOffPlan);
  float2* const s_ml = reinterpret_cast<float2*>(smem + L::kOffMisc + L::kOffMl);
  uint32_t* const s_there = reinterpret_cast<uint32_t*>(smem + L::kOffMisc + L::kOffThere);
  // the same in all lanes, and known to be: what depends on it alone stays on the uniform data path
  const uint32_t warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31u;
  auto bar = [&](uint32_t off, uint32_t i) { return misc + off + 8u * i; };

  if (smem0 & 1023u) {  // nothing is placed before it, so this does not happen
    if (threadIdx.x == 0) atomicOr(p.ws.status, TQ_STATUS_WAIT_EXPIRED);
    return;
  }
  if (threadIdx.x == 0) {
    *dead = 0u;
    for (uint32_t i = 0; i < L::kKeys; ++i) {
      mbar_init(bar(L::kBarKFull, i), TMA ? 2 : kLoadWarps / L::kTeams);
      mbar_init(bar(L::kBarKEmpty, i), 1);
    }
    for (uint32_t i = 0; i < L::kValues; ++i) {
      mbar_init(bar(L::kBarVFull, i), TMA ? 2 : kLoadWarps / L::kTeams);
      mbar_init(bar(L::kBarVEmpty, i), 1);
    }
    for (uint32_t i = 0; i < L::kQueries; ++i) {
      mbar_init(bar(L::kBarQFull, i), kQueryWarps);
      mbar_init(bar(L::kBarQEmpty, i), 1);
    }
    for (uint32_t i = 0; i < 2; ++i) {
      mbar_init(bar(L::kBarSFull, i), 2);  // the products' completion, and the issuing thread, which has seen the words of present states
      mbar_init(bar(L::kBarPFull, i), WIDE ? kSoftWarps / 2 : kSoftWarps);
      if (WIDE) mbar_init(bar(L::kBarPFull, i + 2u), kSoftWarps / 2);
      mbar_init(bar(L::kBarODone, i), 1);
    }
    mbar_init(bar(L::kBarMl, 0), kSoftWarps);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (TMA && threadIdx.x == 32u * kLoadWarp) {  // the maps are on their way before the first copy wants them
    asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  if (warp == kQueryWarp) {
    const Plan mine = make_plan(p, lane);
    if (lane == 0) *s_plan = mine;
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = *tmem_slot;
  const Plan& plan = *s_plan;

  bool ok = true;
  auto wait = [&](uint32_t b, uint32_t parity) {
    ok = ok && mbar_wait(b, parity, dead);
    ok = __all_sync(kFull, ok);
  };
  Walk g = plan.at;
  // the tiles of states of group w that are this CTA's
  auto in_share = [&](const Walk& w) { return w.b < p.n_seqs && w.unit < plan.u1; };
  auto clip = [&](const Walk& w, uint32_t u) { return u > w.unit + kGroupUnits ? min(u - w.unit - kGroupUnits, w.tiles) : 0u; };
  auto begin_of = [&](const Walk& w) { return plan.cut ? clip(w, plan.u0) : 0u; };
  auto end_of = [&](const Walk& w) { return plan.cut ? clip(w, plan.u1) : w.tiles; };
  // (the share's last group may have none of its tiles in it: then the share has ended)
  auto more = [&](const Walk& w) { return in_share(w) && begin_of(w) < end_of(w); };

  if (warp >= kSoftWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
  if (TMA && warp < kLoadWarp + kLoadWarps) {
    // ---- K and V by tensor copies: two warps for each, which share a tile's boxes, a lane to a box ------------------
    const uint32_t values = (warp - kLoadWarp) >> 1, part = (warp - kLoadWarp) & 1u;
    const CUtensorMap* const map = values ? &v_map : &k_map;
    uint32_t t = more(g) ? begin_of(g) : 0u, t1 = more(g) ? end_of(g) : 0u;
    // the page of this lane's box of the next tile, asked for one tile ahead of its copies
    bool f_any = false, f_live = false, bad = false;
    uint32_t f_slot = 0, f_kvh = 0, f_valid = 0;
    int32_t f_page = 0;
    auto fetch = [&]() {
      f_any = more(g);
      if (!f_any) return;
      const uint32_t s0 = t * kStates, s = s0 + lane * p.box, pg = s / p.page_size;
      f_live = lane < p.boxes && s < g.end;
      f_slot = s - pg * p.page_size;
      f_kvh = g.kvh;
      f_valid = g.end > s0 ? min(kStates, g.end - s0) : 0u;
      if (f_live) f_page = __ldg(p.page_table + (size_t)g.b * p.max_pages + pg);
      if (t == 0u && lane == 0u && __ldg(p.lens + g.b) > 0 && (uint32_t)__ldg(p.lens + g.b) > g.len) bad = true;
      if (++t == t1) {
        g.next(p);
        if (more(g)) {
          t = begin_of(g);
          t1 = end_of(g);
        }
      }
    };
    const uint32_t ring = values ? L::kValues : L::kKeys, offset = values ? L::kOffV : L::kOffK;
    const uint32_t bar_full = values ? L::kBarVFull : L::kBarKFull, bar_empty = values ? L::kBarVEmpty : L::kBarKEmpty;
    uint32_t st = 0, round = 0, count = 0;
    fetch();
    while (f_any && ok) {
      const uint32_t kvh = f_kvh, slot = f_slot, valid = f_valid;
      const int32_t page = f_page;
      const bool live = f_live && (uint32_t)page < p.n_pages, absent = f_live && !live;
      bad = bad || absent;
      fetch();
      const uint32_t there = __ballot_sync(kFull, live);
      if (warp == kLoadWarp && lane < 4u) {  // states that are there, 32 to a word
        uint32_t word = low_bits((int)valid - 32 * (int)lane);
        if ((uint32_t)__popc(there) * p.box < valid) {  // a page outside the pool
          for (uint32_t i = 0; i < 32u; ++i)
            if (!((there >> ((lane * 32u + i) / p.box)) & 1u)) word &= ~(1u << i);
        }
        s_there[(count % kThere) * 4u + lane] = word;
      }
      ++count;
      if (round) wait(bar(bar_empty, st), (round - 1u) & 1u);
      if (!ok) break;
      // columns of 64 to a warp, or, where there are no more, boxes in turn
      const bool mine = L::kSlabs == 2u ? live : live && (lane & 1u) == part;
      const uint32_t slab = L::kSlabs == 2u ? part : 0u;
      const uint32_t full = bar(bar_full, st), dst = smem0 + offset + st * L::kTileBytes + slab * kStates * 128u + lane * p.box * 128u;
      const uint32_t bytes = (uint32_t)__popc(__ballot_sync(kFull, mine)) * p.box * 128u;
      // a box on a page outside the pool: zeros, for values (0 x what the stage held before may be NaN; scores are hidden whatever they are)
      uint32_t gone = values ? __ballot_sync(kFull, L::kSlabs == 2u ? absent : absent && (lane & 1u) == part) : 0u;
      if (gone) {
        for (; gone; gone &= gone - 1u) {
          uint8_t* const box = smem + offset + st * L::kTileBytes + slab * kStates * 128u + (__ffs(gone) - 1u) * p.box * 128u;
          for (uint32_t i = lane; i < p.box * 8u; i += 32u) reinterpret_cast<uint4*>(box)[i] = make_uint4(0u, 0u, 0u, 0u);
        }
        copies_fence();
      }
      __syncwarp();  // the words of present states are written
      if (lane == 0) mbar_expect_tx(full, bytes);
      __syncwarp();
      if (mine) tma_load_4d(dst, map, (int)(slab * 64u), (int)slot, (int)kvh, page, full);
      __syncwarp();
      if (++st == ring) {
        st = 0;
        ++round;
      }
    }
    if (warp == kLoadWarp && __any_sync(kFull, bad) && lane == 0u && p.status != nullptr) atomicOr(p.status, TQ_STATUS_BAD_PAGE);
  } else if (warp < kLoadWarp + kLoadWarps) {
    // ---- K and V ----------------------------------------------------------------------------------------
    constexpr uint32_t kTeams = L::kTeams, kTeamWarps = kLoadWarps / kTeams, kMine = kStates / kTeamWarps, kLanes = kMine / 32u;  // states of a warp, of a lane
    const uint32_t team = (warp - kLoadWarp) / kTeamWarps, s_mine = (warp - kLoadWarp) % kTeamWarps * kMine;
    uint32_t t = more(g) ? begin_of(g) : 0u, t1 = more(g) ? end_of(g) : 0u;
    auto step = [&]() {  // to the next tile
      if (!more(g) || ++t < t1) return;
      g.next(p);
      if (more(g)) {
        t = begin_of(g);
        t1 = end_of(g);
      }
    };
    for (uint32_t i = 0; i < team; ++i) step();
    // the pages of this lane's states of the team's next tile, asked for one tile ahead of its copies
    bool f_any = false, bad = false;
    uint32_t f_slot[kLanes], f_kvh = 0, f_live = 0;
    int32_t f_page[kLanes];
    auto fetch = [&]() {
      f_any = more(g);
      if (!f_any) return;
      f_kvh = g.kvh;
      f_live = 0u;
#pragma unroll
      for (uint32_t i = 0; i < kLanes; ++i) {
        const uint32_t s = t * kStates + s_mine + i * 32u + lane, pg = s / p.page_size;
        f_slot[i] = s - pg * p.page_size;
        f_page[i] = 0;
        if (s < g.end) {
          f_live |= 1u << i;
          f_page[i] = __ldg(p.page_table + (size_t)g.b * p.max_pages + pg);
        }
      }
      if (t == 0u && lane == 0u && __ldg(p.lens + g.b) > 0 && (uint32_t)__ldg(p.lens + g.b) > g.len) bad = true;
      for (uint32_t i = 0; i < kTeams; ++i) step();
    };
    constexpr uint32_t kChunks = D / 8, kAtOnce = 32 / kChunks;  // 16 bytes of a row; rows of a warp-wide copy
    // A lane copies the same 16 bytes of rows lane / kChunks, + kAtOnce, ...: the swizzle turns the place in a row with the row's last three
    // bits, of which kAtOnce's own are the lane's and the others the loop's.
    const uint32_t c = lane % kChunks, r_mine = lane / kChunks;
    const uint32_t place = smem0 + (c / 8u) * (kStates * 128u) + (s_mine + r_mine) * 128u + (((c % 8u) ^ r_mine) << 4);
    const char* const k_mine = reinterpret_cast<const char*>(p.k + c * 8u);
    const int64_t k_to_v = reinterpret_cast<const char*>(p.v) - reinterpret_cast<const char*>(p.k);
    uint32_t count = team;  // tile
    fetch();
    while (f_any && ok) {
      int64_t off[kLanes];  // bytes
      uint32_t there[kLanes];
#pragma unroll
      for (uint32_t i = 0; i < kLanes; ++i) {
        bool live = (f_live >> i) & 1u;
        if (live && (uint32_t)f_page[i] >= p.n_pages) {
          live = false;
          bad = true;
        }
        off[i] = live ? 2 * ((int64_t)f_page[i] * p.page_stride + (int64_t)f_kvh * p.head_stride + (int64_t)f_slot[i] * p.slot_stride) : 0;
        there[i] = __ballot_sync(kFull, live);
      }
      fetch();
      const uint32_t k_round = count / L::kKeys, k_st = count - k_round * L::kKeys, v_round = count / L::kValues, v_st = count - v_round * L::kValues;
      if (k_round) wait(bar(L::kBarKEmpty, k_st), (k_round - 1u) & 1u);
      if (v_round && ok) wait(bar(L::kBarVEmpty, v_st), (v_round - 1u) & 1u);
      if (!ok) break;
#pragma unroll
      for (uint32_t i = 0; i < kLanes; ++i) {
        if (lane == 0) s_there[(count % kThere) * 4u + s_mine / 32u + i] = there[i];
        const uint32_t k_dst = place + L::kOffK + k_st * L::kTileBytes + i * 4096u, v_dst = place + L::kOffV + v_st * L::kTileBytes + i * 4096u;
        auto copy = [&](bool all) {
#pragma unroll
          for (uint32_t r0 = 0; r0 < 32u; r0 += kAtOnce) {
            const char* const from = k_mine + __shfl_sync(kFull, off[i], r0 + r_mine);
            const uint32_t turn = (r0 & 7u) << 4, bytes = all || ((there[i] >> (r0 + r_mine)) & 1u) ? 16u : 0u;  // 0: zeros, nothing is read
            cp_async16((k_dst ^ turn) + r0 * 128u, from, bytes);
            cp_async16((v_dst ^ turn) + r0 * 128u, from + k_to_v, bytes);
          }
        };
        if (there[i] == 0xFFFFFFFFu)
          copy(true);
        else
          copy(false);
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(bar(L::kBarKFull, k_st));
        mbar_arrive(bar(L::kBarVFull, v_st));
      }
      count += kTeams;
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
    if (bad && p.status != nullptr) atomicOr(p.status, TQ_STATUS_BAD_PAGE);
  } else if (warp >= kQueryWarp) {
    // ---- queries ----------------------------------------------------------------------------------------
    constexpr uint32_t kChunks = D / 8, kAtOnce = 32 / kChunks;
    const uint32_t c = lane % kChunks;
    uint32_t count = 0;
    uint4 open = make_uint4(0u, 0u, 0u, 0u);  // the last group that begins in this share, the only one that can go on in the next
    for (; more(g) && ok; g.next(p)) {
      const uint32_t qb = count % L::kQueries;
      if (count >= L::kQueries) wait(bar(L::kBarQEmpty, qb), (count / L::kQueries - 1u) & 1u);
      if (!ok) break;
      const uint32_t first = g.rt << p.row_bits, rows = (uint32_t)min((uint64_t)1 << p.row_bits, (uint64_t)g.n * p.group - first);
      const uint32_t dst = smem0 + qb * L::kQueryBytes + (c / 8u) * (kRows * 128u);
      const __nv_bfloat16* const q = p.q + (int64_t)g.lo * p.q_stride + (size_t)g.kvh * p.group * D + c * 8u;
      // rows that are not there are zeros: products with them draw less power (64 chains of 40 rows: 1500 MHz under the power limit without that)
      for (uint32_t r = (warp - kQueryWarp) * kAtOnce + lane / kChunks; r < (WIDE ? 2u : 1u) * kRows; r += kQueryWarps * kAtOnce) {
        const uint32_t row = first + min(r, rows - 1u), tok = row / p.group;
        cp_async16(dst + (r / kRows) * L::kTileBytes + (r % kRows) * 128u + (((c % 8u) ^ (r & 7u)) << 4), q + (int64_t)tok * p.q_stride + (row - tok * p.group) * D, r < rows ? 16u : 0u);
      }
      asm volatile("cp.async.wait_all;" ::: "memory");
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(L::kBarQFull, qb));
      ++count;
      open = make_uint4(0u, (uint32_t)g.lo, g.kvh, g.rt);
      if (begin_of(g) == 0u && end_of(g) < g.tiles) open.x = plan.cta_of(g.unit + kGroupUnits + g.tiles - 1u) - blockIdx.x + 1u | rows << 16;
    }
    if (warp == kQueryWarp && lane == 0) p.ws.open[blockIdx.x] = open;  // for the joining kernel
  } else if (warp == kMmaWarp) {
    // ---- products ---------------------------------------------------------------------------------------
    // past the last state memory may hold anything, and 0 x NaN is NaN
    auto zero_behind = [&](uint32_t st, uint32_t valid) {
      if (valid == kStates) return;
      constexpr uint32_t kChunks = D / 8, kStep = 32 / kChunks;  // of 16 bytes of a row; rows at once
      const uint32_t c = lane % kChunks;
      uint8_t* const tile = smem + L::kOffV + st * L::kTileBytes + (c / 8u) * (kStates * 128u) + (c % 8u) * 16u;
#pragma unroll 4
      for (uint32_t r = valid + lane / kChunks; r < kStates; r += kStep) *reinterpret_cast<uint4*>(tile + r * 128u) = make_uint4(0, 0, 0, 0);
      copies_fence();
    };
    // Scores of the next tile or the product of an earlier one with V, whichever is ready: up to two tiles' scores may wait for their p.
    uint32_t done = 0, asked = 0, q_count = 0;  // tiles multiplied with V, tiles with scores, groups
    uint32_t k_st = 0, k_round = 0, v_st = 0, v_round = 0;
    uint32_t flags[2] = {0, 0};  // of the tiles in between, by buffer: 1: not the group's first tile; states that are there << 8
    const uint32_t idesc_qk = umma_idesc(128, 128), idesc_pv = umma_idesc(128, D) | kIdescNMajorB;
    const uint64_t q_desc = umma_desc(smem0), k_desc = umma_desc(smem0 + L::kOffK), v_desc = umma_desc_n_major(smem0 + L::kOffV, kStates);
    bool any = more(g);
    uint32_t t = any ? begin_of(g) : 0u, t0 = t, t1 = any ? end_of(g) : 0u;
    if constexpr (WIDE) {
      // Two products a tile, in turn: while one half's softmax is taken the other's scores and its product with V are formed.
      bool pending = false;  // a tile with scores waits for its p
      uint32_t states = 0, adds = 0;  // of it: states that are there, whether it is not the group's first
      auto product = [&](uint32_t r) {
        if (r == 0u) {
          wait(bar(L::kBarVFull, v_st), v_round & 1u);
          if (!ok) return;
          if (TMA)
            zero_behind(v_st, states);
          else
            copies_fence();
        }
#pragma unroll 1
        for (uint32_t h = 0; h < 2u; ++h) {  // the first half of the states while p of the second is being taken
          wait(bar(L::kBarPFull, 2u * r + h), done & 1u);
          if (!ok) return;
          tmem_fence_after();
          __syncwarp();
          if (elect_one()) {
            const uint64_t b = v_desc + v_st * (L::kTileBytes >> 4) + h * (4u * 2048u >> 4);
#pragma unroll
            for (uint32_t kk = 0; kk < kStates / 32u; ++kk)
              umma_bf16_ts(tmem + 2u * kStates + r * D, tmem + r * kStates + (4u * h + kk) * 8u, b + kk * (2048u >> 4), idesc_pv, adds | h | kk);
            if (h == 1u) {
              umma_commit(bar(L::kBarODone, r));
              if (r == 1u) umma_commit(bar(L::kBarVEmpty, v_st));
            }
          }
          __syncwarp();
        }
        if (r == 0u) return;
        ++done;
        if (++v_st == L::kValues) {
          v_st = 0;
          ++v_round;
        }
      };
      auto scores = [&](uint32_t r) {
        const uint32_t qb = q_count % L::kQueries;
        if (r == 0u) {
          wait(bar(L::kBarKFull, k_st), k_round & 1u);
          if (t == t0 && ok) wait(bar(L::kBarQFull, qb), (q_count / L::kQueries) & 1u);
        }
        if (!ok) return;
        if (!TMA || t == t0) copies_fence();
        tmem_fence_after();
        if (elect_one()) {
          const uint64_t a = q_desc + (qb * L::kQueryBytes + r * L::kTileBytes >> 4), b = k_desc + k_st * (L::kTileBytes >> 4);
#pragma unroll
          for (uint32_t kk = 0; kk < D / 16; ++kk) {
            constexpr uint32_t kSlab = (kStates * 128u) >> 4;
            const uint32_t off = (kk / 4u) * kSlab + (kk % 4u) * 2u;  // in 16 bytes
            umma_bf16(tmem + r * kStates, a + off, b + off, idesc_qk, kk != 0u);
          }
          umma_commit(bar(L::kBarSFull, r));
          if (r == 1u) umma_commit(bar(L::kBarKEmpty, k_st));
          if (r == 1u && t + 1u == t1) umma_commit(bar(L::kBarQEmpty, qb));
          mbar_arrive(bar(L::kBarSFull, r));
        }
        __syncwarp();
      };
      while (ok && (any || pending)) {
        const bool same = any && t != t0;  // the next tile is of the pending one's group: its queries are there
#pragma unroll 1
        for (uint32_t r = 0; r < 2u && ok; ++r) {
          if (pending) product(r);
          if (same && ok) scores(r);
        }
#pragma unroll 1
        for (uint32_t r = 0; r < 2u && ok && any && !same; ++r) scores(r);
        pending = any;
        if (!any) break;
        states = g.end > t * kStates ? min(kStates, g.end - t * kStates) : 0u;
        adds = same ? 1u : 0u;
        if (++k_st == L::kKeys) {
          k_st = 0;
          ++k_round;
        }
        if (++t == t1) {
          g.next(p);
          ++q_count;
          any = more(g);
          if (any) {
            t = t0 = begin_of(g);
            t1 = end_of(g);
          }
        }
      }
    } else {
      uint32_t idle = 0;
      while (ok && (any || done != asked)) {
        const uint32_t sb = done & 1u;
        // the tile's p times V, both halves of its states
        if (done != asked && mbar_test(bar(L::kBarPFull, sb), (done >> 1) & 1u) && mbar_test(bar(L::kBarVFull, v_st), v_round & 1u)) {
          idle = 0;
          if (TMA) {
            zero_behind(v_st, flags[sb] >> 8);
          }
          copies_fence();
          tmem_fence_after();
          __syncwarp();
          if (elect_one()) {
            const uint64_t b = v_desc + v_st * (L::kTileBytes >> 4);
#pragma unroll
            for (uint32_t kk = 0; kk < kStates / 16u; ++kk) {
              const uint32_t w = kk / 4u;
              umma_bf16_ts(tmem + 2u * kStates + w * D, tmem + sb * kStates + w * kSide + (kk % 4u) * 8u, b + kk * (2048u >> 4), idesc_pv,
                           (flags[sb] & 1u) | (kk % 4u));
            }
            umma_commit(bar(L::kBarODone, sb));
            umma_commit(bar(L::kBarVEmpty, v_st));
          }
          __syncwarp();
          ++done;
          if (++v_st == L::kValues) {
            v_st = 0;
            ++v_round;
          }
          continue;
        }
        // the next tile's scores, when the buffer's last p is spent
        if (any && asked - done < 2u && mbar_test(bar(L::kBarKFull, k_st), k_round & 1u) &&
            (t != t0 || mbar_test(bar(L::kBarQFull, q_count % L::kQueries), (q_count / L::kQueries) & 1u))) {
          idle = 0;
          const uint32_t qb = q_count % L::kQueries, to = asked & 1u;
          copies_fence();
          tmem_fence_after();
          if (elect_one()) {
            const uint64_t a = q_desc + qb * (L::kTileBytes >> 4), b = k_desc + k_st * (L::kTileBytes >> 4);
#pragma unroll
            for (uint32_t kk = 0; kk < D / 16; ++kk) {
              constexpr uint32_t kSlab = (kStates * 128u) >> 4;
              const uint32_t off = (kk / 4u) * kSlab + (kk % 4u) * 2u;  // in 16 bytes
              umma_bf16(tmem + to * kStates, a + off, b + off, idesc_qk, kk != 0u);
            }
            umma_commit(bar(L::kBarSFull, to));
            umma_commit(bar(L::kBarKEmpty, k_st));
            if (t + 1u == t1) umma_commit(bar(L::kBarQEmpty, qb));
            mbar_arrive(bar(L::kBarSFull, to));
          }
          __syncwarp();
          if (++k_st == L::kKeys) {
            k_st = 0;
            ++k_round;
          }
          const uint32_t f = (t != t0 ? 1u : 0u) | (g.end > t * kStates ? min(kStates, g.end - t * kStates) << 8 : 0u);
          if (to)
            flags[1] = f;
          else
            flags[0] = f;
          ++asked;
          if (++t == t1) {
            g.next(p);
            ++q_count;
            any = more(g);
            if (any) {
              t = t0 = begin_of(g);
              t1 = end_of(g);
            }
          }
          continue;
        }
        if (++idle == kSpinLimit || ((idle & 1023u) == 1023u && *dead)) ok = false;
        ok = __all_sync(kFull, ok);
      }
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    // ---- softmax: a thread a row, half the states ---------------------------------------------------------
    const uint32_t w = warp >> 2, row_in = threadIdx.x & 127u;
    const uint32_t lane_field = (warp & 3u) << 21;  // 32 lanes of tensor memory to a warp
    const uint32_t o_addr = tmem + lane_field + 2u * kStates;
    constexpr uint32_t kParts = WIDE ? 1 : 2;  // threads of a row at the group's end, each with its part of the columns
    const float c = p.scale_log2;
    uint32_t count = 0, groups = 0;
    for (; more(g) && ok; g.next(p), ++groups) {
      const uint32_t t0 = begin_of(g), t1 = end_of(g);
      const uint64_t rows = (uint64_t)g.n * p.group;
      const uint64_t row = ((uint64_t)g.rt << p.row_bits) + (WIDE ? threadIdx.x : row_in);
      const bool live = row < rows, warp_live = row - lane < rows;
      const uint32_t tok = live ? (uint32_t)row / p.group : 0u, head = g.kvh * p.group + ((uint32_t)row - tok * p.group);
      const uint32_t* const bits_row = p.mask ? p.mask + (size_t)(g.lo + (int32_t)tok) * p.mask_words : nullptr;
      float m = -INFINITY, l = 0.f;
      // bit i: this row sees state s0 + i, as far as the order of the new tokens goes
      auto visible = [&](int64_t s0) -> uint64_t {
        const int64_t j0 = s0 - g.before;  // new token of the first of the 64 states
        if (j0 <= -(int64_t)kSide) return ~0ull;
        if (bits_row == nullptr) {
          const int64_t n = (int64_t)tok + 1 - j0;
          return n <= 0 ? 0ull : n >= 64 ? ~0ull : (1ull << n) - 1ull;
        }
        const int64_t from = max((int64_t)0, j0);
        const uint32_t word = (uint32_t)(from >> 5), off = (uint32_t)from & 31u;
        auto at = [&](uint32_t i) { return (int64_t)(from >> 5) + i < p.mask_words ? __ldg(bits_row + word + i) : 0u; };
        const uint32_t a = at(0), b = at(1), e = at(2);
        const uint64_t v = ((uint64_t)__funnelshift_r(b, e, off) << 32) | __funnelshift_r(a, b, off);
        return j0 >= 0 ? v : (v << -j0) | ((1ull << -j0) - 1ull);
      };
      if constexpr (WIDE) {
        const uint32_t s_addr = tmem + lane_field + w * kStates;
        for (uint32_t t = t0; t < t1; ++t, ++count) {
          const uint64_t order[2] = {warp_live ? visible((int64_t)t * kStates) : 0ull, warp_live ? visible((int64_t)t * kStates + kSide) : 0ull};
          wait(bar(L::kBarSFull, w), count & 1u);
          if (!ok) break;
          tmem_fence_after();
          if (warp_live) {
            const uint4 here = *reinterpret_cast<const uint4*>(s_there + (count % kThere) * 4u);
            const uint32_t seen[4] = {(uint32_t)order[0] & here.x, (uint32_t)(order[0] >> 32) & here.y, (uint32_t)order[1] & here.z, (uint32_t)(order[1] >> 32) & here.w};
            uint32_t s[kStates];
#pragma unroll
            for (int i = 0; i < 4; ++i) TMEM_LD32(s + 32 * i, s_addr + 32u * i);
            tmem_wait_ld();
            if (__any_sync(kFull, (seen[0] & seen[1] & seen[2] & seen[3]) != ~0u)) {
#pragma unroll
              for (int i = 0; i < 128; ++i) s[i] = (seen[i / 32] >> (i % 32)) & 1u ? s[i] : 0xFF800000u;
            }
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < 128; i += 8) {
#pragma unroll
              for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], __uint_as_float(s[i + 2 * k]), __uint_as_float(s[i + 2 * k + 1]));
            }
            const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]) * c;
            if (__any_sync(kFull, live && top > m + kRescale)) {
              const float mn = fmaxf(m, top), f = mn == -INFINITY ? 1.f : exp2_fast(m - mn);
              m = mn;
              l *= f;
              if (t != t0) {
                wait(bar(L::kBarODone, w), (count - 1u) & 1u);
                if (!ok) break;
                tmem_fence_after();
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                  uint32_t o[16];
                  TMEM_LD16(o, o_addr + w * D + 16u * i);
                  tmem_wait_ld();
#pragma unroll
                  for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                  TMEM_ST16(o_addr + w * D + 16u * i, o);
                }
              }
            }
            const float ref = !live ? INFINITY : m == -INFINITY ? 0.f : m;
            const uint64_t c2 = pair(c, c), ref2 = pair(-ref, -ref);
            uint64_t sum[2] = {0, 0};
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              uint32_t pk[16];
#pragma unroll
              for (int i = 0; i < 16; ++i) {
                float a, b;
                unpair(fma2(pair(__uint_as_float(s[32 * h + 2 * i]), __uint_as_float(s[32 * h + 2 * i + 1])), c2, ref2), a, b);
                a = exp2_fast(a);
                b = exp2_fast(b);
                sum[i & 1] = add2(sum[i & 1], pair(a, b));
                pk[i] = pack_bf16(a, b);
              }
              TMEM_ST16(s_addr + 16u * h, pk);
              if (h == 1) {
                tmem_wait_st();
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(L::kBarPFull, 2u * w));
              }
            }
            float l0, l1;
            unpair(add2(sum[0], sum[1]), l0, l1);
            l += l0 + l1;
            tmem_wait_st();
          }
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) {
            if (!warp_live) mbar_arrive(bar(L::kBarPFull, 2u * w));
            mbar_arrive(bar(L::kBarPFull, 2u * w + 1u));
          }
        }
        if (ok) wait(bar(L::kBarODone, w), (count - 1u) & 1u);
        if (!ok) break;
      } else {
        for (uint32_t t = t0; t < t1; ++t, ++count) {
          const uint32_t sb = count & 1u, s_addr = tmem + lane_field + sb * kStates + w * kSide;
          const uint64_t order = warp_live ? visible((int64_t)t * kStates + w * kSide) : 0ull;
          wait(bar(L::kBarSFull, sb), (count >> 1) & 1u);
          if (!ok) break;
          tmem_fence_after();
          if (warp_live) {
            const uint2 here = *reinterpret_cast<const uint2*>(s_there + (count % kThere) * 4u + w * 2u);
            const uint64_t seen = order & (((uint64_t)here.y << 32) | here.x);
            uint32_t s[kSide];
            TMEM_LD32(s, s_addr);
            TMEM_LD32(s + 32, s_addr + 32u);
            tmem_wait_ld();
            if (__any_sync(kFull, seen != ~0ull)) {
              const uint32_t lo = (uint32_t)seen, hi = (uint32_t)(seen >> 32);
#pragma unroll
              for (int i = 0; i < 64; ++i) s[i] = ((i < 32 ? lo : hi) >> (i % 32)) & 1u ? s[i] : 0xFF800000u;
            }
            float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
            for (int i = 0; i < 64; i += 8) {
#pragma unroll
              for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], __uint_as_float(s[i + 2 * k]), __uint_as_float(s[i + 2 * k + 1]));
            }
            const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]) * c;
            if (__any_sync(kFull, live && top > m + kRescale)) {  // (what lies in a dead row must not decide for the others)
              const float mn = fmaxf(m, top), f = mn == -INFINITY ? 1.f : exp2_fast(m - mn);
              m = mn;
              l *= f;
              if (t != t0) {
                wait(bar(L::kBarODone, sb ^ 1u), ((count - 1u) >> 1) & 1u);  // the products with V up to the tile before
                if (!ok) break;
                tmem_fence_after();
#pragma unroll
                for (int i = 0; i < D / 16; ++i) {
                  uint32_t o[16];
                  TMEM_LD16(o, o_addr + w * D + 16u * i);
                  tmem_wait_ld();
#pragma unroll
                  for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
                  TMEM_ST16(o_addr + w * D + 16u * i, o);
                }
              }
            }
            const float ref = !live ? INFINITY : m == -INFINITY ? 0.f : m;  // p of a dead row is 0
            const uint64_t c2 = pair(c, c), ref2 = pair(-ref, -ref);
            uint64_t sum[2] = {0, 0};
            uint32_t pk[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
              float a, b;
              unpair(fma2(pair(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), c2, ref2), a, b);
              a = exp2_fast(a);
              b = exp2_fast(b);
              sum[i & 1] = add2(sum[i & 1], pair(a, b));
              pk[i] = pack_bf16(a, b);
            }
            TMEM_ST32(s_addr, pk);
            float l0, l1;
            unpair(add2(sum[0], sum[1]), l0, l1);
            l += l0 + l1;
            tmem_wait_st();
          }
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(L::kBarPFull, sb));
        }
        if (!ok) break;
        // ---- end of the group, or of this CTA's part of it: the two halves of the states become one ---------------
        // Two sets, in turn.  A warp is a group ahead of its partner at most: the next tile's scores wait for the product before the last, not for the
        // partner's reading of this group, so where the next group has one or two tiles here it may write its entries while the partner still reads
        // these.  Two groups ahead it cannot be: the wait below, of the group between, is for the partner's arrival, which follows its reading.
        float2* const ml = s_ml + groups % kMlSets * 2u * kRows;
        ml[w * kRows + row_in] = make_float2(m, l);
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(L::kBarMl, 0));
        wait(bar(L::kBarODone, (count - 1u) & 1u), ((count - 1u) >> 1) & 1u);
        if (ok) wait(bar(L::kBarMl, 0), groups & 1u);
        if (!ok) break;
      }
      if (!warp_live) continue;
      tmem_fence_after();
      float M = m, fa = 1.f, fb = 0.f, sum = l;
      if constexpr (!WIDE) {
        const float2* const ml = s_ml + groups % kMlSets * 2u * kRows;
        const float2 a = ml[row_in], b = ml[kRows + row_in];
        M = fmaxf(a.x, b.x);
        const float ref = M == -INFINITY ? 0.f : M;
        fa = exp2_fast(a.x - ref), fb = exp2_fast(b.x - ref), sum = a.y * fa + b.y * fb;
      }
      const float ref = M == -INFINITY ? 0.f : M;
      const bool whole = t0 == 0u && t1 == g.tiles;
      float* const mine = p.ws.parts + (size_t)((2u * blockIdx.x + (t0 == 0u ? 1u : 0u)) * (WIDE ? 2u : 1u) + (WIDE ? w : 0u)) * kTreePartFloats;
      const size_t at = (size_t)(g.lo + (int32_t)tok) * p.n_q_heads + head;
      const float inv = 1.0f / sum;
      bool nan = false;
      constexpr uint32_t kColumns = D / kParts;  // of a row, for each of its threads
      const uint32_t col0 = WIDE ? 0u : w * kColumns;
#pragma unroll
      for (uint32_t i = 0; i < kColumns; i += 32u) {
        const uint32_t col = col0 + i;
        uint32_t x[32], y[32];
        TMEM_LD32(x, o_addr + (WIDE ? w * D : 0u) + col);
        if constexpr (!WIDE) TMEM_LD32(y, o_addr + D + col);
        tmem_wait_ld();
#pragma unroll
        for (int k = 0; k < 32; ++k) {
          const float o = WIDE ? __uint_as_float(x[k]) : __uint_as_float(x[k]) * fa + __uint_as_float(y[k]) * fb;
          nan = nan || o != o;
          x[k] = __float_as_uint(o);
        }
        if (!live) continue;
        if (whole) {
#pragma unroll
          for (int k = 0; k < 32; k += 8) {
            float f[8];
#pragma unroll
            for (int z = 0; z < 8; ++z) f[z] = sum == 0.f ? 0.f : __uint_as_float(x[k + z]) * inv;
            store8<TQ_TYPE_BF16>(p.out, at * D + col + k, f);
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k)
            reinterpret_cast<uint4*>(mine)[(col / 4u + k) * kRows + row_in] = make_uint4(x[4 * k], x[4 * k + 1], x[4 * k + 2], x[4 * k + 3]);
        }
      }
      if (live && (WIDE || w == 0u)) {
        if (!whole) {
          mine[kRows * 128 + row_in] = M;
          mine[kRows * 129 + row_in] = sum;
        } else if (p.lse) {
          p.lse[at] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * 0.6931471805599453f;
        }
      }
      // rows that a state they do not see has spoiled: again, a warp a row
      uint32_t again = __ballot_sync(kFull, live && nan && sum < INFINITY);
#pragma unroll 1
      while (again) {
        const int src = __ffs(again) - 1;
        again &= again - 1u;
        constexpr int kPer = D / 32, kOwn = kPer / kParts;  // elements of a row a lane, and of this warp's part of it
        const uint32_t rt = __shfl_sync(kFull, tok, src), rh = __shfl_sync(kFull, head, src), rs = __shfl_sync(kFull, row_in, src);
        const float rm = __shfl_sync(kFull, ref, src), rl = __shfl_sync(kFull, sum, src);
        const __nv_bfloat16* q = p.q + (int64_t)(g.lo + (int32_t)rt) * p.q_stride + (size_t)rh * D + lane * kPer;
        float acc[kOwn], qv[kPer];
#pragma unroll
        for (int i = 0; i < kOwn; ++i) acc[i] = 0.f;
#pragma unroll
        for (int i = 0; i < kPer; ++i) qv[i] = __bfloat162float(q[i]);
        const uint32_t s1 = min(t1 * kStates, g.end);
#pragma unroll 1
        for (uint32_t s0 = t0 * kStates; s0 < s1; s0 += 32u) {  // a lane looks a state up; four of those that are seen are loaded together
          const uint32_t s = s0 + lane, pg = s / p.page_size;
          const int64_t j = (int64_t)s - g.before;
          bool seen = s < s1;
          if (seen && j >= 0)
            seen = p.mask ? (j >> 5) < (int64_t)p.mask_words && ((__ldg(p.mask + (size_t)(g.lo + (int32_t)rt) * p.mask_words + (j >> 5)) >> (j & 31)) & 1u) != 0u
                          : j <= (int64_t)rt;
          int64_t place = 0;
          if (seen) {
            const int32_t page = __ldg(p.page_table + (size_t)g.b * p.max_pages + pg);
            seen = (uint32_t)page < p.n_pages;
            place = (int64_t)page * p.page_stride + (int64_t)g.kvh * p.head_stride + (int64_t)(s - pg * p.page_size) * p.slot_stride;
          }
          uint32_t left = __ballot_sync(kFull, seen);
#pragma unroll 1
          while (left) {
            constexpr int kAtOnce = 4;
            int64_t from[kAtOnce];
            float x[kAtOnce], v[kAtOnce][kOwn];
            bool on[kAtOnce];
#pragma unroll
            for (int z = 0; z < kAtOnce; ++z) {
              on[z] = left != 0u;
              from[z] = __shfl_sync(kFull, (long long)place, on[z] ? __ffs(left) - 1 : 0);
              left &= left - 1u;
            }
#pragma unroll
            for (int z = 0; z < kAtOnce; ++z) {
              x[z] = 0.f;
#pragma unroll
              for (int i = 0; i < kPer; ++i) x[z] += on[z] ? qv[i] * __bfloat162float(p.k[from[z] + lane * kPer + i]) : 0.f;
#pragma unroll
              for (int i = 0; i < kOwn; ++i) v[z][i] = on[z] ? __bfloat162float(p.v[from[z] + col0 + lane * kOwn + i]) : 0.f;
            }
#pragma unroll
            for (int z = 0; z < kAtOnce; ++z) {
#pragma unroll
              for (int d = 16; d > 0; d >>= 1) x[z] += __shfl_xor_sync(kFull, x[z], d);
              const float pr = on[z] ? exp2_fast(fmaf(x[z], c, -rm)) : 0.f;
#pragma unroll
              for (int i = 0; i < kOwn; ++i) acc[i] += pr * v[z][i];
            }
          }
        }
        __syncwarp();  // after the row's own thread has written it
#pragma unroll
        for (int i = 0; i < kOwn; ++i) {
          const uint32_t col = col0 + lane * kOwn + i;
          if (whole)
            p.out[((size_t)(g.lo + (int32_t)rt) * p.n_q_heads + rh) * D + col] = __float2bfloat16_rn(rl == 0.f ? 0.f : acc[i] / rl);
          else
            mine[(col / 4u * kRows + rs) * 4u + col % 4u] = acc[i];
        }
      }
    }
  }

  if (!ok) {
    *dead = 1u;
    if (lane == 0) atomicOr(p.ws.status, TQ_STATUS_WAIT_EXPIRED);
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);  // products in flight still read shared memory: give them time to end
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tmem_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// Joins the parts of the groups that were cut.  grid (CTAs of the kernel above, slices of 8 rows): the group whose first tile is in CTA x's share and
// whose last is not, if there is one; a thread has four columns of a row and adds the parts up in their order, kJoinAtOnce of them asked for together.
constexpr uint32_t kJoinRows = 8, kJoinAtOnce = 8;
template <int D, bool WIDE>
__global__ void __launch_bounds__(kJoinRows * D / 4) tree_join_kernel(const TreeParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint4 e = p.ws.open[blockIdx.x];  // parts and rows << 16, first row of the sequence, key-value head, tile of rows
  const uint32_t parts = e.x & 0xFFFFu, slot = blockIdx.y * kJoinRows + threadIdx.x % kJoinRows, quad = threadIdx.x / kJoinRows;
  if (parts < 2u || parts > gridDim.x - blockIdx.x || slot >= e.x >> 16) return;  // none, or not valid after an expired wait
  const uint32_t row = (e.w << p.row_bits) + slot, tok = row / p.group;
  const uint32_t half = WIDE ? slot / kRows : 0u, lane_row = slot % kRows;
  const uint64_t out_row = (uint64_t)e.y + tok;
  if (e.z >= p.n_kv_heads || out_row >= p.n_tokens) return;
  float M = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
  for (uint32_t i0 = 0; i0 < parts; i0 += kJoinAtOnce) {
    float mi[kJoinAtOnce], li[kJoinAtOnce];
    float4 y[kJoinAtOnce];
#pragma unroll
    for (uint32_t i = 0; i < kJoinAtOnce; ++i) {
      const uint32_t at = min(i0 + i, parts - 1u);
      const float* const src = p.ws.parts + (size_t)((2u * (blockIdx.x + at) + (at == 0u ? 1u : 0u)) * (WIDE ? 2u : 1u) + half) * kTreePartFloats;
      mi[i] = __ldcg(src + kRows * 128 + lane_row);
      li[i] = __ldcg(src + kRows * 129 + lane_row);
      y[i] = __ldcg(reinterpret_cast<const float4*>(src) + quad * kRows + lane_row);
    }
#pragma unroll
    for (uint32_t i = 0; i < kJoinAtOnce; ++i) {
      if (i0 + i >= parts) break;
      const float mn = fmaxf(M, mi[i]), ref = mn == -INFINITY ? 0.f : mn, f = exp2_fast(M - ref), h = exp2_fast(mi[i] - ref);
      M = mn;
      l = l * f + li[i] * h;
      o.x = o.x * f + y[i].x * h;
      o.y = o.y * f + y[i].y * h;
      o.z = o.z * f + y[i].z * h;
      o.w = o.w * f + y[i].w * h;
    }
  }
  const size_t at = (size_t)out_row * p.n_q_heads + e.z * p.group + (row - tok * p.group);
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  *reinterpret_cast<uint2*>(p.out + at * D + 4u * quad) =
      l == 0.f ? make_uint2(0u, 0u) : make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
  if (quad == 0u && p.lse) p.lse[at] = l == 0.f ? -INFINITY : (M + log2f(l)) * 0.6931471805599453f;
}

// The tensor map of a pool: (column, slot, head, page), boxes of 64 columns x `box` slots, 128-byte swizzle.
bool encode(CUtensorMap* map, const void* base, const tq_kv_cache* c, uint32_t box) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t row = c->head_dim * 2u;
  const cuuint64_t dims[4] = {c->head_dim, c->page_size, c->n_kv_heads, c->n_pages};
  cuuint64_t strides[3] = {(cuuint64_t)c->slot_stride * 2u, (cuuint64_t)c->head_stride * 2u, (cuuint64_t)c->page_stride * 2u};
  for (int i = 0; i < 3; ++i) {
    if (dims[i + 1] == 1u) strides[i] = row;  // means nothing
    if (strides[i] == 0u) return false;
  }
  const cuuint32_t boxes[4] = {64u, box, 1u, 1u}, step[4] = {1u, 1u, 1u, 1u};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, boxes, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D, bool TMA, bool WIDE>
int launch(const TreeParams& p, const CUtensorMap& k_map, const CUtensorMap& v_map, cudaStream_t st) {
  auto kern = tree_attention_kernel<D, TMA, WIDE>;
  constexpr size_t smem = TreeSmem<D, WIDE>::kTotal;
  const char* what = "tree attention launch";
  if (int rc = tq_ensure_dynamic_smem((const void*)kern, smem, what)) return rc;
  static std::atomic<int> known{0};  // registers a thread; a query that has failed is made again
  int regs = known.load(std::memory_order_relaxed);
  if (regs == 0) {
    cudaFuncAttributes a{};
    if (int rc = tq_cuda_status((int)cudaFuncGetAttributes(&a, (const void*)kern), what)) return rc;
    known.store(regs = a.numRegs, std::memory_order_relaxed);
  }
  if (256 * kSoftRegs + 256 * kOtherRegs > kTreeThreads * regs) return tq_cuda_status((int)cudaErrorInvalidConfiguration, what);
  const uint32_t grid = min((uint32_t)sm_count(), kAttnMaxCtas);
  if (int rc = launch_pdl(kern, dim3(grid), kTreeThreads, smem, st, what, p, k_map, v_map)) return rc;
  if (p.whole) return TQ_OK;
  const uint32_t rows = (uint32_t)min((uint64_t)1 << p.row_bits, (uint64_t)p.n_tokens * p.group);
  return launch_pdl(tree_join_kernel<D, WIDE>, dim3(grid, (rows + kJoinRows - 1u) / kJoinRows), kJoinRows * D / 4, 0, st, "tree attention (join) launch", p);
}

template <int D, bool TMA>
int launch_rows(TreeParams& p, const CUtensorMap& k_map, const CUtensorMap& v_map, cudaStream_t st) {
  const bool wide = (uint64_t)p.n_tokens * p.group >= (uint64_t)kWideRows * p.n_seqs;
  p.row_bits = wide ? 8u : 7u;
  return wide ? launch<D, TMA, true>(p, k_map, v_map, st) : launch<D, TMA, false>(p, k_map, v_map, st);
}

bool misaligned(const void* ptr, uintptr_t align) { return ptr == nullptr || ((uintptr_t)ptr & (align - 1u)) != 0; }

}  // namespace

// two parts a CTA, of 256 rows
uint64_t tq_tree_workspace_bytes() { return (uint64_t)min((uint32_t)sm_count(), kAttnMaxCtas) * 2u * 2u * kTreePartFloats * sizeof(float); }

extern "C" int tq_tree_attention(const tq_kv_cache* cache, const void* d_q, int64_t q_stride, uint32_t n_tokens, uint32_t n_seqs,
                                 uint32_t n_q_heads, const int32_t* d_first, const int32_t* d_page_table, uint32_t max_pages,
                                 const int32_t* d_lens, const uint32_t* d_mask, uint32_t mask_words, float scale, void* d_out,
                                 float* d_lse, void* d_ws, uint64_t ws_bytes, void* cuda_stream) {
  if (int rc = tq_check_cache(cache)) return rc;
  if (n_q_heads == 0 || n_q_heads % cache->n_kv_heads || q_stride % 8 || max_pages == 0 || !(scale > 0.f && scale < INFINITY) || (d_mask && mask_words == 0)) return TQ_ERR_INVALID_ARG;
  if (n_q_heads > 65536u || n_tokens > 0x7FFFFFFFu || n_seqs > 0x7FFFFFFEu || (uint64_t)n_tokens * n_q_heads > 0x7FFFFFFFull) return TQ_ERR_UNSUPPORTED_SHAPE;
  const uint64_t group = n_q_heads / cache->n_kv_heads, states = (uint64_t)max_pages * cache->page_size;
  // units of work are counted in 32 bits: those of a group are its tiles of states and kGroupUnits; a sequence without rows has no group
  const uint64_t units = (states < 0x7FFFFFFFull ? states : 0x7FFFFFFFull) / 128u + 1u + kGroupUnits;
  const uint64_t row_tiles = ((uint64_t)n_tokens * group + 127u) / 128u + min(n_seqs, n_tokens);
  if (row_tiles > 0xFFFFFFFFull / cache->n_kv_heads / units) return TQ_ERR_UNSUPPORTED_SHAPE;
  if (n_seqs == 0 || n_tokens == 0) return TQ_OK;
  if (misaligned(d_q, 16) || misaligned(d_first, 4) || misaligned(d_page_table, 4) || misaligned(d_lens, 4) || ((uintptr_t)d_mask & 3u) || misaligned(d_out, 16) ||
      ((uintptr_t)d_lse & 3u) || misaligned(d_ws, 256))
    return TQ_ERR_INVALID_ARG;
  TreeParams p{};
  p.ws = tq_attn_ws_plan(d_ws, ws_bytes);
  if (!p.ws.counters) return TQ_ERR_BUFFER_TOO_SMALL;
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
  p.n_kv_heads = cache->n_kv_heads;
  p.group = n_q_heads / cache->n_kv_heads;
  p.scale_log2 = scale * 1.4426950408889634f;
  p.status = cache->d_status;
  p.whole = states <= kStates * kNeverCutTiles;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  // Boxes that fit pages and tiles alike; the swizzle repeats every 8 rows, so pages of other sizes are copied row by row.
  p.box = 128u;
  while (cache->page_size % p.box) p.box /= 2u;
  p.boxes = kStates / p.box;
  CUtensorMap k_map{}, v_map{};
  if (p.box >= 8u && encode(&k_map, cache->d_k, cache, p.box) && encode(&v_map, cache->d_v, cache, p.box))
    return cache->head_dim == 64 ? launch_rows<64, true>(p, k_map, v_map, st) : launch_rows<128, true>(p, k_map, v_map, st);
  return cache->head_dim == 64 ? launch_rows<64, false>(p, k_map, v_map, st) : launch_rows<128, false>(p, k_map, v_map, st);
}
