// Attention of many queries to an encoder's states (tq_cross_attention but for a few tokens, see there) on the
// 5th-generation tensor cores.
//
//   out = sum_s p_s v_s / sum_s p_s,   p_s = exp(scale q.k_s - m),   m a running maximum
//
// 4 D operations per query, state and head against a few bytes: bound by the tensor cores and, next to
// them, by the exponentials (a 128 x 128 tile of scores costs 1024 cycles of an SM's tensor core at
// head_dim 128 and 1024 cycles of its 16 exponentials a cycle).
//
// Work.  The G query heads that share a key-value head and the tokens are one list of rows (row r = token
// r / G, head r % G); 256 of them are a group's tile.  The units are (sequence, key-value head, tile of
// rows, 128 states), and, as in the one-token kernel, each CTA takes an equal share of consecutive units:
// a group that lies in several shares leaves its parts in the workspace, and a second, small kernel on all SMs joins
// them in order.  (Joined by the CTA that finishes last: 1 x 17 tokens, 64 / 8 heads, 6404 states, 19 parts to a group: 77 us
// instead of 38, now 34; 1 x 600 tokens, two or three parts: 132.8 instead of 135.3.)  So short prompts use all SMs too, and long ones have no last wave.
//
// CTA, one to an SM.  Warp 8 loads: it decides which tiles of states some row of the group
// sees, announces them one by one in a ring of entries that all roles follow, and brings their K and V
// (128-byte swizzled, 2 x 64 columns) with TMA into a ring of stages.  One thread of warp 9 issues the
// products.  Warps 0-3 and 4-7 each own 128 rows, a thread a row: scores from tensor memory, mask,
// maximum, exponentials, p as bf16 back to tensor memory over the scores, where it is the A operand of the
// product with V.  The two halves alternate: the tensor core multiplies for one while the other takes its
// exponentials.  Tensor memory: 2 x 128 columns of scores, 2 x head_dim columns of output.
//
// The output is rescaled only when a row's maximum has grown by more than 2^8 since the last rescaling (the online softmax of
// Milakov and Gimelshein, 2018, with the rescaling delayed up to a threshold, a published refinement of it): p then stays
// below 2^8, which costs no precision in bf16 or in the fp32 sum, and nearly all of the passes over the output in tensor
// memory are saved.
//
// States that no row may see are not multiplied: whole tiles are skipped, the tail past kv_len is zeroed in
// shared memory.  A state that only some rows see enters the others' sums with p = 0; if its value is Inf or
// NaN that product is NaN, so a row whose sum of p is finite but whose output has a NaN is computed again
// from the states it sees (slow, and only with a mask).
//
// Every wait is bounded; one that runs out raises TQ_STATUS_WAIT_EXPIRED, all roles leave their loops and
// tensor memory is released on every path.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <atomic>
#include <cstdint>

#include "tq_internal.h"
#include "tq_ops_common.cuh"

namespace {

using namespace tq_ops;
using namespace tq_sm100;

constexpr uint32_t kRows = 256;        // rows of a group's tile
constexpr uint32_t kHalf = 128;        // rows of a half: one thread each
constexpr uint32_t kStates = 128;      // states of a unit
constexpr int kSoftWarps = 8, kLoadWarp = 8, kMmaWarp = 9;
constexpr int kCrossThreads = 384;  // 12 warps: the last two only make the third warpgroup whole for its register split
// registers a thread: 168 at launch (12 warps of an SM's 65536); 200 for the softmax warps, whose row of scores is 128 of
// them, 96 for the others.  The launch checks the kernel's own count: a split above it would wait for ever.
constexpr int kSoftRegs = 200, kOtherRegs = 96;
constexpr uint32_t kEntries = 4;       // announced tiles that may be under way
constexpr uint32_t kTmemCols = 512;
// With a mask of few large blocks (kCountBlocks at most, kCountBytes of mask in all, kCounts pairs of sequence and tile of
// rows), every CTA first counts the tiles of states that each pair's rows see, and the shares are equal in those; otherwise
// a unit is any tile below kv_len, and the shares of a CTA whose tiles are hidden are finished early.
constexpr uint32_t kCounts = 512, kCountBlocks = 32, kCountBytes = 1u << 18;
// Where whole groups spread evenly enough none is cut: up to a quarter of a share, or kCutTiles tiles of states, over the shares
// that cuts would give.  Parts go through memory to the joining kernel, and the long shares of CTAs that go through the same states
// side by side fall apart.  Measured (us, cut | whole; tiles of a cut share | over it): 152 groups of 3 tiles (4 | 2) 32.3 | 35.5, of
// 5 (6 | 4) 36.0 | 42.4; 64 / 8 heads of 64, 2 x 600 tokens, 1024 states (17 | 7) 57.0 | 68.5; 32 / 8 heads of 64, 1 x 1024 tokens,
// 6404 states (45 | 6) 105 | 112; 32 / 8 heads of 128, 3 x 1000 tokens, 1601 states (34 | 5) 119 | 116; 64 / 8, 1 x 4096 tokens, 6404
// states (353 | 4) 719 | 715.
constexpr uint32_t kCutTiles = 5;
constexpr int kChunks = 2;              // p of a tile is handed to the product with V in so many pieces
constexpr float kRescale = 8.0f;       // log2 of how far p may exceed 1

// What the loader announces, in the first word of an entry: a tile of states for the group's rows, the end of the
// group (or of this CTA's part of it), the end of the work; with a tile, whether it is the first of the part, whether
// the group has rows in the second half, and how many of the tile's states are there (1 .. 128).
enum : uint32_t { kTile = 0, kEnd = 1, kStop = 2, kKind = 3, kFirst = 4, kTwoHalves = 8, kValidShift = 8 };

// The first four words are all that a tile needs; the rest is read with the first tile and the end.
struct Entry {
  uint32_t ctl, tile, len, qt;      // tile of states; states of the sequence; tile of rows
  uint32_t b, kvh, t0, t1;          // sequence, key-value head; kEnd: first and one past the last of the part's tiles of states
  uint32_t c0, parts, unused0, unused1;  // kEnd: first CTA with a part of the group, number of parts
};

struct CrossParams {
  const __nv_bfloat16* k;
  const __nv_bfloat16* v;
  int64_t batch_stride, state_stride, head_stride;
  const __nv_bfloat16* q;
  int64_t q_batch_stride, q_token_stride;
  __nv_bfloat16* out;
  float* lse;
  const int32_t* kv_len;
  const uint8_t* mask;
  uint32_t n_states, block_len, n_blocks;
  uint32_t n_seqs, n_tokens, n_q_heads, n_kv_heads, group;
  uint32_t rows, row_tiles;  // n_tokens * group, and its tiles of 256
  float scale_log2;
  uint32_t by_group;  // the joining kernel finds the cut groups by their number (few groups), not by the CTA they begin in
  uint32_t counted;  // the units are the tiles of states that some row of the group sees (see kCounts)
  uint32_t test_withhold;  // test hook (tq_test_withhold_cross_entry): the loader gives up where it would announce
  tq_attn_ws ws;
};

template <int D>
struct CrossSmem {
  static constexpr uint32_t kSlabs = D / 64;                       // 64 columns = 128 bytes of a swizzled row
  static constexpr uint32_t kQHalf = kSlabs * kHalf * 128;         // queries of a half
  static constexpr uint32_t kStageBytes = kSlabs * kStates * 128;  // K or V of a tile
  static constexpr uint32_t kStages = D == 128 ? 5 : 8;
  static constexpr uint32_t kOffKv = 2 * kQHalf;
  static constexpr uint32_t kOffMisc = kOffKv + kStages * kStageBytes;
  // misc: [0] dead flag, [4] tensor-memory base, barriers from 16 on, entries behind them
  static constexpr uint32_t kBarKvFull = 16, kBarKvEmpty = kBarKvFull + 8 * kStages, kBarQFull = kBarKvEmpty + 8 * kStages;
  static constexpr uint32_t kBarSFull = kBarQFull + 16, kBarPFull = kBarSFull + 16, kBarODone = kBarPFull + 16 * kChunks;
  static constexpr uint32_t kBarEFull = kBarODone + 16, kBarEEmpty = kBarEFull + 8 * kEntries;
  static constexpr uint32_t kOffEntries = (kBarEEmpty + 8 * kEntries + 15) / 16 * 16;
  static_assert(sizeof(Entry) % 16 == 0, "entries are read in 16-byte words");
  static constexpr uint32_t kOffCounts = kOffEntries + kEntries * sizeof(Entry);
  static constexpr uint32_t kTotal = kOffMisc + kOffCounts + kCounts * sizeof(uint16_t);
  static_assert(kTotal + 1024 <= 232448, "shared memory of one CTA");
};
// a part of a split group: [D / 4][256] float4 of output, then the rows' maxima and sums
constexpr uint64_t kCrossPartFloats = kRows * (128 + 2);

__device__ __forceinline__ void tma_load_4d(uint32_t dst, const CUtensorMap* map, int x, int y, int z, int w, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(dst),
               "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(bar)
               : "memory");
}
// A operand in tensor memory, B described in shared memory.
__device__ __forceinline__ void umma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d_tmem),
      "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// V as it lies, states x columns: the operand's N index (column) is contiguous.  128-byte swizzle: 64 columns x 8
// states are 1024 bytes, the next 8 states follow, the next 64 columns are a slab of 128 states away.
__device__ __forceinline__ uint64_t umma_desc_n_major(uint32_t smem_addr) {
  uint64_t d = umma_desc(smem_addr);
  d &= ~((uint64_t)0x3FFF << 16);
  return d | ((uint64_t)((kStates * 128u) >> 4) << 16);
}
constexpr uint32_t kIdescNMajorB = 1u << 16;

#define TMEM_LD32(r, addr)                                                                                                          \
  asm volatile(                                                                                                                     \
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,"  \
      "%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"                                                                                \
      : "=r"((r)[0]), "=r"((r)[1]), "=r"((r)[2]), "=r"((r)[3]), "=r"((r)[4]), "=r"((r)[5]), "=r"((r)[6]), "=r"((r)[7]),             \
        "=r"((r)[8]), "=r"((r)[9]), "=r"((r)[10]), "=r"((r)[11]), "=r"((r)[12]), "=r"((r)[13]), "=r"((r)[14]), "=r"((r)[15]),       \
        "=r"((r)[16]), "=r"((r)[17]), "=r"((r)[18]), "=r"((r)[19]), "=r"((r)[20]), "=r"((r)[21]), "=r"((r)[22]), "=r"((r)[23]),     \
        "=r"((r)[24]), "=r"((r)[25]), "=r"((r)[26]), "=r"((r)[27]), "=r"((r)[28]), "=r"((r)[29]), "=r"((r)[30]), "=r"((r)[31])      \
      : "r"(addr))
#define TMEM_ST32(addr, r)                                                                                                          \
  asm volatile(                                                                                                                     \
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,"   \
      "%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),                                                                  \
      "r"((r)[0]), "r"((r)[1]), "r"((r)[2]), "r"((r)[3]), "r"((r)[4]), "r"((r)[5]), "r"((r)[6]), "r"((r)[7]), "r"((r)[8]),          \
      "r"((r)[9]), "r"((r)[10]), "r"((r)[11]), "r"((r)[12]), "r"((r)[13]), "r"((r)[14]), "r"((r)[15]), "r"((r)[16]), "r"((r)[17]),  \
      "r"((r)[18]), "r"((r)[19]), "r"((r)[20]), "r"((r)[21]), "r"((r)[22]), "r"((r)[23]), "r"((r)[24]), "r"((r)[25]),               \
      "r"((r)[26]), "r"((r)[27]), "r"((r)[28]), "r"((r)[29]), "r"((r)[30]), "r"((r)[31])                                            \
      : "memory")
#define TMEM_LD16(r, addr)                                                                                                          \
  asm volatile(                                                                                                                     \
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"                      \
      : "=r"((r)[0]), "=r"((r)[1]), "=r"((r)[2]), "=r"((r)[3]), "=r"((r)[4]), "=r"((r)[5]), "=r"((r)[6]), "=r"((r)[7]),             \
        "=r"((r)[8]), "=r"((r)[9]), "=r"((r)[10]), "=r"((r)[11]), "=r"((r)[12]), "=r"((r)[13]), "=r"((r)[14]), "=r"((r)[15])        \
      : "r"(addr))
#define TMEM_ST16(addr, r)                                                                                                          \
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr), \
               "r"((r)[0]), "r"((r)[1]), "r"((r)[2]), "r"((r)[3]), "r"((r)[4]), "r"((r)[5]), "r"((r)[6]), "r"((r)[7]), "r"((r)[8]), \
               "r"((r)[9]), "r"((r)[10]), "r"((r)[11]), "r"((r)[12]), "r"((r)[13]), "r"((r)[14]), "r"((r)[15])                      \
               : "memory")
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tmem_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void lds128(uint32_t addr, uint32_t& a, uint32_t& b, uint32_t& c, uint32_t& d) {
  asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(a), "=r"(b), "=r"(c), "=r"(d) : "r"(addr) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}
// One lane of a converged warp, chosen so that the compiler knows it is one.
__device__ __forceinline__ bool elect_one() {
  uint32_t yes;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(yes));
  return yes != 0;
}
// Two fp32 operations in one instruction.
__device__ __forceinline__ uint64_t pair(float lo, float hi) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(lo), "f"(hi));
  return r;
}
__device__ __forceinline__ void unpair(uint64_t v, float& lo, float& hi) { asm("mov.b64 {%0, %1}, %2;" : "=f"(lo), "=f"(hi) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}

__device__ __forceinline__ uint32_t states_of(const CrossParams& p, uint32_t b) {
  if (p.kv_len == nullptr) return p.n_states;
  const int32_t n = __ldg(p.kv_len + b);
  return n <= 0 ? 0u : min((uint32_t)n, p.n_states);
}
__device__ __forceinline__ uint32_t units_of(uint32_t len) { return len == 0u ? 1u : (len + kStates - 1u) / kStates; }
// The low n bits, n clamped to 0..32.
__device__ __forceinline__ uint32_t low_bits(int n) { return n <= 0 ? 0u : (n >= 32 ? 0xFFFFFFFFu : (1u << n) - 1u); }

template <int D>
__global__ void __launch_bounds__(kCrossThreads, 1)
    cross_attention_kernel(const CrossParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map) {
  using L = CrossSmem<D>;
  extern __shared__ __align__(16) uint8_t smem_raw[];
  uint8_t* const smem = smem_raw + ((1024u - (smem_u32(smem_raw) & 1023u)) & 1023u);  // swizzled tiles start on 1024 bytes
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t smem0 = smem_u32(smem), misc = smem0 + L::kOffMisc;
  volatile uint32_t* const dead = reinterpret_cast<uint32_t*>(smem + L::kOffMisc);
  uint32_t* const tmem_slot = reinterpret_cast<uint32_t*>(smem + L::kOffMisc + 4);
  const uint32_t entries = misc + L::kOffEntries;
  // the same in all lanes, and known to be: what depends on it alone stays on the uniform data path
  const uint32_t warp = __shfl_sync(kFull, threadIdx.x >> 5, 0), lane = threadIdx.x & 31u;
  auto bar = [&](uint32_t off, uint32_t i) { return misc + off + 8u * i; };

  if (threadIdx.x == 0) {
    *dead = 0u;
    for (uint32_t i = 0; i < L::kStages; ++i) {
      mbar_init(bar(L::kBarKvFull, i), 1);
      mbar_init(bar(L::kBarKvEmpty, i), 1);
    }
    for (uint32_t i = 0; i < 2; ++i) {
      mbar_init(bar(L::kBarQFull, i), 4);
      mbar_init(bar(L::kBarSFull, i), 1);
      for (uint32_t x = 0; x < kChunks; ++x) mbar_init(bar(L::kBarPFull, i * kChunks + x), 4);
      mbar_init(bar(L::kBarODone, i), 1);
    }
    for (uint32_t i = 0; i < kEntries; ++i) {
      mbar_init(bar(L::kBarEFull, i), 1);
      mbar_init(bar(L::kBarEEmpty, i), kSoftWarps + 1);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(kTmemCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tmem_fence_before();
  __syncthreads();
  tmem_fence_after();
  const uint32_t tmem = *tmem_slot;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  uint16_t* const counts = reinterpret_cast<uint16_t*>(smem + L::kOffMisc + L::kOffCounts);
  if (p.counted) {
    uint32_t* const seen = reinterpret_cast<uint32_t*>(smem + L::kOffKv);  // the blocks that a pair's rows see, a bit each
    const uint32_t pairs = p.n_seqs * p.row_tiles, bytes = p.n_seqs * p.n_tokens * p.n_blocks;
    for (uint32_t i = threadIdx.x; i < pairs; i += kCrossThreads) seen[i] = 0u;
    __syncthreads();
    const bool words = ((uintptr_t)p.mask & 3u) == 0u;
#pragma unroll 4
    for (uint32_t i = threadIdx.x * 4u; i < bytes; i += kCrossThreads * 4u) {
      uint32_t v = 0;
      if (words && i + 4u <= bytes) {
        v = __ldg(reinterpret_cast<const uint32_t*>(p.mask + i));
      } else {
        for (uint32_t k = i; k < min(i + 4u, bytes); ++k) v |= (uint32_t)__ldg(p.mask + k) << (8u * (k - i));
      }
      for (uint32_t k = 0; v != 0u; ++k, v >>= 8) {
        if ((v & 255u) == 0u) continue;
        const uint32_t bt = (i + k) / p.n_blocks, bit = 1u << ((i + k) - bt * p.n_blocks);
        const uint32_t b = bt / p.n_tokens, r = (bt - b * p.n_tokens) * p.group;
        for (uint32_t q = r / kRows; q <= (r + p.group - 1u) / kRows; ++q) {
          uint32_t* at = seen + b * p.row_tiles + q;
          if ((*(volatile uint32_t*)at & bit) == 0u) atomicOr(at, bit);
        }
      }
    }
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < pairs; i += kCrossThreads) {
      const uint32_t len = states_of(p, i / p.row_tiles);
      uint32_t n = 0, next = 0;  // tiles; the first one that is not counted yet
      for (uint32_t bits = seen[i]; bits != 0u; bits &= bits - 1u) {
        const uint32_t blk = __ffs(bits) - 1u, from = blk * p.block_len;
        if (from >= len) break;
        const uint32_t t0 = max(from / kStates, next), t1 = (min(from + p.block_len, len) - 1u) / kStates + 1u;
        if (t1 > t0) n += t1 - t0;
        next = max(next, t1);
      }
      counts[i] = (uint16_t)max(n, 1u);
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");  // the stages are TMA's from here on
    __syncthreads();
  }

  bool ok = true;
  auto wait = [&](uint32_t b, uint32_t parity) {
    ok = ok && mbar_wait(b, parity, dead);
    ok = __all_sync(kFull, ok);
  };
  uint32_t e_slot = 0, e_round = 0;  // slot of the next entry this warp takes (or announces), and how often the slots have wrapped
  auto next_slot = [&]() {
    if (++e_slot == kEntries) {
      e_slot = 0;
      ++e_round;
    }
  };
  // the next entry: all of it, or its first words unless it opens or closes a group
  auto take = [&](Entry& e) {
    wait(bar(L::kBarEFull, e_slot), e_round & 1u);
    if (!ok) return;
    const uint32_t at = entries + e_slot * (uint32_t)sizeof(Entry);
    lds128(at, e.ctl, e.tile, e.len, e.qt);
    if ((e.ctl & (kKind | kFirst)) != kTile) {
      lds128(at + 16u, e.b, e.kvh, e.t0, e.t1);
      lds128(at + 32u, e.c0, e.parts, e.unused0, e.unused1);
    }
    __syncwarp();
    if (lane == 0) mbar_arrive(bar(L::kBarEEmpty, e_slot));
    next_slot();
  };

  if (warp >= kLoadWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
  if (warp == kLoadWarp) {
    // ---- which tiles, and their K and V ---------------------------------------------------------------
    // units of a group; of the row tiles of a sequence for one key-value head
    auto units = [&](uint32_t b, uint32_t qt) { return p.counted ? (uint32_t)counts[b * p.row_tiles + qt] : units_of(states_of(p, b)); };
    auto head_units = [&](uint32_t b) {
      if (!p.counted) return units_of(states_of(p, b)) * p.row_tiles;
      uint32_t n = 0;
      for (uint32_t q = 0; q < p.row_tiles; ++q) n += counts[b * p.row_tiles + q];
      return n;
    };
    uint32_t total = 0, most = 0, least = 0xFFFFFFFFu;  // units of all groups, of one group
    for (uint32_t b = lane; b < p.n_seqs; b += 32u) {
      total += head_units(b);
      for (uint32_t q = 0; q < (p.counted ? p.row_tiles : 1u); ++q) {
        const uint32_t n = units(b, q);
        most = max(most, n);
        least = min(least, n);
      }
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) {
      total += __shfl_xor_sync(kFull, total, d);
      most = max(most, __shfl_xor_sync(kFull, most, d));
      least = min(least, __shfl_xor_sync(kFull, least, d));
    }
    total *= p.n_kv_heads;  // below 2^32: the launch has seen to it
    // CTA i's share: units i * mean + min(i, over) and on
    const uint32_t ctas = min(gridDim.x, total), mean = total / ctas, over = total - mean * ctas;
    auto cta_of = [&](uint32_t u) { return u < over * (mean + 1u) ? u / (mean + 1u) : over + (u - over * (mean + 1u)) / mean; };
    // the longest share without cuts: whole groups of one size, or up to one group over the mean
    const uint32_t n_groups = p.n_seqs * p.n_kv_heads * p.row_tiles;
    const uint32_t longest = most == least ? ((n_groups - 1u) / ctas + 1u) * most : mean + most;
    const bool cut = longest > mean + (over != 0u ? 1u : 0u) + min(kCutTiles, mean / 4u);
    uint32_t u0 = 0, u1 = 0;  // this CTA's share; without cuts, the groups that start in it
    if (blockIdx.x < ctas) {
      u0 = mean * blockIdx.x + min(blockIdx.x, over);
      u1 = u0 + mean + (blockIdx.x < over ? 1u : 0u);
    }
    uint32_t first = 0;  // first unit of the group (b, kvh, qt)
    uint32_t b = 0, kvh = 0, qt = 0, n = 1, st = 0, st_round = 0;
    auto next_group = [&]() {
      first += n;
      if (++qt == p.row_tiles) {
        qt = 0;
        if (++kvh == p.n_kv_heads) {
          kvh = 0;
          ++b;
        }
      }
      if (b < p.n_seqs) n = units(b, qt);
    };
    if (u0 < u1) {
      uint32_t h = head_units(0);
      while (b + 1u < p.n_seqs && u0 - first >= h * p.n_kv_heads) {
        first += h * p.n_kv_heads;
        h = head_units(++b);
      }
      kvh = (u0 - first) / h;
      first += h * kvh;
      n = units(b, 0);
      if (!p.counted) {
        qt = (u0 - first) / n;
        first += n * qt;
      }
      while (b < p.n_seqs && (u0 >= first + n || (!cut && first < u0))) next_group();
    }
    auto announce = [&](const Entry& e) {
      if (p.test_withhold) ok = false;
      if (e_round) wait(bar(L::kBarEEmpty, e_slot), (e_round - 1u) & 1u);
      if (!ok) return;
      if (lane == 0) {
        const uint32_t at = entries + e_slot * (uint32_t)sizeof(Entry);
        sts128(at, e.ctl, e.tile, e.len, e.qt);
        sts128(at + 16u, e.b, e.kvh, e.t0, e.t1);
        sts128(at + 32u, e.c0, e.parts, 0u, 0u);
        mbar_arrive(bar(L::kBarEFull, e_slot));
      }
      __syncwarp();
      next_slot();
    };
    auto load = [&](const CUtensorMap* map, const Entry& e) {
      if (st_round) wait(bar(L::kBarKvEmpty, st), (st_round - 1u) & 1u);
      if (!ok) return;
      if (lane == 0) {
        const uint32_t full = bar(L::kBarKvFull, st), dst = smem0 + L::kOffKv + st * L::kStageBytes;
        mbar_expect_tx(full, L::kStageBytes);
#pragma unroll
        for (uint32_t s = 0; s < L::kSlabs; ++s)
          tma_load_4d(dst + s * kStates * 128u, map, (int)(s * 64u), (int)(e.tile * kStates), p.head_stride ? (int)e.kvh : 0, p.batch_stride ? (int)e.b : 0, full);
      }
      __syncwarp();
      if (++st == L::kStages) {
        st = 0;
        ++st_round;
      }
    };
    uint4 open = make_uint4(0u, 0u, 0u, 0u);  // the last group that begins in this share, the only one that can go on in the next
    for (; first < u1 && b < p.n_seqs && ok; next_group()) {
      const uint32_t len = states_of(p, b);
      // this CTA's units of the group
      const uint32_t x0 = cut && u0 > first ? u0 - first : 0u, x1 = cut && u1 - first < n ? u1 - first : n;
      Entry e{};
      e.b = b;
      e.len = len;
      e.kvh = kvh;
      e.qt = qt;
      const uint32_t two = p.rows - e.qt * kRows > kHalf ? kTwoHalves : 0u;
      uint32_t opens = kFirst;
      // tokens of the group's rows, whose mask bytes decide which tiles are needed
      const uint32_t tok0 = e.qt * kRows / p.group, tok1 = (min(p.rows, (e.qt + 1u) * kRows) - 1u) / p.group + 1u;
      uint32_t known = 0xFFFFFFFFu;  // block whose visibility is known (blocks of at least a tile), and it
      bool known_seen = false;
      auto seen = [&](uint32_t tile) {
        const uint32_t s0 = tile * kStates, s1 = min(s0 + kStates, len);
        if (s0 >= s1) return false;
        if (p.mask == nullptr) return true;
        const uint32_t b0 = s0 / p.block_len, b1 = (s1 - 1u) / p.block_len;
        const uint8_t* m = p.mask + (size_t)b * p.n_tokens * p.n_blocks;
        if (p.block_len >= kStates) {  // at most two blocks: lanes over the tokens
          for (uint32_t blk = b0; blk <= b1; ++blk) {
            if (blk != known) {
              bool any = false;
              for (uint32_t t = tok0 + lane; t < tok1; t += 32u) any = any || __ldg(m + (size_t)t * p.n_blocks + blk) != 0;
              known_seen = __any_sync(kFull, any);
              known = blk;
            }
            if (known_seen) return true;
          }
          return false;
        }
        for (uint32_t t = tok0; t < tok1; ++t) {  // many blocks: lanes over the blocks
          bool any = false;
          for (uint32_t blk = b0 + lane; blk <= b1; blk += 32u) any = any || __ldg(m + (size_t)t * p.n_blocks + blk) != 0;
          if (__any_sync(kFull, any)) return true;
        }
        return false;
      };
      const uint32_t tiles = (len + kStates - 1u) / kStates;
      uint32_t x = p.counted ? 0u : x0;  // the unit that the next tile is
      for (uint32_t t = x; t < tiles && x < x1 && ok; ++t) {
        const bool yes = seen(t);
        if (!yes) {
          if (!p.counted) ++x;
          continue;
        }
        if (x++ < x0) continue;
        e.ctl = kTile | opens | two | (min(kStates, len - t * kStates) << kValidShift);
        e.tile = t;
        announce(e);
        if (ok) load(&k_map, e);
        if (ok) load(&v_map, e);
        if (opens) e.t0 = t;
        e.t1 = t + 1u;
        opens = 0u;
      }
      if (!ok) break;
      e.ctl = kEnd;
      e.c0 = blockIdx.x;
      e.parts = 1u;
      if (cut && (first < u0 || u1 - first < n)) {
        e.c0 = cta_of(first);
        e.parts = cta_of(first + n - 1u) - e.c0 + 1u;
      }
      announce(e);
      if (first >= u0) {  // the CTA in which a group begins tells the joining kernel of it
        const uint32_t id = (b * p.n_kv_heads + kvh) * p.row_tiles + qt;
        const uint4 r = make_uint4(e.parts > 1u ? e.parts : 0u, blockIdx.x, id, 0u);
        if (!p.by_group)
          open = r;
        else if (lane == 0)
          p.ws.open[id] = r;
      }
    }
    if (lane == 0 && !p.by_group) p.ws.open[blockIdx.x] = open;
    if (ok) {
      Entry e{};
      e.ctl = kStop;
      announce(e);
    }
  } else if (warp == kMmaWarp) {
    // ---- products -------------------------------------------------------------------------------------
    // This warp's path between two waits is on the critical path of both halves, and it shares its scheduler with the long
    // softmax code: it is kept short, with operand descriptors that one addition moves on.
    uint32_t st = 0, st_round = 0;  // stage of the next K
    bool have = false;
    uint32_t accumulate = 0, v_st = 0, v_round = 0, v_valid = kStates, halves = 2;
    uint32_t p_phase = 0, q_phase = 0;  // bit w: half w
    const uint32_t idesc_qk = umma_idesc(128, 128), idesc_pv = umma_idesc(128, D) | kIdescNMajorB;
    const uint64_t q_desc = umma_desc(smem0), kv_desc = umma_desc(smem0 + L::kOffKv), v_desc = umma_desc_n_major(smem0 + L::kOffKv);
    auto qk = [&](uint32_t w, uint32_t k_st) {
      if (elect_one()) {
        const uint64_t a = q_desc + w * (L::kQHalf >> 4), b = kv_desc + k_st * (L::kStageBytes >> 4);
#pragma unroll
        for (uint32_t kk = 0; kk < D / 16; ++kk) {
          constexpr uint32_t kSlab = (kHalf * 128u) >> 4;
          const uint32_t off = (kk / 4u) * kSlab + (kk % 4u) * 2u;  // in 16 bytes
          umma_bf16(tmem + w * kStates, a + off, b + off, idesc_qk, kk != 0u);
        }
        umma_commit(bar(L::kBarSFull, w));
      }
      __syncwarp();
    };
    auto pv = [&](uint32_t w) {
      const uint64_t b = v_desc + v_st * (L::kStageBytes >> 4);
      const uint32_t d = tmem + 2 * kStates + w * D, a = tmem + w * kStates;
#pragma unroll 1
      for (uint32_t x = 0; x < kChunks; ++x) {
        wait(bar(L::kBarPFull, w * kChunks + x), (p_phase >> w) & 1u);
        if (!ok) return;
        tmem_fence_after();
        if (elect_one()) {
          constexpr uint32_t kSteps = kStates / 16 / kChunks;
#pragma unroll
          for (uint32_t kk = 0; kk < kSteps; ++kk)
            umma_bf16_ts(d, a + (x * kSteps + kk) * 8u, b + (x * kSteps + kk) * (2048u >> 4), idesc_pv, accumulate | x | kk);
        }
        __syncwarp();
      }
      p_phase ^= 1u << w;
      if (w + 1u == halves && elect_one()) umma_commit(bar(L::kBarKvEmpty, v_st));
      __syncwarp();
    };
    auto wait_v = [&]() {
      wait(bar(L::kBarKvFull, v_st), v_round & 1u);
      if (!ok || v_valid >= kStates) return;
      // past the sequence's last state memory may hold anything, and 0 x NaN is NaN
      constexpr uint32_t kChunks = D / 8;
      uint8_t* tile = smem + L::kOffKv + v_st * L::kStageBytes;
      for (uint32_t i = lane; i < (kStates - v_valid) * kChunks; i += 32u) {
        const uint32_t r = v_valid + i / kChunks, c = i % kChunks;
        *reinterpret_cast<uint4*>(tile + (c / 8u) * (kStates * 128u) + r * 128u + (c % 8u) * 16u) = make_uint4(0, 0, 0, 0);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
    };
    auto bump = [&]() {
      if (++st == L::kStages) {
        st = 0;
        ++st_round;
      }
    };
    Entry e;
    while (ok) {
      take(e);
      const uint32_t kind = e.ctl & kKind;
      if (!ok || kind == kStop) break;
      if (have) wait_v();
      if (!ok) break;
      if (kind == kTile) {
        if (e.ctl & kFirst) halves = e.ctl & kTwoHalves ? 2u : 1u;
        const uint32_t k_st = st;
        wait(bar(L::kBarKvFull, k_st), st_round & 1u);
        bump();
        for (uint32_t w = 0; w < halves && ok; ++w) {
          if (have) pv(w);
          if (e.ctl & kFirst) {
            wait(bar(L::kBarQFull, w), (q_phase >> w) & 1u);
            q_phase ^= 1u << w;
          }
          if (ok) qk(w, k_st);
        }
        if (!ok) break;
        if (elect_one()) umma_commit(bar(L::kBarKvEmpty, k_st));
        __syncwarp();
        accumulate = have ? 1u : 0u;
        have = true;
        v_st = st;
        v_round = st_round;
        v_valid = e.ctl >> kValidShift;
        bump();
      } else if (have) {
        for (uint32_t w = 0; w < halves && ok; ++w) {
          pv(w);
          if (ok && elect_one()) umma_commit(bar(L::kBarODone, w));
          __syncwarp();
        }
        have = false;
      }
    }
  }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftRegs));
    // ---- softmax: a thread a row ------------------------------------------------------------------------
    const uint32_t w = warp >> 2, row_in = threadIdx.x & 127u;
    const uint32_t lane_field = (warp & 3u) << 21;  // 32 lanes of tensor memory to a warp
    const uint32_t s_addr = tmem + lane_field + w * kStates, o_addr = tmem + lane_field + 2 * kStates + w * D;
    const float c = p.scale_log2;
    uint32_t s_phase = 0, o_phase = 0;
    float m = -INFINITY, l = 0.f;
    bool any_tile = false, q_ready = false;
    uint32_t row = 0, tok = 0;
    bool live = false, half_live = false;

    auto place = [&](const Entry& e) {  // this thread's row in the entry's group
      row = e.qt * kRows + w * kHalf + row_in;
      live = row < p.rows;
      half_live = e.qt * kRows + w * kHalf < p.rows;
      tok = live ? row / p.group : 0u;
    };
    auto q_row = [&](const Entry& e) {
      return p.q + (int64_t)e.b * p.q_batch_stride + (int64_t)tok * p.q_token_stride + (size_t)(e.kvh * p.group + row % p.group) * D;
    };
    auto load_q = [&](const Entry& e) {
      if (!half_live) return;
      const uint4* src = reinterpret_cast<const uint4*>(q_row(e));
      uint8_t* dst = smem + w * L::kQHalf + row_in * 128u;
      uint4 v[D / 8];
#pragma unroll
      for (uint32_t i = 0; i < D / 8; ++i) v[i] = live ? __ldg(src + i) : make_uint4(0, 0, 0, 0);
#pragma unroll
      for (uint32_t i = 0; i < D / 8; ++i) *reinterpret_cast<uint4*>(dst + (i / 8u) * (kHalf * 128u) + (((i % 8u) ^ (row_in & 7u)) << 4)) = v[i];
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(bar(L::kBarQFull, w));
    };
    // bit i: this row sees state s0 + i
    auto visible = [&](const Entry& e, uint32_t (&bits)[4]) {
      const uint32_t s0 = e.tile * kStates, s1 = min(s0 + kStates, e.len);
      if (p.mask == nullptr) {
#pragma unroll
        for (int i = 0; i < 4; ++i) bits[i] = low_bits((int)(s1 - s0) - 32 * i);
        return;
      }
      bits[0] = bits[1] = bits[2] = bits[3] = 0u;
      const uint8_t* mr = p.mask + ((size_t)e.b * p.n_tokens + tok) * p.n_blocks;
      for (uint32_t blk = s0 / p.block_len; blk <= (s1 - 1u) / p.block_len; ++blk) {
        const uint64_t from = (uint64_t)blk * p.block_len;
        const int lo = from > s0 ? (int)(from - s0) : 0, hi = (int)min((uint64_t)s1 - s0, from + p.block_len - s0);
        if (__ldg(mr + blk) == 0) continue;
#pragma unroll
        for (int i = 0; i < 4; ++i) bits[i] |= low_bits(hi - 32 * i) & ~low_bits(lo - 32 * i);
      }
    };

    Entry e;
    bool pending = false;  // e holds an entry that was taken early
    while (ok) {
      if (!pending) take(e);
      pending = false;
      if (!ok || (e.ctl & kKind) == kStop) break;
      if ((e.ctl & kKind) == kTile) {
        if (e.ctl & kFirst) {
          place(e);
          if (!q_ready) load_q(e);
          q_ready = false;
          m = -INFINITY;
          l = 0.f;
          any_tile = true;
        }
        if (!half_live) continue;
        uint32_t bits[4];
        bool partial = (e.ctl >> kValidShift) != kStates;  // some row does not see some state
        if (p.mask != nullptr || partial) {
          visible(e, bits);
          partial = __any_sync(kFull, (bits[0] & bits[1] & bits[2] & bits[3]) != 0xFFFFFFFFu);
        }
        wait(bar(L::kBarSFull, w), s_phase);
        s_phase ^= 1u;
        if (!ok) break;
        tmem_fence_after();
        uint32_t s[128];
#pragma unroll
        for (int i = 0; i < 4; ++i) TMEM_LD32(s + 32 * i, s_addr + 32u * i);
        tmem_wait_ld();
        if (partial) {
#pragma unroll
          for (int i = 0; i < 128; ++i) s[i] = (bits[i / 32] >> (i % 32)) & 1u ? s[i] : 0xFF800000u;
        }
        float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int i = 0; i < 128; i += 8) {
#pragma unroll
          for (int k = 0; k < 4; ++k) mx[k] = max3(mx[k], __uint_as_float(s[i + 2 * k]), __uint_as_float(s[i + 2 * k + 1]));
        }
        const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]) * c;
        const bool grow = top > m + kRescale;
        if (__any_sync(kFull, grow)) {
          const float mn = fmaxf(m, top);
          const float f = mn == -INFINITY ? 1.f : exp2_fast(m - mn);
          m = mn;
          l *= f;
          if (!(e.ctl & kFirst)) {  // these scores were committed after the products with V before them: the output is complete
#pragma unroll
            for (int i = 0; i < D / 16; ++i) {
              uint32_t o[16];
              TMEM_LD16(o, o_addr + 16u * i);
              tmem_wait_ld();
#pragma unroll
              for (int k = 0; k < 16; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * f);
              TMEM_ST16(o_addr + 16u * i, o);
            }
          }
        }
        const float ref = m == -INFINITY ? 0.f : m;
        const uint64_t c2 = pair(c, c), ref2 = pair(-ref, -ref);
        uint64_t sum[2] = {0, 0};
        auto hand_over = [&](int x) {  // piece x of p is in tensor memory
          tmem_wait_st();
          tmem_fence_before();
          __syncwarp();
          if (lane == 0) mbar_arrive(bar(L::kBarPFull, w * kChunks + x));
        };
        constexpr int kPairs = 64 / kChunks, kLate = 3;
        static_assert(kPairs == 32, "one store of 32 columns a piece");
#pragma unroll
        for (int x = 0; x < kChunks; ++x) {
          uint32_t pk[kPairs];
#pragma unroll
          for (int i = 0; i < kPairs; ++i) {
            if (x != 0 && i == kLate) hand_over(x - 1);  // its stores have had time to land
            const int at = 2 * (x * kPairs + i);
            float a, b;
            unpair(fma2(pair(__uint_as_float(s[at]), __uint_as_float(s[at + 1])), c2, ref2), a, b);
            a = exp2_fast(a);
            b = exp2_fast(b);
            sum[i & 1] = add2(sum[i & 1], pair(a, b));
            pk[i] = pack_bf16(a, b);
          }
          TMEM_ST32(s_addr + kPairs * x, pk);
        }
        hand_over(kChunks - 1);
        float l0, l1;
        unpair(add2(sum[0], sum[1]), l0, l1);
        l += l0 + l1;
        continue;
      }
      // ---- end of the group, or of this CTA's part: the next group's queries first, they are waited for ------
      const Entry g = e;
      const bool had = any_tile;
      if (!had) {
        place(g);
        m = -INFINITY;
        l = 0.f;
      }
      any_tile = false;
      const uint32_t g_row = row, g_tok = tok;
      const bool g_live = live, g_half = half_live;
      take(e);
      pending = true;
      if (!ok) break;
      if ((e.ctl & kKind) == kTile) {
        place(e);
        load_q(e);
        q_ready = true;
        row = g_row, tok = g_tok, live = g_live, half_live = g_half;
      }
      const bool real = had && g_half;  // there is an output in tensor memory
      if (real) {
        wait(bar(L::kBarODone, w), o_phase);
        o_phase ^= 1u;
        if (!ok) break;
        tmem_fence_after();
      }
      const size_t at = ((size_t)g.b * p.n_tokens + tok) * p.n_q_heads + g.kvh * p.group + row % p.group;
      auto part = [&](uint32_t i) { return p.ws.parts + (size_t)(2u * (g.c0 + i) + (i == 0u ? 1u : 0u)) * kCrossPartFloats; };
      const uint32_t slot = threadIdx.x;  // 0 .. 255
      const bool whole = g.parts == 1u;
      float* const mine = part(blockIdx.x - g.c0);
      auto write = [&](int i, const uint32_t (&o)[32]) {  // columns 32 i .. 32 i + 31 of a finished row
        if (!live) return;
        const float inv = 1.0f / l;
#pragma unroll
        for (int k = 0; k < 32; k += 8) {
          float f[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) f[x] = l == 0.f ? 0.f : __uint_as_float(o[k + x]) * inv;
          store8<TQ_TYPE_BF16>(p.out, at * D + 32 * i + k, f);
        }
        if (i == 0 && p.lse) p.lse[at] = l == 0.f ? -INFINITY : (m + log2f(l)) * 0.6931471805599453f;
      };
      bool nan = false;
#pragma unroll 1
      for (int i = 0; i < D / 32; ++i) {
        uint32_t o[32];
        if (real) {
          TMEM_LD32(o, o_addr + 32u * i);
          tmem_wait_ld();
        } else {
#pragma unroll
          for (int k = 0; k < 32; ++k) o[k] = 0u;
        }
#pragma unroll
        for (int k = 0; k < 32; ++k) nan = nan || __uint_as_float(o[k]) != __uint_as_float(o[k]);
        if (whole) {
          write(i, o);
        } else if (live) {
#pragma unroll
          for (int k = 0; k < 8; ++k) reinterpret_cast<uint4*>(mine)[(8 * i + k) * kRows + slot] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
        }
      }
      tmem_fence_before();
      if (p.mask != nullptr) {  // rows that a state they do not see has spoiled: again, a warp a row, D / 32 columns a lane
        uint32_t again = __ballot_sync(kFull, live && nan && l < INFINITY);
#pragma unroll 1
        while (again) {
          const int src = __ffs(again) - 1;
          again &= again - 1u;
          constexpr int kPer = D / 32;
          const uint32_t rr = __shfl_sync(kFull, row, src), rt = __shfl_sync(kFull, tok, src), rs = __shfl_sync(kFull, slot, src);
          const float rm = __shfl_sync(kFull, m, src), rl = __shfl_sync(kFull, l, src);
          const __nv_bfloat16* q = p.q + (int64_t)g.b * p.q_batch_stride + (int64_t)rt * p.q_token_stride + (size_t)(g.kvh * p.group + rr % p.group) * D + lane * kPer;
          const uint8_t* mr = p.mask + ((size_t)g.b * p.n_tokens + rt) * p.n_blocks;
          float acc[kPer], qv[kPer];
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            acc[i] = 0.f;
            qv[i] = __bfloat162float(q[i]);
          }
          const int64_t base = (int64_t)g.b * p.batch_stride + (int64_t)g.kvh * p.head_stride + lane * kPer;
          const uint32_t s1 = min(g.t1 * kStates, g.len);
#pragma unroll 1
          for (uint32_t s = g.t0 * kStates; s < s1; ++s) {
            if (__ldg(mr + s / p.block_len) == 0) continue;
            const int64_t from = base + (int64_t)s * p.state_stride;
            float x = 0.f;
#pragma unroll
            for (int i = 0; i < kPer; ++i) x += qv[i] * __bfloat162float(p.k[from + i]);
#pragma unroll
            for (int d = 16; d > 0; d >>= 1) x += __shfl_xor_sync(kFull, x, d);
            const float pr = exp2_fast(fmaf(x, c, -rm));
#pragma unroll
            for (int i = 0; i < kPer; ++i) acc[i] += pr * __bfloat162float(p.v[from + i]);
          }
          const size_t ra = ((size_t)g.b * p.n_tokens + rt) * p.n_q_heads + g.kvh * p.group + rr % p.group;
          __syncwarp();  // after the row's own thread has written it
#pragma unroll
          for (int i = 0; i < kPer; ++i) {
            const uint32_t col = lane * kPer + i;
            if (whole)
              p.out[ra * D + col] = __float2bfloat16_rn(rl == 0.f ? 0.f : acc[i] / rl);
            else
              mine[(col / 4u * kRows + rs) * 4u + col % 4u] = acc[i];
          }
        }
      }
      if (!whole && live) {
        mine[kRows * 128 + slot] = m;
        mine[kRows * 129 + slot] = l;
      }
    }
  }

  if (!ok) {
    *dead = 1u;
    if (lane == 0) atomicOr(p.ws.status, TQ_STATUS_WAIT_EXPIRED);
    // copies that are still in flight target this CTA's shared memory: give them time to land
    for (int i = 0; i < 2000; ++i) __nanosleep(1000);
  }
  tmem_fence_before();
  __syncthreads();
  if (warp == kMmaWarp) {
    tmem_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kTmemCols) : "memory");
  }
}

// Joins the parts of the groups that were cut.  grid (groups, or CTAs of the kernel above, slices of 8 rows): block (x, y) has
// the cut group x, or the one that begins in CTA x's share and goes on, if there is one; a thread has four columns of a
// row and adds the parts up in their order.  After an expired wait the entries may be an earlier call's (then the outputs are
// not valid, and nothing beside them is written): a block that goes by the group's number takes no other group, and a number past the
// last group is not followed.
constexpr uint32_t kJoinRows = 8;
template <int D>
__global__ void __launch_bounds__(kJoinRows * D / 4) cross_join_kernel(const CrossParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const uint4 g = p.ws.open[blockIdx.x];  // parts, first CTA, number of the group
  const uint32_t id = p.by_group ? blockIdx.x : g.z;
  if (g.x == 0u || id >= p.n_seqs * p.n_kv_heads * p.row_tiles) return;
  const uint32_t bh = id / p.row_tiles, qt = id - bh * p.row_tiles, b = bh / p.n_kv_heads, kvh = bh - b * p.n_kv_heads;
  const uint32_t slot = blockIdx.y * kJoinRows + threadIdx.x % kJoinRows, row = qt * kRows + slot, quad = threadIdx.x / kJoinRows;
  if (row >= p.rows) return;
  auto part = [&](uint32_t i) { return p.ws.parts + (size_t)(2u * (g.y + i) + (i == 0u ? 1u : 0u)) * kCrossPartFloats; };
  float M = -INFINITY, l = 0.f;
  float4 o = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (uint32_t i = 0; i < g.x; ++i) {
    const float* src = part(i);
    const float mi = __ldcg(src + kRows * 128 + slot), li = __ldcg(src + kRows * 129 + slot);
    const float4 y = __ldcg(reinterpret_cast<const float4*>(src) + quad * kRows + slot);
    const float mn = fmaxf(M, mi), ref = mn == -INFINITY ? 0.f : mn, f = exp2_fast(M - ref), h = exp2_fast(mi - ref);
    M = mn;
    l = l * f + li * h;
    o.x = o.x * f + y.x * h;
    o.y = o.y * f + y.y * h;
    o.z = o.z * f + y.z * h;
    o.w = o.w * f + y.w * h;
  }
  const size_t at = ((size_t)b * p.n_tokens + row / p.group) * p.n_q_heads + kvh * p.group + row % p.group;
  const float inv = l == 0.f ? 0.f : 1.0f / l;
  *reinterpret_cast<uint2*>(p.out + at * D + 4u * quad) =
      l == 0.f ? make_uint2(0u, 0u) : make_uint2(pack_bf16(o.x * inv, o.y * inv), pack_bf16(o.z * inv, o.w * inv));
  if (quad == 0u && p.lse) p.lse[at] = l == 0.f ? -INFINITY : (M + log2f(l)) * 0.6931471805599453f;
}

// The tensor map of K or V: (column, state, head, sequence), boxes of 64 columns x 128 states, 128-byte swizzle.
// A dimension of stride 0 is one that every index shares.
bool encode(CUtensorMap* map, const void* base, const tq_encoder_kv* kv) {
  EncodeTiledFn fn = encode_fn();
  if (!fn) return false;
  const cuuint64_t row = kv->head_dim * 2u;
  const cuuint64_t dims[4] = {kv->head_dim, kv->n_states, kv->head_stride ? kv->n_kv_heads : 1u, kv->batch_stride ? kv->n_seqs : 1u};
  const cuuint64_t strides[3] = {kv->state_stride ? (cuuint64_t)kv->state_stride * 2u : row, kv->head_stride ? (cuuint64_t)kv->head_stride * 2u : row,
                                 kv->batch_stride ? (cuuint64_t)kv->batch_stride * 2u : row};
  const cuuint32_t box[4] = {64u, kStates, 1u, 1u}, step[4] = {1u, 1u, 1u, 1u};
  return fn(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
int launch(const CrossParams& p, const CUtensorMap& k_map, const CUtensorMap& v_map, cudaStream_t st) {
  auto kern = cross_attention_kernel<D>;
  constexpr size_t smem = CrossSmem<D>::kTotal + 1024;
  const char* what = "cross attention (tensor core) launch";
  if (int rc = tq_ensure_dynamic_smem((const void*)kern, smem, what)) return rc;
  static const int regs = [&] {
    cudaFuncAttributes a{};
    return cudaFuncGetAttributes(&a, (const void*)kern) == cudaSuccess ? a.numRegs : 0;
  }();
  if (256 * kSoftRegs + 128 * kOtherRegs > kCrossThreads * regs) return tq_cuda_status((int)cudaErrorInvalidConfiguration, what);
  const uint32_t grid = min((uint32_t)sm_count(), kAttnMaxCtas);
  if (int rc = launch_pdl(kern, dim3(grid), kCrossThreads, smem, st, what, p, k_map, v_map)) return rc;
  const uint32_t x = p.by_group ? p.n_seqs * p.n_kv_heads * p.row_tiles : grid;
  return launch_pdl(cross_join_kernel<D>, dim3(x, (min(kRows, p.rows) + kJoinRows - 1u) / kJoinRows), kJoinRows * D / 4, 0, st, "cross attention (join) launch", p);
}

std::atomic<int> g_test_withhold{0};

}  // namespace

extern "C" void tq_test_withhold_cross_entry(int on) { g_test_withhold.store(on ? 1 : 0); }

uint64_t tq_cross_workspace_bytes() { return (uint64_t)min((uint32_t)sm_count(), kAttnMaxCtas) * 2u * kCrossPartFloats * sizeof(float); }

int tq_cross_launch(const tq_encoder_kv* kv, const void* d_q, int64_t q_batch_stride, int64_t q_token_stride, uint32_t n_tokens,
                    uint32_t n_q_heads, const int32_t* d_kv_len, const uint8_t* d_mask, uint32_t block_len, uint32_t n_blocks,
                    float scale_log2, void* d_out, float* d_lse, const tq_attn_ws& ws, void* cuda_stream, bool* served) {
  CUtensorMap k_map, v_map;
  const uint64_t units = (uint64_t)kv->n_seqs * kv->n_kv_heads * (((uint64_t)n_tokens * (n_q_heads / kv->n_kv_heads) + kRows - 1u) / kRows) *
                         (((uint64_t)kv->n_states + kStates - 1u) / kStates);
  *served = units < 0xFFFFFFFFull && kv->n_states != 0 && (kv->state_stride != 0 || kv->n_states == 1) && encode(&k_map, kv->d_k, kv) && encode(&v_map, kv->d_v, kv);
  if (!*served) return TQ_OK;
  CrossParams p{};
  p.k = (const __nv_bfloat16*)kv->d_k;
  p.v = (const __nv_bfloat16*)kv->d_v;
  p.batch_stride = kv->batch_stride;
  p.state_stride = kv->state_stride;
  p.head_stride = kv->head_stride;
  p.q = (const __nv_bfloat16*)d_q;
  p.q_batch_stride = q_batch_stride;
  p.q_token_stride = q_token_stride;
  p.out = (__nv_bfloat16*)d_out;
  p.lse = d_lse;
  p.kv_len = d_kv_len;
  p.mask = d_mask;
  p.n_states = kv->n_states;
  p.block_len = block_len;
  p.n_blocks = n_blocks;
  p.n_seqs = kv->n_seqs;
  p.n_tokens = n_tokens;
  p.n_q_heads = n_q_heads;
  p.n_kv_heads = kv->n_kv_heads;
  p.group = n_q_heads / kv->n_kv_heads;
  p.rows = n_tokens * p.group;
  p.row_tiles = (p.rows + kRows - 1u) / kRows;
  p.scale_log2 = scale_log2;
  p.by_group = (uint64_t)kv->n_seqs * kv->n_kv_heads * p.row_tiles <= kAttnMaxCtas;
  p.counted = d_mask != nullptr && block_len >= kStates && n_blocks <= kCountBlocks && kv->n_states <= 65535u * kStates &&
              (uint64_t)kv->n_seqs * p.row_tiles <= kCounts && (uint64_t)kv->n_seqs * n_tokens * n_blocks <= kCountBytes;
  p.test_withhold = (uint32_t)g_test_withhold.load();
  p.ws = ws;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  return kv->head_dim == 64 ? launch<64>(p, k_map, v_map, st) : launch<128>(p, k_map, v_map, st);
}
