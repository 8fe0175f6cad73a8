// Root-mean-square norm of the residual stream with the addition of a layer's output (tq_rmsnorm,
// tq_rmsnorm_q8).
//
//   s = h + delta,  r = 1 / sqrt(mean_c s_c^2 + eps),  n_c = (s_c * r) * w_c
//
// One pass: a row's sums s stay in the registers of the threads that read it (8 or 16 a thread), so
// h and delta are read once and the row is scaled from registers when its sum of squares is known.
// Everything is fp32; h_out is rounded to h's type after s has gone into the norm, out once.  r is rsqrtf's (within 2 units of
// the last place), so that it is the r of elementary operations wherever the sum is: of the rows of 8-bit levels fewer differ in
// single levels from such a form (1023 x 4096: 2.8 of 4.2 million levels with 1 / sqrtf, 1.8 with rsqrtf; the rest is the order of
// the sum and the division by 127).
// A call moves 2-12 bytes per element for about 6 operations: memory bound, and for few rows bound by
// the latency of one load, one reduction and one store.
#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "tq_internal.h"
#include "tq_ops_common.cuh"

namespace {

using namespace tq_ops;

struct NormParams {
  const void* h;
  const void* delta;
  const float* w;
  void* h_out;
  __nv_bfloat16* out;
  int8_t* q;
  float* q_scale;
  int64_t h_stride, delta_stride;
  float eps;
  uint32_t rows, cols;
};

enum { kNone = 2 };  // beside TQ_TYPE_BF16 and TQ_TYPE_F32: no delta

// Where element e of unit u of a thread lies in its row: eight consecutive columns to a unit, or single
// columns a row's threads apart where 16-byte accesses are not allowed.
template <bool VEC>
__device__ __forceinline__ uint32_t column(uint32_t u, int e, uint32_t tid, uint32_t threads) {
  return VEC ? (u * threads + tid) * 8u + (uint32_t)e : (u * 8u + (uint32_t)e) * threads + tid;
}

// The sums of a unit.
template <int HT, int DT, class H, class Dl>
__device__ __forceinline__ void add(const H& h, const Dl& d, float (&s)[8]) {
  h.get(s);
  if constexpr (DT != kNone) {
    float x[8];
    d.get(x);
#pragma unroll
    for (int e = 0; e < 8; ++e) s[e] += x[e];
  }
}
__device__ __forceinline__ float squares(const float (&s)[8]) {
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum = fmaf(s[e], s[e], sum);
  return sum;
}
__device__ __forceinline__ void load_weights(const float* w, float (&f)[8]) {
  Raw8<TQ_TYPE_F32> raw;
  raw.load_cached(w, 0);
  raw.get(f);
}
// 8 bits by the rule of tq_quantize_rows: amax is the row's largest magnitude (NaN if it has one), then IEEE division and
// rounding half to even.  Where amax / 127 rounds to 0 (below 64 * 2^-149) the row counts as zeros.
__device__ __forceinline__ float scale_of(float amax) {
  const float s = __fdiv_rn(amax, 127.0f);
  return s == 0.f ? 1.0f : s;
}
__device__ __forceinline__ void levels(float (&n)[8], float scale, int8_t (&b)[8]) {
  if (scale < 0x1p-100f) {  // 1 / scale may overflow: both sides of the quotient 2^64 times as large, which is exact
    scale *= 0x1p64f;
#pragma unroll
    for (int e = 0; e < 8; ++e) n[e] *= 0x1p64f;
  }
  const float inv = 1.0f / scale;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    // the product with 1 / scale is within 2^-16 of the quotient: only near a half can the two round differently, and there
    // the quotient itself is taken
    const float v = n[e] * inv;
    float r = rintf(v);
    if (fabsf(fabsf(v - r) - 0.5f) < 1e-3f) r = rintf(__fdiv_rn(n[e], scale));
    b[e] = scale == scale ? (int8_t)fminf(fmaxf(r, -127.f), 127.f) : (int8_t)0;
  }
}

// One row to a block.
template <int HT, int DT, bool VEC, int NU>
__global__ void __launch_bounds__(1024) rmsnorm_kernel(const NormParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t threads = blockDim.x, tid = threadIdx.x, row = blockIdx.x;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  float s[NU][8];
  const size_t hb = (size_t)row * p.h_stride, db = (size_t)row * p.delta_stride, ob = (size_t)row * p.cols;
  if constexpr (VEC) {
    Raw8<HT> hr[NU];
    Raw8<DT == kNone ? TQ_TYPE_BF16 : DT> dr[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const uint32_t c = column<true>(u, 0, tid, threads);
      hr[u].clear();
      dr[u].clear();
      if (c < p.cols) {
        hr[u].load(p.h, hb + c);
        if constexpr (DT != kNone) dr[u].load(p.delta, db + c);
      }
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) add<HT, DT>(hr[u], dr[u], s[u]);
  } else {
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t c = column<false>(u, e, tid, threads);
        float v = 0.f;
        if (c < p.cols) {
          v = load1<HT>(p.h, hb + c);
          if constexpr (DT != kNone) v += load1<DT>(p.delta, db + c);
        }
        s[u][e] = v;
      }
  }

  // the weights and the store of the sums do not wait for the reduction
  Raw8<TQ_TYPE_F32> w[NU];
  if constexpr (VEC) {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const uint32_t c = column<true>(u, 0, tid, threads);
      if (c >= p.cols) continue;
      w[u].load_cached(p.w, c);
      if (p.h_out) store8<HT>(p.h_out, hb + c, s[u]);
    }
  }
  float sum = 0.f;
#pragma unroll
  for (int u = 0; u < NU; ++u) sum += squares(s[u]);
  __shared__ float red[2][32];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
  if (lane == 0) red[0][warp] = sum;
  __syncthreads();
  sum = lane < (blockDim.x >> 5) ? red[0][lane] : 0.f;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
  const float r = rsqrtf(sum / (float)p.cols + p.eps);

  float amax = 0.f;
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    if constexpr (VEC) {
      const uint32_t c = column<true>(u, 0, tid, threads);
      if (c >= p.cols) continue;
      float f[8];
      w[u].get(f);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[u][e] = s[u][e] * r * f[e];
      if (p.out) store8<TQ_TYPE_BF16>(p.out, ob + c, s[u]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t c = column<false>(u, e, tid, threads);
        if (c >= p.cols) continue;
        if (p.h_out) store1<HT>(p.h_out, hb + c, s[u][e]);
        s[u][e] = s[u][e] * r * __ldg(p.w + c);
        if (p.out) store1<TQ_TYPE_BF16>(p.out, ob + c, s[u][e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = max_nan(amax, fabsf(s[u][e]));
  }
  if (p.q == nullptr) return;

#pragma unroll
  for (int d = 16; d > 0; d >>= 1) amax = max_nan(amax, __shfl_xor_sync(kFull, amax, d));
  if (lane == 0) red[1][warp] = amax;
  __syncthreads();
  amax = lane < (blockDim.x >> 5) ? red[1][lane] : 0.f;
#pragma unroll
  for (int d = 16; d > 0; d >>= 1) amax = max_nan(amax, __shfl_xor_sync(kFull, amax, d));
  const float scale = scale_of(amax);
  if (tid == 0) p.q_scale[row] = scale;
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    int8_t b[8];
    levels(s[u], scale, b);
    if constexpr (VEC) {
      const uint32_t c = column<true>(u, 0, tid, threads);
      if (c < p.cols) *reinterpret_cast<uint2*>(p.q + ob + c) = *reinterpret_cast<const uint2*>(b);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t c = column<false>(u, e, tid, threads);
        if (c < p.cols) p.q[ob + c] = b[e];
      }
    }
  }
}

// Short rows (heads): TPR lanes to a row, one unit of eight columns a lane, shuffles only; a lane works on NR rows at once, so
// that it has NR loads under way, with one load of its weights.  Rows that are not aligned for units go the long way above.
constexpr uint32_t kShortThreads = 128;
template <int HT, int DT, int TPR, int NR>
__global__ void __launch_bounds__(kShortThreads) rmsnorm_short_kernel(const NormParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  constexpr uint32_t kSide = kShortThreads / TPR;
  const uint32_t c = threadIdx.x % TPR * 8u, row0 = blockIdx.x * (kSide * NR) + threadIdx.x / TPR;
  const bool live = c < p.cols;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  Raw8<HT> hr[NR];
  Raw8<DT == kNone ? TQ_TYPE_BF16 : DT> dr[NR];
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    const uint32_t row = row0 + k * kSide;
    hr[k].clear();
    dr[k].clear();
    if (live && row < p.rows) {
      hr[k].load(p.h, (size_t)row * p.h_stride + c);
      if constexpr (DT != kNone) dr[k].load(p.delta, (size_t)row * p.delta_stride + c);
    }
  }
  float w[8] = {};
  if (live) load_weights(p.w + c, w);
#pragma unroll
  for (int k = 0; k < NR; ++k) {
    const uint32_t row = row0 + k * kSide;
    const bool mine = live && row < p.rows;
    float s[8];
    add<HT, DT>(hr[k], dr[k], s);
    float sum = squares(s);
#pragma unroll
    for (int d = TPR / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
    const float r = rsqrtf(sum / (float)p.cols + p.eps);
    if (mine && p.h_out) store8<HT>(p.h_out, (size_t)row * p.h_stride + c, s);
    float amax = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      s[e] = s[e] * r * w[e];
      if (live) amax = max_nan(amax, fabsf(s[e]));
    }
    if (mine && p.out) store8<TQ_TYPE_BF16>(p.out, (size_t)row * p.cols + c, s);
    if (p.q == nullptr) continue;
#pragma unroll
    for (int d = TPR / 2; d > 0; d >>= 1) amax = max_nan(amax, __shfl_xor_sync(kFull, amax, d));
    const float scale = scale_of(amax);
    int8_t b[8];
    levels(s, scale, b);
    if (mine) *reinterpret_cast<uint2*>(p.q + (size_t)row * p.cols + c) = *reinterpret_cast<const uint2*>(b);
    if (mine && c == 0u) p.q_scale[row] = scale;
  }
}

template <int HT, int DT, bool VEC>
int launch(const NormParams& p, cudaStream_t st) {
  const char* what = "rmsnorm launch";
  const uint32_t units = (p.cols + 7u) / 8u, sms = (uint32_t)sm_count();
  if constexpr (VEC) {
    if (units <= 32u) {
      // one row a lane until the device is full of blocks, four beyond (51232 rows of 128: 7.9 us with one, 5.7 with four)
      auto grid = [&](uint32_t tpr, uint32_t nr) { return (p.rows + kShortThreads / tpr * nr - 1u) / (kShortThreads / tpr * nr); };
      const uint32_t tpr = units <= 16u ? 16u : 32u;
      const bool many = grid(tpr, 4u) >= 4u * sms;
      if (tpr == 16u)
        return many ? launch_pdl(rmsnorm_short_kernel<HT, DT, 16, 4>, dim3(grid(16, 4)), kShortThreads, 0, st, what, p)
                    : launch_pdl(rmsnorm_short_kernel<HT, DT, 16, 1>, dim3(grid(16, 1)), kShortThreads, 0, st, what, p);
      return many ? launch_pdl(rmsnorm_short_kernel<HT, DT, 32, 4>, dim3(grid(32, 4)), kShortThreads, 0, st, what, p)
                  : launch_pdl(rmsnorm_short_kernel<HT, DT, 32, 1>, dim3(grid(32, 1)), kShortThreads, 0, st, what, p);
    }
  }
  // One unit a thread where rows are few and the latency of a row counts, two where there are many (2049 rows of 8192 fp32
  // with an fp32 delta: 36.9 us = 6.4 TB/s with two, 40.5 with one, 40.9 with four).  1024 threads of two units are
  // TQ_NORM_MAX_COLS columns.
  auto threads = [&](uint32_t nu) { return ((units + nu - 1u) / nu + 31u) / 32u * 32u; };
  if (p.rows < 2u * sms && units <= 1024u) return launch_pdl(rmsnorm_kernel<HT, DT, VEC, 1>, dim3(p.rows), threads(1), 0, st, what, p);
  return launch_pdl(rmsnorm_kernel<HT, DT, VEC, 2>, dim3(p.rows), threads(2), 0, st, what, p);
}

template <int HT, int DT>
int launch_vec(const NormParams& p, cudaStream_t st) {
  auto fits = [](const void* ptr, int64_t stride, int type) {
    return ((uintptr_t)ptr & (type == TQ_TYPE_F32 ? 31u : 15u)) == 0 && stride % 8 == 0;  // eight elements are one access
  };
  bool vec = p.cols % 8u == 0 && fits(p.h, p.h_stride, HT) && fits(p.w, 0, TQ_TYPE_F32);
  if (DT != kNone) vec = vec && fits(p.delta, p.delta_stride, DT);
  if (p.h_out) vec = vec && fits(p.h_out, p.h_stride, HT);
  vec = vec && ((uintptr_t)p.out & 15u) == 0 && ((uintptr_t)p.q & 7u) == 0;
  return vec ? launch<HT, DT, true>(p, st) : launch<HT, DT, false>(p, st);
}

int norm(const void* d_h, int h_type, int64_t h_stride, const void* d_delta, int delta_type, int64_t delta_stride,
         const float* d_weight, float eps, uint32_t rows, uint32_t cols, void* d_h_out, void* d_out, int8_t* d_q,
         float* d_scale, void* cuda_stream) {
  auto type_ok = [](int t) { return t == TQ_TYPE_BF16 || t == TQ_TYPE_F32; };
  auto aligned = [](const void* ptr, int type) { return ((uintptr_t)ptr & (type == TQ_TYPE_F32 ? 3u : 1u)) == 0; };
  if (!type_ok(h_type) || (d_delta && !type_ok(delta_type)) || cols == 0 || !(eps >= 0.f)) return TQ_ERR_INVALID_ARG;
  if (cols > TQ_NORM_MAX_COLS || rows > 0x7FFFFFFFu) return TQ_ERR_UNSUPPORTED_SHAPE;
  if (rows == 0) return TQ_OK;
  if (!d_h || !d_weight || !aligned(d_h, h_type) || !aligned(d_weight, TQ_TYPE_F32) || !aligned(d_h_out, h_type)) return TQ_ERR_INVALID_ARG;
  if (d_delta && !aligned(d_delta, delta_type)) return TQ_ERR_INVALID_ARG;
  if ((rows > 1 && (h_stride < (int64_t)cols || (d_delta && delta_stride < (int64_t)cols)))) return TQ_ERR_INVALID_ARG;
  NormParams p{d_h, d_delta, d_weight, d_h_out, (__nv_bfloat16*)d_out, d_q, d_scale, h_stride, delta_stride, eps, rows, cols};
  cudaStream_t st = (cudaStream_t)cuda_stream;
  const int dt = d_delta ? delta_type : kNone;
  if (h_type == TQ_TYPE_BF16) {
    if (dt == kNone) return launch_vec<TQ_TYPE_BF16, kNone>(p, st);
    return dt == TQ_TYPE_BF16 ? launch_vec<TQ_TYPE_BF16, TQ_TYPE_BF16>(p, st) : launch_vec<TQ_TYPE_BF16, TQ_TYPE_F32>(p, st);
  }
  if (dt == kNone) return launch_vec<TQ_TYPE_F32, kNone>(p, st);
  return dt == TQ_TYPE_BF16 ? launch_vec<TQ_TYPE_F32, TQ_TYPE_BF16>(p, st) : launch_vec<TQ_TYPE_F32, TQ_TYPE_F32>(p, st);
}

}  // namespace

extern "C" {

int tq_rmsnorm(const void* d_h, int h_type, int64_t h_stride, const void* d_delta, int delta_type, int64_t delta_stride,
               const float* d_weight, float eps, uint32_t rows, uint32_t cols, void* d_h_out, void* d_out_bf16,
               void* cuda_stream) {
  if (rows && (!d_out_bf16 || ((uintptr_t)d_out_bf16 & 1u))) return TQ_ERR_INVALID_ARG;
  return norm(d_h, h_type, h_stride, d_delta, delta_type, delta_stride, d_weight, eps, rows, cols, d_h_out, d_out_bf16, nullptr,
              nullptr, cuda_stream);
}

int tq_rmsnorm_q8(const void* d_h, int h_type, int64_t h_stride, const void* d_delta, int delta_type, int64_t delta_stride,
                  const float* d_weight, float eps, uint32_t rows, uint32_t cols, void* d_h_out, int8_t* d_q, float* d_scale,
                  void* cuda_stream) {
  if (rows && (!d_q || !d_scale || ((uintptr_t)d_scale & 3u))) return TQ_ERR_INVALID_ARG;
  return norm(d_h, h_type, h_stride, d_delta, delta_type, delta_stride, d_weight, eps, rows, cols, d_h_out, nullptr, d_q, d_scale,
              cuda_stream);
}

}  // extern "C"
