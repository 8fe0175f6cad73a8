// Root-mean-square norm of the residual stream with the addition of a layer's output (tq_rmsnorm,
// tq_rmsnorm_q8).
//
//   s = h + delta,  r = 1 / sqrt(mean_c s_c^2 + eps),  n_c = (s_c * r) * w_c
//
// One pass: a row's sums s stay in the registers of the threads that read it (8, 16 or 32 a thread), so
// h and delta are read once and the row is scaled from registers when its sum of squares is known.
// Everything is fp32; h_out is rounded to h's type after s has gone into the norm, out once.
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

// TPR: threads of a row: 16 or 32 (several rows to a block of 128, shuffles only) or 0 (the whole block).
template <int HT, int DT, bool VEC, int TPR, int NU>
__global__ void __launch_bounds__(TPR ? 128 : (NU == 4 ? 512 : 1024)) rmsnorm_kernel(const NormParams p) {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  const uint32_t threads = TPR ? TPR : blockDim.x;
  const uint32_t tid = TPR ? threadIdx.x % (TPR ? TPR : 1) : threadIdx.x;
  const uint32_t row = TPR ? blockIdx.x * (128u / (TPR ? TPR : 1)) + threadIdx.x / (TPR ? TPR : 1) : blockIdx.x;
  const bool live = row < p.rows;
  asm volatile("griddepcontrol.wait;" ::: "memory");

  float s[NU][8];
  const size_t hb = (size_t)row * p.h_stride, db = (size_t)row * p.delta_stride;
  if constexpr (VEC) {
    Raw8<HT> hr[NU];
    Raw8<DT == kNone ? TQ_TYPE_BF16 : DT> dr[NU];
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      const uint32_t c = column<true>(u, 0, tid, threads);
      if (live && c < p.cols) {
        hr[u].load(p.h, hb + c);
        if constexpr (DT != kNone) dr[u].load(p.delta, db + c);
      } else {
        hr[u].clear();
        if constexpr (DT != kNone) dr[u].clear();
      }
    }
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      hr[u].get(s[u]);
      if constexpr (DT != kNone) {
        float d[8];
        dr[u].get(d);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[u][e] += d[e];
      }
    }
  } else {
#pragma unroll
    for (int u = 0; u < NU; ++u)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t c = column<false>(u, e, tid, threads);
        float v = 0.f;
        if (live && c < p.cols) {
          v = load1<HT>(p.h, hb + c);
          if constexpr (DT != kNone) v += load1<DT>(p.delta, db + c);
        }
        s[u][e] = v;
      }
  }

  float sum = 0.f;
#pragma unroll
  for (int u = 0; u < NU; ++u)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf(s[u][e], s[u][e], sum);
  __shared__ float red[2][32];
  const uint32_t lane = threadIdx.x & 31u, warp = threadIdx.x >> 5;
#pragma unroll
  for (int d = (TPR ? TPR : 32) / 2; d > 0; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
  if (TPR == 0) {
    if (lane == 0) red[0][warp] = sum;
    __syncthreads();
    sum = lane < (blockDim.x >> 5) ? red[0][lane] : 0.f;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) sum += __shfl_xor_sync(kFull, sum, d);
  }
  const float r = 1.0f / sqrtf(sum / (float)p.cols + p.eps);

  const size_t ob = (size_t)row * p.cols;
  if (p.h_out != nullptr) {
#pragma unroll
    for (int u = 0; u < NU; ++u) {
      if constexpr (VEC) {
        const uint32_t c = column<true>(u, 0, tid, threads);
        if (live && c < p.cols) store8<HT>(p.h_out, hb + c, s[u]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint32_t c = column<false>(u, e, tid, threads);
          if (live && c < p.cols) store1<HT>(p.h_out, hb + c, s[u][e]);
        }
      }
    }
  }
  float amax = 0.f;
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    if constexpr (VEC) {
      const uint32_t c = column<true>(u, 0, tid, threads);
      if (!(live && c < p.cols)) continue;
      float w[8];
      Raw8<TQ_TYPE_F32> wr;
      wr.load_cached(p.w, c);
      wr.get(w);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[u][e] = s[u][e] * r * w[e];
      if (p.out) store8<TQ_TYPE_BF16>(p.out, ob + c, s[u]);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t c = column<false>(u, e, tid, threads);
        if (!(live && c < p.cols)) continue;
        s[u][e] = s[u][e] * r * __ldg(p.w + c);
        if (p.out) store1<TQ_TYPE_BF16>(p.out, ob + c, s[u][e]);
      }
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) amax = max_nan(amax, fabsf(s[u][e]));
  }
  if (p.q == nullptr) return;

  // 8 bits: the row's largest magnitude (a NaN anywhere makes it NaN), then IEEE division and rounding
  // half to even, as tq_quantize_rows does it
#pragma unroll
  for (int d = (TPR ? TPR : 32) / 2; d > 0; d >>= 1) amax = max_nan(amax, __shfl_xor_sync(kFull, amax, d));
  if (TPR == 0) {
    if (lane == 0) red[1][warp] = amax;
    __syncthreads();
    amax = lane < (blockDim.x >> 5) ? red[1][lane] : 0.f;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) amax = max_nan(amax, __shfl_xor_sync(kFull, amax, d));
  }
  const float scale = amax == 0.f ? 1.0f : __fdiv_rn(amax, 127.0f);
  if (live && tid == 0) p.q_scale[row] = scale;
#pragma unroll
  for (int u = 0; u < NU; ++u) {
    int8_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float v = rintf(__fdiv_rn(s[u][e], scale));
      b[e] = amax == amax ? (int8_t)fminf(fmaxf(v, -127.f), 127.f) : (int8_t)0;
    }
    if constexpr (VEC) {
      const uint32_t c = column<true>(u, 0, tid, threads);
      if (live && c < p.cols) *reinterpret_cast<uint2*>(p.q + ob + c) = *reinterpret_cast<const uint2*>(b);
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const uint32_t c = column<false>(u, e, tid, threads);
        if (live && c < p.cols) p.q[ob + c] = b[e];
      }
    }
  }
}

template <int HT, int DT, bool VEC>
int launch(const NormParams& p, cudaStream_t st) {
  const uint32_t units = (p.cols + 7u) / 8u;
  if (units <= 16u) return launch_pdl(rmsnorm_kernel<HT, DT, VEC, 16, 1>, dim3((p.rows + 7u) / 8u), 128, 0, st, "rmsnorm launch", p);
  if (units <= 32u) return launch_pdl(rmsnorm_kernel<HT, DT, VEC, 32, 1>, dim3((p.rows + 3u) / 4u), 128, 0, st, "rmsnorm launch", p);
  // few rows: as many threads as the row has units, for latency; many rows: four units a thread, for
  // bytes in flight (512 threads of four units or 1024 of two are TQ_NORM_MAX_COLS columns)
  const bool few = p.rows < 2u * (uint32_t)sm_count();
  auto threads_for = [&](uint32_t nu) { return ((units + nu - 1u) / nu + 31u) / 32u * 32u; };
  if (!few) return launch_pdl(rmsnorm_kernel<HT, DT, VEC, 0, 4>, dim3(p.rows), threads_for(4), 0, st, "rmsnorm launch", p);
  if (units <= 1024u) return launch_pdl(rmsnorm_kernel<HT, DT, VEC, 0, 1>, dim3(p.rows), threads_for(1), 0, st, "rmsnorm launch", p);
  return launch_pdl(rmsnorm_kernel<HT, DT, VEC, 0, 2>, dim3(p.rows), threads_for(2), 0, st, "rmsnorm launch", p);
}

template <int HT, int DT>
int launch_vec(const NormParams& p, cudaStream_t st) {
  auto fits = [](const void* ptr, int64_t stride, int type) {
    const int64_t step = type == TQ_TYPE_F32 ? 4 : 8;  // elements in 16 bytes
    return ((uintptr_t)ptr & 15u) == 0 && stride % step == 0;
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
