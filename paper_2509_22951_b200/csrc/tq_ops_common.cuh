// What the operators between the linear layers share: typed loads and stores of eight elements, the
// launch with programmatic stream serialisation.
#pragma once

#include <cuda_bf16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "tq_internal.h"
#include "tq_sm100.cuh"

namespace tq_ops {

constexpr unsigned kFull = 0xFFFFFFFFu;
using tq_sm100::sm_count;

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xFFFF0000u); }
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
// A NaN on either side is the result (fmaxf drops it).
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// Data read once: not kept in L1.  (Plain loads, not .nc: a kernel may write the array it reads, in place.)
__device__ __forceinline__ uint4 load_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p) : "memory");
  return v;
}

// 32 bytes to a lane in one access: a warp's lanes fill whole sectors.  (Two accesses of 16 bytes 32 bytes apart touch every
// sector twice: the norm of an fp32 stream moved 2.1 x its bytes through L2 that way.)
__device__ __forceinline__ void load_once_32(const void* p, uint4& a, uint4& b) {
  asm volatile("ld.global.L1::no_allocate.v8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
               : "=r"(a.x), "=r"(a.y), "=r"(a.z), "=r"(a.w), "=r"(b.x), "=r"(b.y), "=r"(b.z), "=r"(b.w)
               : "l"(p)
               : "memory");
}
__device__ __forceinline__ void store_32(void* p, const float (&f)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]),
               "f"(f[6]), "f"(f[7])
               : "memory");
}

// Eight consecutive elements as they lie in memory; the conversion waits for the data, so a thread asks
// for all of its units before it converts the first.
template <int TYPE>
struct Raw8;
template <>
struct Raw8<TQ_TYPE_BF16> {
  uint4 a;
  __device__ __forceinline__ void load(const void* base, size_t i) { a = load_once((const __nv_bfloat16*)base + i); }
  __device__ __forceinline__ void clear() { a = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = bf16_lo(a.x), f[1] = bf16_hi(a.x), f[2] = bf16_lo(a.y), f[3] = bf16_hi(a.y);
    f[4] = bf16_lo(a.z), f[5] = bf16_hi(a.z), f[6] = bf16_lo(a.w), f[7] = bf16_hi(a.w);
  }
};
template <>
struct Raw8<TQ_TYPE_F32> {
  uint4 a, b;
  __device__ __forceinline__ void load(const void* base, size_t i) {
    load_once_32((const float*)base + i, a, b);
  }
  __device__ __forceinline__ void load_cached(const void* base, size_t i) {
    a = __ldg(reinterpret_cast<const uint4*>((const float*)base + i));
    b = __ldg(reinterpret_cast<const uint4*>((const float*)base + i + 4));
  }
  __device__ __forceinline__ void clear() { a = b = make_uint4(0, 0, 0, 0); }
  __device__ __forceinline__ void get(float (&f)[8]) const {
    f[0] = __uint_as_float(a.x), f[1] = __uint_as_float(a.y), f[2] = __uint_as_float(a.z), f[3] = __uint_as_float(a.w);
    f[4] = __uint_as_float(b.x), f[5] = __uint_as_float(b.y), f[6] = __uint_as_float(b.z), f[7] = __uint_as_float(b.w);
  }
};

__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack_bf16(f[0], f[1]), pack_bf16(f[2], f[3]), pack_bf16(f[4], f[5]), pack_bf16(f[6], f[7]));
}
template <int TYPE>
__device__ __forceinline__ void store8(void* base, size_t i, const float (&f)[8]) {
  if constexpr (TYPE == TQ_TYPE_BF16) {
    *reinterpret_cast<uint4*>((__nv_bfloat16*)base + i) = pack8(f);
  } else {
    store_32((float*)base + i, f);
  }
}
template <int TYPE>
__device__ __forceinline__ float load1(const void* base, size_t i) {
  if constexpr (TYPE == TQ_TYPE_BF16) return __bfloat162float(((const __nv_bfloat16*)base)[i]);
  return ((const float*)base)[i];
}
template <int TYPE>
__device__ __forceinline__ void store1(void* base, size_t i, float v) {
  if constexpr (TYPE == TQ_TYPE_BF16)
    ((__nv_bfloat16*)base)[i] = __float2bfloat16_rn(v);
  else
    ((float*)base)[i] = v;
}

// Launch with programmatic stream serialisation: the kernel may start while the one before it in the
// stream still runs, so it executes griddepcontrol.wait before it touches memory.
template <class... Formal, class... Actual>
int launch_pdl(void (*kern)(Formal...), dim3 grid, uint32_t threads, size_t smem, cudaStream_t st, const char* what, const Actual&... args) {
  cudaLaunchConfig_t cfg{};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return tq_cuda_status((int)cudaLaunchKernelEx(&cfg, kern, args...), what);
}

}  // namespace tq_ops
