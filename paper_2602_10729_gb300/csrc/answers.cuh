// What the kernels over a model's answers share: the logits' element types,
// the checks of their C entry points, and the shared memory of a cluster's blocks.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.h"
#include "regions.h"
#include "warp_select.cuh"

namespace boute {

__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
// (one rounding to nearest even)
template <class T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __half from_float<__half>(float x) { return __float2half_rn(x); }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) {
  return __float2bfloat16_rn(x);
}

// A word's two 16-bit elements as floats, and back with one rounding each.
__device__ __forceinline__ void unpack2(__half, uint32_t w, float &a, float &b) {
  unpack_f16x2(w, a, b);
}
__device__ __forceinline__ void unpack2(__nv_bfloat16, uint32_t w, float &a, float &b) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ uint32_t pack2(__half, float a, float b) { return pack_f16x2(a, b); }
__device__ __forceinline__ uint32_t pack2(__nv_bfloat16, float a, float b) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}

// The 16 bytes from byte sh (even, below 16) of the words a and b on.
__device__ __forceinline__ uint4 shifted(uint4 a, uint4 b, int sh) {
  uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
  if (sh & 8)
#pragma unroll
    for (int q = 0; q < 6; ++q) w[q] = w[q + 2];
  if (sh & 4)
#pragma unroll
    for (int q = 0; q < 5; ++q) w[q] = w[q + 1];
  const int bits = 8 * (sh & 3);
  return {__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
          __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits)};
}

// go(T{}) for the element type of a boute_dtype.
template <class Go>
inline int with_dtype(int dtype, Go go) {
  switch (dtype) {
    case BOUTE_F32: return go(float{});
    case BOUTE_F16: return go(__half{});
    case BOUTE_BF16: return go(__nv_bfloat16{});
  }
  return BOUTE_ERR_INVALID_ARG;
}

inline size_t dtype_bytes(int dtype) { return dtype == BOUTE_F32 ? 4 : 2; }
inline bool dtype_known(int dtype) {
  return dtype == BOUTE_F32 || dtype == BOUTE_F16 || dtype == BOUTE_BF16;
}
// A device array that the call needs: there, and aligned to its elements.
inline bool array_ok(const void *p, size_t bytes) {
  return p != nullptr && (uintptr_t)p % bytes == 0;
}
inline bool optional_ok(const void *p, size_t bytes) { return p == nullptr || array_ok(p, bytes); }

constexpr unsigned kAll = 0xffffffffu;
constexpr float kLog2e = 1.4426950408889634f;
// Gradients take ln s and the largest logit from the row itself where |lse| is beyond this.
constexpr float kLargeLse = 1024.f;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
// The warp's maximum in one instruction; a NaN anywhere wins.
__device__ __forceinline__ float warp_max_nan(float v) {
  float r;
  asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b, float c) {
  float r;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}
__device__ __forceinline__ float exp2_fast(float y) {  // (2 ulp; what is below 2^-126 is 0)
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}
__device__ __forceinline__ float exp2_gradual(float y) {  // (2 ulp; down to 2^-149)
  float r;
  asm("ex2.approx.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}
// Order-preserving bits of a float, and back.
__device__ __forceinline__ unsigned order_bits(float v) {
  const unsigned u = __float_as_uint(v);
  return u ^ ((unsigned)((int)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_order_bits(unsigned o) {
  return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

// ---- clusters (a block launched alone is a cluster of one) ---------------------------
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::
                   : "memory");
}
// A block's shared memory may be written by others once it runs. Every thread arrives at
// cluster_begin (at the kernel's start, before its loads) and waits at cluster_runs before the
// first store to a peer; by then the others have long begun.
__device__ __forceinline__ void cluster_begin() {
  asm volatile("barrier.cluster.arrive.relaxed.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_runs() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of block r's copy of a shared variable.
__device__ __forceinline__ uint32_t peer(const void *p, int r) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(r));
  return a;
}
__device__ __forceinline__ void store_peer(uint32_t a, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory");
}
__device__ __forceinline__ void store_peer(uint32_t a, unsigned long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}
__device__ __forceinline__ int add_peer(uint32_t a, int v) {
  int old;
  asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;"
               : "=r"(old)
               : "r"(a), "r"(v)
               : "memory");
  return old;
}

// Launches blocks of `threads` in clusters of `cluster` (1: none). As with launch_pdl, the kernel
// may be set up while the previous one on the stream ends, and begins with pdl_wait.
template <class... KArgs, class... Args>
inline int launch_cluster(void (*kernel)(KArgs...), long long blocks, int threads, int cluster,
                          size_t smem, cudaStream_t s, Args &&...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)blocks);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = cluster;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = cluster > 1 ? 2 : 1;
  cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
  count_launch();
  return last_launch_status();
}

}  // namespace boute
