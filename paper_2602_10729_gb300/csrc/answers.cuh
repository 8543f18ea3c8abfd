// What the kernels over a model's answers share: the logits' element types,
// and the checks of their C entry points.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>

#include "internal.h"
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

}  // namespace boute
