// The dynamic shared memory that kernels may have. (A header of its own, on the runtime's two calls
// alone, so that it can be built on fakes of them.)
#pragma once

#include <cstddef>
#include <map>
#include <mutex>
#include <utility>

namespace boute {

// Lets a kernel have `bytes` on the current device. The limit is the process's: set to each call's
// own size, it would be lowered under another thread's launch of more, which is then refused. So it
// is set to the most that any call has asked for, under a lock; each time, as a reset of the device
// takes it back; whatever the size, as static arrays count against the 48 KB that kernels have
// unasked.
inline cudaError_t raise_smem(const void *kernel, size_t bytes) try {
  static std::mutex lock;
  static std::map<std::pair<const void *, int>, size_t> limits;
  int dev = 0;
  if (cudaError_t e = cudaGetDevice(&dev)) return e;
  const std::lock_guard<std::mutex> guard(lock);
  size_t &limit = limits[{kernel, dev}];
  const size_t most = bytes > limit ? bytes : limit;
  const cudaError_t e =
      cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
  if (e == cudaSuccess) limit = most;
  return e;
} catch (...) {  // (no memory for the table, or no lock: the callers are C entry points)
  return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
}
template <class... Args>
inline cudaError_t raise_smem(void (*kernel)(Args...), size_t bytes) {
  return raise_smem((const void *)kernel, bytes);
}

}  // namespace boute
