// What the library asks of a device on every call, asked of the runtime once. (A header of its own,
// on the runtime's three calls alone, so that it can be built on fakes of them.)
#pragma once

#include <atomic>

#include "boute.h"

namespace boute {

struct DeviceInfo {
  int ok;   // BOUTE_OK for sm_103a
  int sms;  // multiprocessors
};
constexpr int kKnownDevices = 64;

// Of the current device. The kernels are built for sm_103a only: other devices are refused up front,
// and a device that cannot be asked is, until it can (a failed query leaves no error behind for
// later calls to report, and nothing in `known`). known: 0, or sms * 2 + (ok: 1); a device's answer
// does not change, and asking took 0.7 us a call.
inline DeviceInfo ask_device(std::atomic<int> *known) {
  int dev = 0, major = 0, minor = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) {
    cudaGetLastError();
    return {BOUTE_ERR_UNSUPPORTED, 152};
  }
  int v = dev < kKnownDevices ? known[dev].load(std::memory_order_relaxed) : 0;
  if (v == 0) {
    if (cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&minor, cudaDevAttrComputeCapabilityMinor, dev) != cudaSuccess ||
        cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
      cudaGetLastError();
      return {BOUTE_ERR_UNSUPPORTED, 152};
    }
    v = sms * 2 + (major == 10 && minor == 3);
    if (dev < kKnownDevices) known[dev].store(v, std::memory_order_relaxed);
  }
  return {v & 1 ? BOUTE_OK : BOUTE_ERR_UNSUPPORTED, v / 2};
}

}  // namespace boute
