"""What the library remembers of a device, on fakes of the runtime's calls: a query that fails once
does not make the device unsupported for good."""
import os
import subprocess

from paper_2602_10729_gb300 import build as bld

HOST = r"""
#include <cstdio>
enum { cudaSuccess, cudaFailed };
enum { cudaDevAttrComputeCapabilityMajor, cudaDevAttrComputeCapabilityMinor,
       cudaDevAttrMultiProcessorCount };
static int device = 0, asked = 0, fail_at = -1, errors = 0, no_device = 0;
static int cudaGetLastError() { const int e = errors; errors = 0; return e; }
static int cudaGetDevice(int *d) {
  *d = device;
  return no_device ? (errors = cudaFailed) : cudaSuccess;
}
static int cudaDeviceGetAttribute(int *v, int what, int dev) {
  if (asked++ == fail_at) return errors = cudaFailed;
  const int of[2][3] = {{10, 3, 152}, {9, 0, 132}};
  *v = of[dev == 1][what];
  return cudaSuccess;
}
#include "device_info.h"
using namespace boute;
static std::atomic<int> known[kKnownDevices];
static int bad = 0;
static void want(int ok, int sms, int calls, const char *what) {
  asked = 0;
  const DeviceInfo i = ask_device(known);
  if (i.ok != ok || i.sms != sms || asked != calls || errors) {
    ++bad;
    std::printf("%s: ok %d sms %d calls %d errors %d\n", what, i.ok, i.sms, asked, errors);
  }
}
int main() {
  for (fail_at = 0; fail_at < 3; ++fail_at)
    want(BOUTE_ERR_UNSUPPORTED, 152, fail_at + 1, "a query fails");
  fail_at = -1;
  no_device = 1;
  want(BOUTE_ERR_UNSUPPORTED, 152, 0, "no device");
  no_device = 0;
  want(BOUTE_OK, 152, 3, "after the failures");
  want(BOUTE_OK, 152, 0, "known");
  device = 1;
  want(BOUTE_ERR_UNSUPPORTED, 132, 3, "another device");
  want(BOUTE_ERR_UNSUPPORTED, 132, 0, "another device, known");
  device = kKnownDevices;
  want(BOUTE_OK, 152, 3, "beyond the table");
  want(BOUTE_OK, 152, 3, "beyond the table again");
  return bad;
}
"""


def test_a_failed_query_is_not_remembered(tmp_path):
    src, exe = tmp_path / "ask.cc", tmp_path / "ask"
    src.write_text(HOST)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-I", bld.CSRC,
                    "-I", os.path.join(bld.ROOT, "include"), str(src), "-o", str(exe)], check=True)
    p = subprocess.run([str(exe)], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout
