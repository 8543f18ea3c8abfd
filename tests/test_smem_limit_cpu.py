"""The limit of a kernel's shared memory, on fakes of the runtime's calls: it is the process's, so that a
call raises it and none lowers it."""
import os
import subprocess

from paper_2602_10729_gb300 import build as bld

HOST = r"""
#include <atomic>
#include <cstdio>
#include <cstdlib>
#include <new>
#include <map>
#include <thread>
enum cudaError_t { cudaSuccess, cudaFailed };
enum { cudaFuncAttributeMaxDynamicSharedMemorySize };
static thread_local int device = 0;
static std::atomic<int> failing{0};
static std::atomic<int> limit[2][2];
static int kernels[2];
static cudaError_t cudaGetDevice(int *d) { *d = device; return device < 0 ? cudaFailed : cudaSuccess; }
static cudaError_t cudaFuncSetAttribute(const void *k, int, int bytes) {
  if (failing) return cudaFailed;
  limit[device][(const int *)k - kernels] = bytes;
  return cudaSuccess;
}
static std::atomic<int> no_memory{0};
void *operator new(size_t n) {
  if (no_memory) throw std::bad_alloc();
  return std::malloc(n);
}
void operator delete(void *p) noexcept { std::free(p); }
void operator delete(void *p, size_t) noexcept { std::free(p); }
#include "smem_limit.h"
using namespace boute;
int main() {
  int bad = 0;
  auto want = [&](bool ok, const char *what) { if (!ok) ++bad, std::printf("%s\n", what); };
  const void *a = &kernels[0], *b = &kernels[1];
  no_memory = 1;
  want(raise_smem(a, 4000) == cudaSuccess && limit[0][0] == 4000, "no memory for the table: set all the same");
  no_memory = 0;
  failing = 1;
  want(raise_smem(a, 5000) == cudaFailed, "a failure is told");
  failing = 0;
  want(raise_smem(a, 5000) == cudaSuccess && limit[0][0] == 5000, "and not remembered");
  raise_smem(a, 3000);
  want(limit[0][0] == 5000, "never lowered");
  limit[0][0] = 0;
  raise_smem(a, 3000);
  want(limit[0][0] == 5000, "set again after a reset of the device");
  raise_smem(a, 7000);
  want(limit[0][0] == 7000 && limit[0][1] == 0, "raised, of this kernel");
  raise_smem(b, 100);
  device = 1;
  raise_smem(a, 200);
  want(limit[0][1] == 100 && limit[1][0] == 200 && limit[0][0] == 7000, "by kernel and device");
  device = -1;
  want(raise_smem(a, 9000) == cudaFailed, "no device");
  device = 0;
  std::thread threads[8];
  std::atomic<int> short_of{0};
  for (int t = 0; t < 8; ++t)
    threads[t] = std::thread([&, t] {
      for (int i = 0; i < 20000; ++i) {
        const int need = 8000 + (i * (t + 1)) % 9000;
        raise_smem(a, need);
        if (limit[0][0] < need) ++short_of;
      }
    });
  for (auto &t : threads) t.join();
  want(short_of == 0, "a launch finds what it asked for, whatever other threads ask");
  return bad;
}
"""


def test_limits_are_raised_and_never_lowered(tmp_path):
    src, exe = tmp_path / "limit.cc", tmp_path / "limit"
    src.write_text(HOST)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-pthread", "-I", bld.CSRC, str(src), "-o", str(exe)],
                   check=True)
    p = subprocess.run([str(exe)], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout
