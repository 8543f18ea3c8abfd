"""Arrays that share memory: the rule against every byte counted, and the calls over experts' rows and
hidden states that refuse outputs in their inputs, in other outputs or in the workspace."""
import ctypes
import os
import subprocess

import pytest

from paper_2602_10729_gb300 import build as bld
from test_abi_answers_cpu import BAD, UNS, call, lib  # noqa: F401

HOST = r"""
#include <cstdio>
#include <set>
#include "regions.h"
using namespace boute;
static unsigned long long state = 1;
static unsigned draw(unsigned n) {
  state = state * 6364136223846793005ull + 1442695040888963407ull;
  return (unsigned)(state >> 33) % n;
}
static std::set<unsigned long long> bytes_of(const Region &r) {
  std::set<unsigned long long> s;
  for (long long i = 0; i < r.rows; ++i)
    for (unsigned long long b = 0; b < r.bytes; ++b) s.insert((uintptr_t)r.p + i * r.pitch + b);
  return s;
}
int main() {
  int shared = 0, apart = 0, bad = 0;
  for (int n = 0; n < 200000; ++n) {
    Region r[2];
    const unsigned pitch = 1 + draw(12);
    for (Region &x : r) {
      const unsigned p = draw(4) ? pitch : 1 + draw(24);
      x = {(const void *)(uintptr_t)(1000 + draw(60)), (long long)draw(5), 1 + draw(p), p};
      if (x.rows == 1) x.pitch = draw(2) ? ~0ull >> 8 : 0;
    }
    bool want = false;
    const auto a = bytes_of(r[0]);
    for (unsigned long long b : bytes_of(r[1])) want |= a.count(b) > 0;
    const bool got = overlap(r[0], r[1]), exact = r[0].rows <= 1 || r[1].rows <= 1 || r[0].pitch == r[1].pitch;
    shared += want, apart += !want;
    if (got != overlap(r[1], r[0]) || (want && !got) || (exact && want != got)) ++bad;
  }
  const Region far = {(const void *)16, 1ll << 31, 1ull << 40, 1ull << 62};
  const Region end = {(const void *)(~(uintptr_t)0 - 15), 1, 16, 0};
  if (!overlap(far, far) || !overlap(far, array_of((void *)32, 4, 4)) || overlap(end, array_of((void *)32, 4, 4)))
    ++bad;
  if (overlap(array_of(nullptr, 4, 4), far) || overlap(array_of((void *)32, 0, 4), far)) ++bad;
  std::printf("%d shared %d apart %d bad\n", shared, apart, bad);
  return bad || shared < 1000 || apart < 1000;
}
"""


def test_rule_against_every_byte(tmp_path):
    src, exe = tmp_path / "regions.cc", tmp_path / "regions"
    src.write_text(HOST)
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-I", bld.CSRC, str(src), "-o", str(exe)],
                   check=True)
    p = subprocess.run([str(exe)], capture_output=True, text=True)
    assert p.returncode == 0, p.stdout


def at(mb, byte=0):
    return ctypes.c_void_p((mb << 20) + byte)


def refused_where(f, good, outs, ins, sizes):
    """`good` has arrays a megabyte apart (and is not called: the addresses are nobody's); each output
    moved into each other array, to its first bytes and to its last ones, is refused."""
    for o in outs:
        for other in [n for n in ins + outs if n != o]:
            base = good[other].value
            for byte in {0, (sizes[other] - 1) // 64 * 64}:
                assert call(f, good, **{o: ctypes.c_void_p(base + byte)}) == BAD, (o, other, byte)
            # its own last bytes at the other's first
            back = (sizes[o] - 1) // 64 * 64
            assert call(f, good, **{o: ctypes.c_void_p(base - back)}) == BAD, (o, other)


def test_sort(lib):  # noqa: F811
    good = dict(idx=at(1), T=400, k=2, E=99, off=at(2), src=at(3), place=at(4), s=None)
    refused_where(lib.boute_expert_sort, good, ["off", "src", "place"], ["idx"],
                  dict(idx=3200, off=400, src=3200, place=3200))


def test_rows(lib):  # noqa: F811
    size = dict(x=40 * 128, rows=80 * 128, place=320, w=320, g=80 * 128, gw=320)
    good = dict(x=at(1), dtype=0, T=40, D=32, ldx=32, place=at(2), k=2, rows=at(3), R=80, ldr=32, s=None)
    refused_where(lib.boute_expert_dispatch, good, ["rows"], ["x", "place"], size)
    good = dict(rows=at(1), dtype=0, R=80, D=32, ldr=32, place=at(2), T=40, k=2, x=at(3), ldx=32, s=None)
    refused_where(lib.boute_expert_dispatch_grad, good, ["x"], ["rows", "place"], size)
    good = dict(rows=at(1), dtype=0, R=80, D=32, ldr=32, place=at(2), w=at(4), T=40, k=2, x=at(3), ldx=32,
                s=None)
    refused_where(lib.boute_expert_combine, good, ["x"], ["rows", "place", "w"], size)
    good = dict(x=at(1), dtype=0, T=40, D=32, ldx=32, rows=at(2), R=80, ldr=32, place=at(3), w=at(4), k=2,
                g=at(5), ldg=32, gw=at(6), s=None)
    f = lib.boute_expert_combine_grad
    refused_where(f, good, ["gw"], ["x", "rows", "place", "w"], size)
    refused_where(f, good, ["g"], ["x", "place", "w"], size)
    assert call(f, good, g=at(2, 64)) == BAD and call(f, good, g=at(2), ldg=33) == BAD


def test_hidden(lib):  # noqa: F811
    vec = {n: 400 for n in ("lp", "H", "lse", "g", "gh")}
    size = dict(vec, h=100 * 128, w=300 * 128, t=800, ws=4096, dh=100 * 128, dw=300 * 128)
    good = dict(h=at(1), dt=2, T=100, D=64, ldh=64, w=at(2), V=300, ldw=64, t=at(3), scale=1.0, lp=at(4),
                H=at(5), lse=at(6), ws=at(64), n=1 << 30, s=None)
    f = lib.boute_hidden_logprobs
    refused_where(f, good, ["lp", "H", "lse"], ["h", "w", "t", "ws"], size)
    for n in ("h", "w", "t"):
        assert call(f, good, **{n: good["ws"]}) == BAD, n
    good = dict(h=at(1), dt=2, T=100, D=64, ldh=64, w=at(2), V=300, ldw=64, t=at(3), scale=1.0, lse=at(4),
                H=at(5), g=at(6), gh=at(7), dh=at(8), lddh=64, dw=at(9), lddw=64, ws=at(64), n=1 << 30,
                s=None)
    f = lib.boute_hidden_logprobs_grad
    refused_where(f, good, ["dh", "dw"], ["h", "w", "t", "lse", "H", "g", "gh", "ws"], size)
    for n in ("h", "w", "t", "lse", "H", "g", "gh"):
        assert call(f, good, **{n: good["ws"]}) == BAD, n


@pytest.mark.parametrize("name,good", [
    ("boute_expert_sort", dict(idx=at(1), T=1 << 30, k=4, E=9, off=at(1), src=at(1), place=at(1), s=None)),
    ("boute_expert_dispatch", dict(x=at(1), dtype=0, T=4, D=10, ldx=10, place=at(1), k=99, rows=at(1), R=8,
                                   ldr=12, s=None))])
def test_limits_come_first(lib, name, good):  # noqa: F811
    assert call(getattr(lib, name), good) == UNS
