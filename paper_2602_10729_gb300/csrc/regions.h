// Whether arrays of rows share memory. (A header of its own, on the standard library alone, so that
// it can be built without a device.)
#pragma once

#include <cstddef>
#include <cstdint>
#include <initializer_list>
#include <numeric>

namespace boute {

// `rows` rows of `bytes` bytes, `pitch` bytes from one to the next.
struct Region {
  const void *p;
  long long rows;
  unsigned long long bytes, pitch;
};
inline Region array_of(const void *p, long long n, size_t size) {
  return {p, p && n > 0 ? 1 : 0, (unsigned long long)n * size, 0};
}
inline Region rows_of(const void *p, long long rows, long long n, long long ld, size_t size) {
  return {p, p ? rows : 0, (unsigned long long)n * size, (unsigned long long)ld * size};
}

// Exact for arrays, for rows of one pitch and for a single row beside them: what lies between the
// other's rows shares nothing. Of two pitches, whatever their greatest common divisor cannot tell
// apart counts as shared.
inline bool overlap(const Region &a, const Region &b) {
  using Wide = unsigned __int128;
  if (a.rows <= 0 || b.rows <= 0) return false;
  const Wide a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
  const Wide a1 = a0 + (Wide)(a.rows - 1) * a.pitch + a.bytes;
  const Wide b1 = b0 + (Wide)(b.rows - 1) * b.pitch + b.bytes;
  if (a1 <= b0 || b1 <= a0) return false;
  const unsigned long long pa = a.rows > 1 ? a.pitch : 0, pb = b.rows > 1 ? b.pitch : 0;
  const unsigned long long g = std::gcd(pa, pb);  // (of 0 and another: the other)
  if (g == 0) return true;
  const unsigned long long at = (uintptr_t)a.p % g, bt = (uintptr_t)b.p % g;
  const unsigned long long d = bt >= at ? bt - at : bt + (g - at);  // from a row of a to one of b
  return d < a.bytes || g - d < b.bytes;
}
// Whether an output shares memory with an input or with another output.
inline bool outputs_overlap(std::initializer_list<Region> outs, std::initializer_list<Region> ins) {
  for (auto o = outs.begin(); o != outs.end(); ++o) {
    for (const Region &i : ins)
      if (overlap(*o, i)) return true;
    for (auto q = o + 1; q != outs.end(); ++q)
      if (overlap(*o, *q)) return true;
  }
  return false;
}

}  // namespace boute
