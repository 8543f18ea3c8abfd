// Routing of queries to experts: scores, the choice within the best groups,
// the weights and the load; and the gradient of the weights.
//
// Instructions bound it, and the wait for each round's logits: a query's are one or two lines,
// its choice some hundred instructions. So as little as possible is compared:
//  - Teams of 8 lanes to a query, four queries to a warp, take up to 8 of up to 256 experts.
//    Each lane's values are parts, 4 K in all, whose maxima's K-th largest is a bound that K
//    values reach, and few others; those alone become keys (order bits over the expert's
//    complement, so that equal values go to the lowest index) and are ranked. 16-bit logits
//    that are compared as they are (no bias, no groups) stay as pairs, two to an instruction;
//    where they are few to a lane, all of them become keys, whole in 32 bits, of which each
//    lane sorts its K largest and the lanes' lists join two by two.
//  - A warp to a query for more choices, more experts, and too few queries to fill the SMs:
//    each lane sorts its own, and k rounds take the largest of the 32 heads.
// Without a bias the logits themselves are compared, which have the order of the scores:
// only the chosen scores are computed then, and a softmax's sum only where the weights are
// not renormalised. 262144 queries of 256 bf16 logits, k = 4: 35.5 us (4.0 TB/s; a floor of
// 21), k = 1: 35.3; 131072 of 256, logistic with bias, k = 4: 37.6, in 8 groups with k = 8: 61.
// The gradient moves bytes: 131072 queries of 160 fp32, k = 6: 26.4 us where they take 25.7; a
// softmax's 29.8 renormalised and 45.8 without.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;

// A score may be as small as fp32 holds, 2^-149; below it is 0. Scores are made with approximate
// instructions (exponential 2 ulp, reciprocal 1), as there are some hundred to a query.
constexpr float kLeastLog2 = -149.f;
// Scores that a sum of small ones is made of are taken relative to the largest of them where fewer
// bits of them are left than fp32 has; beside a sum of 1/8 what is below 2^-126 is below 2^-123.
constexpr float kFewBits = 0x1p-100f, kSmallSum = 0.125f;

__device__ __forceinline__ float logistic(float x) {  // (0 below 2^-126)
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + exp2_fast(-x * kLog2e)));
  return r;
}
// Over teams of lanes (a power of two).
template <int L>
__device__ __forceinline__ float team_sum(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
// Whether a ballot has a bit of this lane's team.
template <int L>
__device__ __forceinline__ bool of_team(unsigned ballot) {
  return (ballot >> (threadIdx.x & 31) / L * L & (unsigned)((1ull << L) - 1)) != 0u;
}
template <int L>
__device__ __forceinline__ float team_max(float v) {
#pragma unroll
  for (int o = L / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
__device__ __forceinline__ float team_max(float v, int team) {
  for (int o = team / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
__device__ __forceinline__ float team_sum(float v, int team) {
  for (int o = team / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

// ---- choosing --------------------------------------------------------------------------
struct RouteArgs {
  const void *logits;
  long long rows, ld;
  const float *bias;
  int dtype, E, mode, G, keep, group_top, k, renorm;
  int by_logits;  // the logits are compared
  int vec;        // rows on 16-byte boundaries, E a multiple of a vector's logits
  int own;  // experts of a lane (route_bound_kernel)
  int group_lanes; // lanes that hold a group, where each holds experts of one; else 0
  float factor;
  int *idx, *load;
  float *weight;
};

__device__ __forceinline__ float logit_at(const RouteArgs &A, long long row, int e) {
  if (!BOUTE_INB(e, A.E) || !BOUTE_INB(row, A.rows)) return -INFINITY;
  const long long i = row * A.ld + e;
  if (A.dtype == BOUTE_F32) return ((const float *)A.logits)[i];
  if (A.dtype == BOUTE_F16) return __half2float(((const __half *)A.logits)[i]);
  return __bfloat162float(((const __nv_bfloat16 *)A.logits)[i]);
}
// N words of 4-byte (PER = 1) or pairs of 2-byte logits from e0 on, by vectors of up to 16 bytes
// where rows allow (`vec`); `none` from `end` on, of a row of E.
template <int N, int PER>
__device__ __forceinline__ void load_words(uint32_t *w, const void *row, int e0, int end, int E,
                                           bool vec, uint32_t none) {
  static_assert(N == 1 || N == 2 || N % 4 == 0, "whole vectors");
  if (vec && N == 1) {
    w[0] = e0 < end && BOUTE_INB(e0 + PER - 1, E) ? *((const uint32_t *)row + e0 / PER) : none;
  } else if (vec && N == 2) {
    uint2 v = {none, none};
    if (e0 < end && BOUTE_INB(e0 + 2 * PER - 1, E))
      v = *(const uint2 *)((const uint32_t *)row + e0 / PER);
    w[0] = v.x, w[N - 1] = v.y;
  } else if (vec) {
#pragma unroll
    for (int i = 0; i < N / 4; ++i) {
      uint4 v = {none, none, none, none};
      if (e0 + 4 * PER * i < end && BOUTE_INB(e0 + 4 * PER * (i + 1) - 1, E))
        v = *(const uint4 *)((const uint32_t *)row + e0 / PER + 4 * i);
      w[4 * i] = v.x, w[4 * i + 1] = v.y, w[4 * i + 2] = v.z, w[4 * i + 3] = v.w;
    }
  } else if constexpr (PER == 1) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      w[i] = e0 + i < end && BOUTE_INB(e0 + i, E) ? ((const uint32_t *)row)[e0 + i] : none;
  } else {
    const unsigned short *h = (const unsigned short *)row;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = e0 + 2 * i;
      w[i] = (e < end && BOUTE_INB(e, E) ? (uint32_t)h[e] : none & 0xffffu) |
             (e + 1 < end && BOUTE_INB(e + 1, E) ? (uint32_t)h[e + 1] << 16 : none & 0xffff0000u);
    }
  }
}
// Pairs of 16-bit logits: f16 or bf16 by HALF.
template <bool HALF>
struct Pair {
  uint32_t w;
  static constexpr unsigned kInf = HALF ? 0x7c00u : 0x7f80u;
  __device__ __forceinline__ Pair swapped() const { return {__byte_perm(w, 0u, 0x1032)}; }
  // with -0 as +0 (and NaNs as one)
  __device__ __forceinline__ Pair plus_zero() const {
    Pair r;
    if (HALF) asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r.w) : "r"(w), "r"(0u));
    else asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r.w) : "r"(w), "r"(0u));
    return r;
  }
  // 0xffff where it is at least o
  __device__ __forceinline__ uint32_t reaches(Pair o) const {
    uint32_t r;
    if (HALF) {
      __half2 a, b;
      memcpy(&a, &w, 4);
      memcpy(&b, &o.w, 4);
      r = __hge2_mask(a, b);
    } else {
      __nv_bfloat162 a, b;
      memcpy(&a, &w, 4);
      memcpy(&b, &o.w, 4);
      r = __hge2_mask(a, b);
    }
    return r;
  }
  static __device__ __forceinline__ float value(unsigned u) {
    return HALF ? __half2float(__ushort_as_half((unsigned short)u)) : __uint_as_float(u << 16);
  }
};
using ::max;
using ::min;
// (a NaN wins in max, and is left behind by min)
template <bool HALF>
__device__ __forceinline__ Pair<HALF> max(Pair<HALF> a, Pair<HALF> b) {
  Pair<HALF> r;
  if (HALF) asm("max.NaN.f16x2 %0, %1, %2;" : "=r"(r.w) : "r"(a.w), "r"(b.w));
  else asm("max.NaN.bf16x2 %0, %1, %2;" : "=r"(r.w) : "r"(a.w), "r"(b.w));
  return r;
}
template <bool HALF>
__device__ __forceinline__ Pair<HALF> min(Pair<HALF> a, Pair<HALF> b) {
  Pair<HALF> r;
  if (HALF) asm("min.f16x2 %0, %1, %2;" : "=r"(r.w) : "r"(a.w), "r"(b.w));
  else asm("min.bf16x2 %0, %1, %2;" : "=r"(r.w) : "r"(a.w), "r"(b.w));
  return r;
}

// L values in descending order (Batcher's odd-even merge sort).
template <int L, class V>
__device__ __forceinline__ void sort_desc(V *v) {
#pragma unroll
  for (int p = 1; p < L; p *= 2)
#pragma unroll
    for (int q = p; q > 0; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < L; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (i + j + q < L && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
            const V a = v[i + j], b = v[i + j + q];
            v[i + j] = max(a, b);
            v[i + j + q] = min(a, b);
          }
}
// v: a bitonic run of L, into descending order.
template <int L, class V>
__device__ __forceinline__ void merge_desc(V *v) {
#pragma unroll
  for (int q = L / 2; q > 0; q /= 2)
#pragma unroll
    for (int i = 0; i < L; ++i)
      if (!(i & q)) {
        const V a = v[i], b = v[i + q];
        v[i] = max(a, b);
        v[i + q] = min(a, b);
      }
}
// The K largest of a lane's S values in descending order, in c[0 .. K): runs of K are sorted, then
// joined two by two (the larger of each and the other's reverse form a bitonic run).
template <int S, int K, class V>
__device__ __forceinline__ void best_in_lane(V (&c)[S]) {
#pragma unroll
  for (int s = 0; s < S; s += K) sort_desc<K>(c + s);
#pragma unroll
  for (int o = K; o < S; o *= 2)
#pragma unroll
    for (int s = 0; s < S; s += 2 * o) {
#pragma unroll
      for (int i = 0; i < K; ++i) c[s + i] = max(c[s + i], c[s + o + K - 1 - i]);
      merge_desc<K>(c + s);
    }
}
template <bool HALF>
__device__ __forceinline__ Pair<HALF> other_lane(Pair<HALF> v, int o) {
  return {__shfl_xor_sync(kAll, v.w, o)};
}
template <class V>
__device__ __forceinline__ V other_lane(V v, int o) {
  return __shfl_xor_sync(kAll, v, o);
}
// The K largest in order of 8 lanes' lists of FROM in order, in every lane.
template <int FROM, int K, class V>
__device__ __forceinline__ void join_lanes(V (&a)[K]) {
  V other[K];
#pragma unroll
  for (int o = 1, n = FROM; o < 8; o *= 2) {
#pragma unroll
    for (int i = 0; i < n; ++i) other[i] = other_lane(a[n - 1 - i], o);
    if (n < K) {
#pragma unroll
      for (int i = 0; i < n; ++i) a[n + i] = other[i];
      n *= 2;
      if (n == 2) merge_desc<2>(a);
      if (n == 4) merge_desc<4>(a);
      if (n == 8) merge_desc<8>(a);
    } else {
#pragma unroll
      for (int i = 0; i < K; ++i) a[i] = max(a[i], other[i]);
      merge_desc<K>(a);
    }
  }
}
// The K <= S largest of the team's keys, S in each of its 8 lanes, in every lane.
template <int S, int K>
__device__ __forceinline__ void best_of(unsigned (&c)[S], unsigned (&best)[K]) {
  best_in_lane<S, K>(c);
#pragma unroll
  for (int i = 0; i < K; ++i) best[i] = c[i];
  join_lanes<K>(best);
}
// A value that K of the team's values reach, N in each of its 8 lanes, and few others: the K-th
// largest of 4 K parts' maxima, K / 2 parts to a lane.
template <int K, int N>
__device__ __forceinline__ float bound_of(const float (&v)[N]) {
  constexpr int kOf = K / 2;
  float a[K];
#pragma unroll
  for (int i = 0; i < kOf; ++i) {
    a[i] = v[i];
#pragma unroll
    for (int s = i + kOf; s < N; s += kOf) a[i] = fmaxf(a[i], v[s]);
  }
  sort_desc<kOf>(a);
  join_lanes<kOf>(a);
  return a[K - 1];
}
// The same of pairs, two lists of halves at once; the bound and the largest value in both halves.
template <int K, int N, bool HALF>
__device__ __forceinline__ Pair<HALF> bound_of(const Pair<HALF> (&w)[N], Pair<HALF> &top) {
  constexpr int kOf = K / 4;
  Pair<HALF> a[K];
#pragma unroll
  for (int i = 0; i < kOf; ++i) {
    a[i] = w[i];
#pragma unroll
    for (int s = i + kOf; s < N; s += kOf) a[i] = max(a[i], w[s]);
  }
  sort_desc<kOf>(a);
  join_lanes<kOf>(a);
  top = max(a[0], a[0].swapped());
  Pair<HALF> bound = max(a[0], a[K - 1].swapped());
#pragma unroll
  for (int i = 1; i < K; ++i) bound = min(bound, max(a[i], a[K - 1 - i].swapped()));
  return bound;
}
// Of the hits of the team's 8 lanes, how many precede lane l's (which has `mine`), and all of them.
__device__ __forceinline__ int hits_before(int mine, int l, int &all) {
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 8; o *= 2) {
    const int v = __shfl_up_sync(kAll, upto, o, 8);
    upto += l >= o ? v : 0;
  }
  all = __shfl_sync(kAll, upto, 7, 8);
  return upto - mine;
}

// The two largest of two pairs a >= b.
__device__ __forceinline__ void join_two(float &a, float &b, float a2, float b2) {
  b = fmaxf(fminf(a, a2), fmaxf(b, b2));
  a = fmaxf(a, a2);
}
// Whether the lane's experts, all of them of one group, are in one that stays; lane l of the team's
// L. (A group's lanes join theirs in its first, in any number of lanes.)
template <int S, int L>
__device__ __forceinline__ bool keeps_lane(const float (&c)[S], const RouteArgs &A, int l) {
  const int n = A.group_lanes, g = l / n, i = l - g * n;
  float a = c[0], b = -INFINITY;
#pragma unroll
  for (int s = 1; s < S; ++s) {
    b = fmaxf(b, fminf(a, c[s]));
    a = fmaxf(a, c[s]);
  }
  for (int o = L / 2; o > 0; o >>= 1) {
    if (o >= n) continue;
    const float a2 = __shfl_down_sync(kAll, a, o, L), b2 = __shfl_down_sync(kAll, b, o, L);
    if (i < o && i + o < n) join_two(a, b, a2, b2);
  }
  const float score = A.group_top == 2 && b > -INFINITY ? a + b : a;
  const float mine = __shfl_sync(kAll, score, l - i, L);
  int rank = 0;
  for (int h = 0; h < A.G; ++h) {
    const float other = __shfl_sync(kAll, score, h * n, L);
    rank += other > mine || (other == mine && h < g);
  }
  return rank < A.keep && mine > -INFINITY;
}
// Bits of the groups that stay, from a query's c in shared memory; lane l of the team's L. Several
// lanes to a group where there are enough, else groups in turn.
template <int L>
__device__ __forceinline__ unsigned keep_groups(const float *c, float *scores, const RouteArgs &A,
                                                int per, int l) {
  int width = 1;
  while (2 * width * A.G <= L) width *= 2;
  for (int g0 = 0; g0 < A.G; g0 += L / width) {
    const int g = g0 + l / width;
    float a = -INFINITY, b = -INFINITY;
    if (g < A.G)
#pragma unroll 4
      for (int i = l % width; i < per; i += width)
        if (BOUTE_INB(g * per + i, A.E)) join_two(a, b, c[g * per + i], -INFINITY);
    for (int o = 1; o < width; o *= 2)
      join_two(a, b, __shfl_xor_sync(kAll, a, o), __shfl_xor_sync(kAll, b, o));
    if (g < A.G && l % width == 0) scores[g] = A.group_top == 2 && b > -INFINITY ? a + b : a;
  }
  __syncwarp();
  unsigned kept = 0u;
  for (int g = l; g < A.G; g += L) {
    const float mine = scores[g];
    int rank = 0;
    for (int h = 0; h < A.G; ++h) rank += scores[h] > mine || (scores[h] == mine && h < g);
    kept |= rank < A.keep && mine > -INFINITY ? 1u << g : 0u;
  }
#pragma unroll
  for (int o = 1; o < L; o *= 2) kept |= __shfl_xor_sync(kAll, kept, o);
  return kept;
}
// -inf for the lane's S experts from e0 on that are in no kept group.
template <int S>
__device__ __forceinline__ void drop_groups(float (&c)[S], unsigned kept, int e0, int per) {
  int g = e0 / per, left = (g + 1) * per - e0;  // (neighbours: one division, then steps)
#pragma unroll
  for (int s = 0; s < S; ++s) {
    if (left-- == 0) {
      ++g;
      left = per - 1;
    }
    if (!(kept >> (g & 31) & 1u)) c[s] = -INFINITY;
  }
}

// Floats of a query's c and groups' scores (teams' rows begin in different banks).
__host__ __device__ inline int shared_stride(int E) {
  return round_up(E + BOUTE_MAX_GROUPS, 32) + 2;
}

// -inf for the lane's experts [e0, end) in groups that do not stay; shared: a query's
// shared_stride(E) floats where lanes hold experts of several groups.
template <int S, int L>
__device__ __forceinline__ void apply_groups(const RouteArgs &A, float (&c)[S], float *shared,
                                             int e0, int end, int l) {
  if (A.keep == A.G) return;
  if (A.group_lanes) {
    const bool kept = keeps_lane<S, L>(c, A, l);
#pragma unroll
    for (int s = 0; s < S; ++s) c[s] = kept ? c[s] : -INFINITY;
    return;
  }
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (e0 + s < end && BOUTE_INB(e0 + s, A.E)) shared[e0 + s] = c[s];
  __syncwarp();
  const unsigned kept = keep_groups<L>(shared, shared + A.E, A, A.E / A.G, l);
  __syncwarp();
  drop_groups(c, kept, e0, A.E / A.G);
}

// What a query's choice among its experts is made of, for a team of L lanes.
struct Query {
  float m, inv_sum;  // of the softmax
  bool bad;          // no distribution
  // c of expert e with logit x: the same sums for every lane and in every place
  __device__ __forceinline__ float value(const RouteArgs &A, float x, int e) const {
    float v = x;
    if (!A.by_logits) {
      v = score(A, x);
      if (A.bias) v = __fadd_rn(v, fmaxf(A.bias[e], -INFINITY));  // (no NaN)
    }
    return x > -INFINITY && !bad ? v : -INFINITY;
  }
  __device__ __forceinline__ float score(const RouteArgs &A, float x) const {
    return A.mode == BOUTE_ROUTE_SOFTMAX ? exp2_fast((x - m) * kLog2e) * inv_sum : logistic(x);
  }
  // the same with all the bits that fp32 has for it, for a weight
  __device__ __forceinline__ float whole_score(const RouteArgs &A, float x) const {
    if (A.mode == BOUTE_ROUTE_SOFTMAX) return exp2_gradual((x - m) * kLog2e) * inv_sum;
    return x < -64.f ? exp2_gradual(x * kLog2e) : logistic(x);  // (1 + exp(x) is 1)
  }
  // a score over that of a logit `of` >= x, both below 1/8; 0 where the score is
  __device__ __forceinline__ float score_over(const RouteArgs &A, float x, float of) const {
    const bool soft = A.mode == BOUTE_ROUTE_SOFTMAX;
    const float least = soft ? (x - m) * kLog2e + __log2f(inv_sum) : x * kLog2e;
    if (!(least >= kLeastLog2)) return 0.f;
    const float e = exp2_fast((x - of) * kLog2e);
    return soft ? e : __fdividef(e, 1.f + exp2_fast(x * kLog2e));  // (but for 1 + exp(of))
  }
};
// c of the lane's S experts from e0 on (-inf: not to be chosen).
template <int S>
__device__ __forceinline__ void load_bias(const RouteArgs &A, int e0, float (&bias)[S]) {
#pragma unroll
  for (int s = 0; s < S; ++s)
    bias[s] = A.bias && e0 + s < A.E ? fmaxf(A.bias[e0 + s], -INFINITY) : 0.f;  // (no NaN)
}
// The lane's logits from e0 on, -inf from `end` on.
template <int S>
__device__ __forceinline__ void load_logits(const RouteArgs &A, long long row, int e0, int end,
                                            float (&c)[S]) {
  if (A.dtype == BOUTE_F32) {
    uint32_t w[S];
    load_words<S, 1>(w, (const float *)A.logits + row * A.ld, e0, end, A.E, A.vec, 0xff800000u);
#pragma unroll
    for (int s = 0; s < S; ++s) c[s] = __uint_as_float(w[s]);
  } else {
    uint32_t w[S / 2];
    load_words<S / 2, 2>(w, (const unsigned short *)A.logits + row * A.ld, e0, end, A.E, A.vec,
                         A.dtype == BOUTE_F16 ? 0xfc00fc00u : 0xff80ff80u);
#pragma unroll
    for (int i = 0; i < S / 2; ++i)
      if (A.dtype == BOUTE_F16) {
        unpack_f16x2(w[i], c[2 * i], c[2 * i + 1]);
      } else {
        c[2 * i] = __uint_as_float(w[i] << 16);
        c[2 * i + 1] = __uint_as_float(w[i] & 0xffff0000u);
      }
  }
}
// A query's statistics, and c of the lane's S logits in their place; bias(s): of the s-th.
template <int S, int L, class Bias>
__device__ __forceinline__ Query score_query(const RouteArgs &A, Bias bias, float (&c)[S]) {
  const bool soft = A.mode == BOUTE_ROUTE_SOFTMAX;
  Query q = {-INFINITY, 1.f, false};
#pragma unroll
  for (int s = 0; s < S; ++s) q.m = max_nan(q.m, c[s]);
  if constexpr (L == 32) {
    q.m = warp_max_nan(q.m);
  } else {
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) q.m = max_nan(q.m, __shfl_xor_sync(kAll, q.m, o));
  }
  q.bad = isnan(q.m) || (soft && q.m == INFINITY);
  if (soft && (!A.by_logits || !A.renorm)) {
    float sum = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) sum += exp2_fast((c[s] - q.m) * kLog2e);
    q.inv_sum = __fdividef(1.f, team_sum<L>(sum));
  }
  if (A.by_logits) {
#pragma unroll
    for (int s = 0; s < S; ++s) c[s] = q.bad ? -INFINITY : c[s];
  } else {
    // (the mode asked once, not for every expert)
    if (soft)
#pragma unroll
      for (int s = 0; s < S; ++s)
        c[s] = c[s] > -INFINITY && !q.bad
                   ? __fadd_rn(exp2_fast((c[s] - q.m) * kLog2e) * q.inv_sum, bias(s))
                   : -INFINITY;
    else
#pragma unroll
      for (int s = 0; s < S; ++s)
        c[s] = c[s] > -INFINITY && !q.bad ? __fadd_rn(logistic(c[s]), bias(s)) : -INFINITY;
  }
  return q;
}
// In place of the first choice of a query whose choice hangs on tiny values, of which those
// compared have too few bits: it is made after the main loop, straight from the definition. (Rare:
// making every value with all its bits took 4 to 8 % longer.)
constexpr int kLater = -2;
// Writes the chosen of a query: this lane's N candidates e (-1: none) of logits x in their places.
// later (if any): the warp's note that a query has been left for later.
template <int N, int L>
__device__ __forceinline__ void write_chosen(const RouteArgs &A, const Query &q, long long row,
                                             bool live, const int (&e)[N], const int (&place)[N],
                                             const float (&x)[N], int *hist, int *later) {
  float w[N], sum = 0.f;
  bool few = false;
#pragma unroll
  for (int j = 0; j < N; ++j) {
    const bool in = e[j] >= 0 && place[j] < A.k;
    w[j] = in ? q.score(A, x[j]) : 0.f;
    sum += w[j];
    few |= in && w[j] < kFewBits;
  }
  if (A.renorm) sum = team_sum<L>(sum);
  const unsigned teams = __ballot_sync(kAll, few);
  if (teams) {  // (a team's, whatever the warp's other queries)
    if (later && !A.by_logits) {
      bool tiny = false;
#pragma unroll
      for (int j = 0; j < N; ++j)
        tiny |= e[j] >= 0 && place[j] < A.k && fabsf(q.value(A, x[j], e[j])) < kFewBits;
      if (of_team<L>(__ballot_sync(kAll, tiny))) {
        if (live && (threadIdx.x & 31) % L == 0) A.idx[row * A.k] = kLater;
        live = false;
        *later = 1;
      }
      __syncwarp();
    }
    float top = -INFINITY, over[N], all = 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) top = e[j] >= 0 && place[j] < A.k ? fmaxf(top, x[j]) : top;
    top = team_max<L>(top);
#pragma unroll
    for (int j = 0; j < N; ++j) {
      const bool in = e[j] >= 0 && place[j] < A.k;
      over[j] = !in ? 0.f
                : A.renorm && sum < kSmallSum ? q.score_over(A, x[j], top)
                                              : q.whole_score(A, x[j]);
      all += over[j];
    }
    all = team_sum<L>(all);
    if (of_team<L>(teams)) {
      sum = all;
#pragma unroll
      for (int j = 0; j < N; ++j) w[j] = over[j];
    }
  }
  if (A.renorm) {
    const float inv = sum > 0.f ? __fdividef(1.f, sum) : 0.f;
#pragma unroll
    for (int j = 0; j < N; ++j) w[j] *= inv;
  }
#pragma unroll
  for (int j = 0; j < N; ++j) {
    if (!live || place[j] >= A.k) continue;
    if (!BOUTE_INB(place[j], A.k) || !BOUTE_INB(row, A.rows)) continue;
    A.idx[row * A.k + place[j]] = e[j];
    A.weight[row * A.k + place[j]] = q.bad ? NAN : A.factor * w[j];
    if (A.load && e[j] >= 0 && BOUTE_INB(e[j], A.E)) atomicAdd(hist + e[j], 1);
  }
}
// c of an expert, with the bits that fp32 has for its score where it is tiny.
__device__ __forceinline__ float value_refined(const RouteArgs &A, const Query &q, long long row,
                                               int e) {
  const float x = logit_at(A, row, e), v = q.value(A, x, e);
  if (!(fabsf(v) < kFewBits)) return v;
  return __fadd_rn(q.whole_score(A, x), A.bias ? A.bias[e] : 0.f);
}
// A query by such values, by a whole warp.
__device__ __forceinline__ void route_refined(const RouteArgs &A, long long row, int *hist) {
  const int lane = threadIdx.x & 31, per = A.E / A.G;
  Query q = {-INFINITY, 1.f, false};  // (a query without a distribution is not marked)
  for (int i = lane; i < A.E; i += 32) q.m = fmaxf(q.m, logit_at(A, row, i));
  q.m = team_max<32>(q.m);
  if (A.mode == BOUTE_ROUTE_SOFTMAX) {
    float sum = 0.f;
    for (int i = lane; i < A.E; i += 32) sum += exp2_fast((logit_at(A, row, i) - q.m) * kLog2e);
    q.inv_sum = __fdividef(1.f, team_sum<32>(sum));
  }
  float score = -INFINITY;  // of group `lane`
  for (int g = 0; g < A.G; ++g) {
    float a = -INFINITY, b = -INFINITY;
    for (int i = lane; i < per; i += 32)
      join_two(a, b, value_refined(A, q, row, g * per + i), -INFINITY);
    for (int o = 16; o > 0; o >>= 1)
      join_two(a, b, __shfl_xor_sync(kAll, a, o), __shfl_xor_sync(kAll, b, o));
    if (lane == g) score = A.group_top == 2 && b > -INFINITY ? a + b : a;
  }
  int rank = 0, e[1] = {-1}, place[1] = {lane};
  for (int h = 0; h < A.G; ++h) {
    const float other = __shfl_sync(kAll, score, h);
    rank += other > score || (other == score && h < lane);
  }
  const unsigned kept =
      __ballot_sync(kAll, A.keep == A.G || (rank < A.keep && score > -INFINITY));
  unsigned long long last = ~0ull;
  for (int r = 0; r < A.k; ++r) {
    unsigned long long best = 0ull;
    for (int i = lane; i < A.E; i += 32) {
      const float v = kept >> (i / per) & 1u ? value_refined(A, q, row, i) : -INFINITY;
      const unsigned long long key = v > -INFINITY ? make_key(v, (unsigned)i) : 0ull;
      if (key < last) best = max(best, key);
    }
    for (int o = 16; o > 0; o >>= 1) best = max(best, shfl_xor64(best, o));
    if (lane == r && best) e[0] = (int)key_index(best);
    last = best;
  }
  const float x[1] = {e[0] >= 0 ? logit_at(A, row, e[0]) : -INFINITY};
  write_chosen<1, 32>(A, q, row, true, e, place, x, hist, nullptr);
}
// A warp's marked queries, of the groups of `of` neighbours that it took.
__device__ __forceinline__ void route_later(const RouteArgs &A, const int *later, int of,
                                            int *hist) {
  __syncwarp();
  if (*later == 0) return;
  const long long step = (long long)gridDim.x * kWarps * of;
  for (long long row0 = ((long long)blockIdx.x * kWarps + (threadIdx.x >> 5)) * of; row0 < A.rows;
       row0 += step)
    for (long long row = row0; row < min(row0 + of, A.rows); ++row)
      if (A.idx[row * A.k] == kLater) {
        __syncwarp();
        route_refined(A, row, hist);
      }
}
// The block's load: cleared, and added to the whole one. (Behind clear_load_kernel too the wait
// comes before any read or write of the call's arrays: that kernel has waited for what came before
// it, but only a grid's own wait makes that visible to it.)
__device__ __forceinline__ void begin_load(const RouteArgs &A, int *hist) {
  pdl_wait();
  pdl_trigger();
  if (!A.load) return;
  for (int e = threadIdx.x; e < A.E; e += kThreads) hist[e] = 0;
  __syncthreads();
}
__device__ __forceinline__ void end_load(const RouteArgs &A, const int *hist) {
  if (!A.load) return;
  __syncthreads();
  for (int e = threadIdx.x; e < A.E; e += kThreads)
    if (gridDim.x == 1) A.load[e] = hist[e];
    else if (hist[e]) atomicAdd(A.load + e, hist[e]);
}

// A team's n <= 8 OWN keys (all different, in its part of shared memory, any order) in order: lane
// l has those of places l, l + 8 .. (0: none). Sums in this order do not depend on how a query's
// team found them.
template <int OWN, class Key>
__device__ __forceinline__ void in_order(Key *to, int n, int l, Key (&key)[OWN],
                                         int (&place)[OWN]) {
  __syncwarp();
  int rank[OWN];
#pragma unroll
  for (int j = 0; j < OWN; ++j) {
    place[j] = l + j * 8;
    key[j] = place[j] < n ? to[place[j]] : Key(0);
    rank[j] = 0;
  }
#pragma unroll
  for (int i = 0; i < 8 * OWN; ++i) {
    const Key o = __shfl_sync(kAll, key[i / 8], i % 8, 8);
#pragma unroll
    for (int j = 0; j < OWN; ++j) rank[j] += o > key[j];
  }
  __syncwarp();
#pragma unroll
  for (int j = 0; j < OWN; ++j)
    if (place[j] < n && BOUTE_INB(rank[j], n)) to[rank[j]] = key[j];
  __syncwarp();
#pragma unroll
  for (int j = 0; j < OWN; ++j) key[j] = place[j] < n ? to[place[j]] : Key(0);
  __syncwarp();
}

// 16-bit logits, compared as they are.
template <int S, int K, bool HALF>
__global__ void __launch_bounds__(kThreads, 4) route_pairs_kernel(RouteArgs A) {
  // Where a lane's logits are many against its list, those that reach a bound are ranked alone
  // (262144 queries of 256, k = 4: 35 us, all as keys 48, k = 8: 51 and 64; but 131072 of 64,
  // k = 8: 23 and 17). All as keys also where more than two lists reach it (many equal ones).
  constexpr bool BOUND = S >= 4 * K;
  // queries of a warp; a lane's candidates
  constexpr int L = 8, kTeams = 32 / L, kOwn = BOUND ? K / 4 : (K + L - 1) / L;
  extern __shared__ int hist[];  // the block's load
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = A.E, l = lane % L, e0 = l * S;
  begin_load(A, hist);
  const long long step = (long long)gridDim.x * kWarps * kTeams;
  for (long long row0 = ((long long)blockIdx.x * kWarps + warp) * kTeams; row0 < A.rows;
       row0 += step) {
    // (a team beyond the last query repeats the last, and writes nothing)
    const bool live = row0 + lane / L < A.rows;
    const long long row = min(row0 + lane / L, A.rows - 1);
    int e[kOwn], place[kOwn];  // candidates l, l + L .., and their ranks
    float x[kOwn];             // their logits
    Query q = {-INFINITY, 1.f, false};
    using P = Pair<HALF>;
    constexpr unsigned inf = P::kInf, kSlots = L * kOwn;
    auto value = [](unsigned key) {
      const unsigned o = key >> 16;
      return P::value(o & 0x8000u ? o ^ 0x8000u : o ^ 0xffffu);
    };
    __shared__ unsigned keys[kWarps * kTeams][kSlots];
    const bool soft = A.mode == BOUTE_ROUTE_SOFTMAX;
    const unsigned short *logits = (const unsigned short *)A.logits + row * A.ld;
    P w[S / 2], top;
    {
      uint32_t v[S / 2];
      load_words<S / 2, 2>(v, logits, e0, E, E, A.vec, (inf | 0x8000u) * 0x10001u);
#pragma unroll
      for (int i = 0; i < S / 2; ++i) w[i].w = v[i];
    }
    // keys: order bits (-0 as +0) over the expert's complement: equal values go to the lowest index
    unsigned hit = 0u, key[kOwn];
    int n = kSlots + 1, first = 0;
    if constexpr (BOUND) {
      // a bound that K reach, of finite values: which of this lane's logits do (of its pair i
      // bits i and 16 + i)
      const P lowest = {((inf | 0x8000u) - 1u) * 0x10001u};
      const P bound = max(bound_of<K>(w, top), lowest);
      q.m = P::value(top.w & 0xffffu);
#pragma unroll
      for (int i = 0; i < S / 2; ++i) hit |= w[i].reaches(bound) & 0x00010001u << i;
      first = hits_before(__popc(hit), l, n);
    }
    if (BOUND && !__any_sync(kAll, n > (int)kSlots)) {
      unsigned *to = keys[warp * kTeams + lane / L];
      for (int at = first; hit; ++at) {
        const int b = __ffs(hit) - 1, index = e0 + 2 * (b & 15) + (b >> 4);
        hit &= hit - 1u;
        if (!BOUTE_INB(index, E)) continue;
        unsigned u = logits[index];
        if (u == 0x8000u) u = 0u;
        u ^= u & 0x8000u ? 0xffffu : 0x8000u;
        if (BOUTE_INB(at, kSlots)) to[at] = u << 16 | (0xffffu - (unsigned)index);
      }
      in_order<kOwn>(to, n, l, key, place);
    } else {  // all as keys; a NaN is largest, +inf next, -inf smallest
      unsigned c[S], best[K];
      const unsigned below = (0xffffu - e0) | (0xffffu - e0 - 1u) << 16;
#pragma unroll
      for (int i = 0; i < S / 2; ++i) {
        const uint32_t v = w[i].plus_zero().w;
        const uint32_t o = v ^ (((v >> 15 & 0x00010001u) * 0x7fffu) | 0x80008000u);
        c[2 * i] = __byte_perm(o, below - 0x00020002u * i, 0x1054);
        c[2 * i + 1] = __byte_perm(o, below - 0x00020002u * i, 0x3276);
      }
      best_of<S, K>(c, best);
      if (!BOUND) q.m = value(best[0]);
#pragma unroll
      for (int j = 0; j < kOwn; ++j) {
        key[j] = 0u;
#pragma unroll
        for (int i = j * L; i < K && i < (j + 1) * L; ++i)
          key[j] = l == i - j * L ? best[i] : key[j];
        if (key[j] >> 16 <= (0x7fffu ^ inf)) key[j] = 0u;  // -inf
        place[j] = l + j * L;
      }
    }
    q.bad = isnan(q.m) || (soft && q.m == INFINITY);
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      e[j] = key[j] && !q.bad ? (int)(0xffffu - (key[j] & 0xffffu)) : -1;
      x[j] = value(key[j]);
    }
    if (soft && !A.renorm) {
      float sum = 0.f;
#pragma unroll
      for (int i = 0; i < S / 2; ++i)
        sum += exp2_fast((P::value(w[i].w & 0xffffu) - q.m) * kLog2e) +
               exp2_fast((P::value(w[i].w >> 16) - q.m) * kLog2e);
      q.inv_sum = __fdividef(1.f, team_sum<L>(sum));
    }
    write_chosen<kOwn, L>(A, q, row, live, e, place, x, hist, nullptr);
  }
  end_load(A, hist);
}

// Teams of 8 lanes with S exact values each, of which those that reach a bound are ranked alone.
// Lane l has the A.own <= S experts from l own on.
template <int S, int K>
__global__ void __launch_bounds__(kThreads, S > 16 ? 4 : 5) route_bound_kernel(RouteArgs A) {
  constexpr int L = 8, kTeams = 32 / L, kOwn = K / 4, kSlots = L * kOwn;
  extern __shared__ int hist[];  // the block's load; then, with groups, c and the groups' scores
  __shared__ unsigned long long keys[kWarps * kTeams][kSlots];
  __shared__ int later[kWarps];
  __shared__ alignas(16) float bias[L * (S + 4)];  // (lanes' parts begin in different banks)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = A.E, l = lane % L;
  const int e0 = l * A.own, end = min(e0 + A.own, E);
  float *shared_c = (float *)(hist + E) + (warp * kTeams + lane / L) * shared_stride(E);
  unsigned long long *to = keys[warp * kTeams + lane / L];
  if (lane == 0) later[warp] = 0;
  begin_load(A, hist);
  for (int i = threadIdx.x; i < L * S; i += kThreads) {
    const int at = i % S, e = i / S * A.own + at;
    bias[i / S * (S + 4) + at] = A.bias && at < A.own && e < E ? fmaxf(A.bias[e], -INFINITY) : 0.f;
  }  // (no NaN)
  __syncthreads();
  const float4 *mine = (const float4 *)(bias + l * (S + 4));
  const long long step = (long long)gridDim.x * kWarps * kTeams;
  for (long long row0 = ((long long)blockIdx.x * kWarps + warp) * kTeams; row0 < A.rows;
       row0 += step) {
    // (a team beyond the last query repeats the last, and writes nothing)
    const bool live = row0 + lane / L < A.rows;
    const long long row = min(row0 + lane / L, A.rows - 1);
    float c[S];
    load_logits(A, row, e0, end, c);
    const Query q = score_query<S, L>(A, [&](int s) {
      const float4 b = mine[s / 4];
      return s % 4 == 0 ? b.x : s % 4 == 1 ? b.y : s % 4 == 2 ? b.z : b.w;
    }, c);
    apply_groups<S, L>(A, c, shared_c, e0, end, l);
    const float bound = fmaxf(bound_of<K>(c), -FLT_MAX);
    unsigned hit = 0u;
#pragma unroll
    for (int s = 0; s < S; ++s) hit |= c[s] >= bound ? 1u << s : 0u;
    int n, e[kOwn], place[kOwn];
    float x[kOwn];
    unsigned long long key[kOwn];
    const int first = hits_before(__popc(hit), l, n);
    if (!__any_sync(kAll, n > kSlots)) {
      for (int at = first; hit; ++at) {
        const int i = e0 + __ffs(hit) - 1;
        hit &= hit - 1u;
        if (BOUTE_INB(i, E) && BOUTE_INB(at, kSlots))
          to[at] = make_key(q.value(A, logit_at(A, row, i), i), (unsigned)i);
      }
      in_order<kOwn>(to, n, l, key, place);
    } else {  // many equal ones: the largest, k times
#pragma unroll
      for (int j = 0; j < kOwn; ++j) key[j] = 0ull, place[j] = l + j * L;
      for (int r = 0; r < A.k; ++r) {
        float top = c[0];
#pragma unroll
        for (int s = 1; s < S; ++s) top = fmaxf(top, c[s]);
#pragma unroll
        for (int o = 1; o < L; o *= 2) top = fmaxf(top, other_lane(top, o));
        int at = S;
#pragma unroll
        for (int s = S - 1; s >= 0; --s) at = c[s] == top ? s : at;
        int from = at < S && top > -INFINITY ? l : L;
#pragma unroll
        for (int o = 1; o < L; o *= 2) from = min(from, __shfl_xor_sync(kAll, from, o));
        const int i = __shfl_sync(kAll, e0 + at, from % L, L);
#pragma unroll
        for (int s = 0; s < S; ++s) c[s] = l == from && s == at ? -INFINITY : c[s];
#pragma unroll
        for (int j = 0; j < kOwn; ++j)
          if (r == l + j * L && from < L) key[j] = make_key(top, (unsigned)i);
      }
    }
#pragma unroll
    for (int j = 0; j < kOwn; ++j) {
      e[j] = key[j] ? (int)key_index(key[j]) : -1;
      x[j] = e[j] >= 0 ? logit_at(A, row, e[j]) : -INFINITY;
    }
    write_chosen<kOwn, L>(A, q, row, live, e, place, x, hist, later + warp);
  }
  route_later(A, later + warp, kTeams, hist);
  end_load(A, hist);
}

// ---- a warp to a query -------------------------------------------------------------------
// The k largest of the lanes' values, lane r with the r-th: its value and its expert (-1: none).
// Each lane sorts its K >= min(k, S) best; k rounds take the largest head of the 32 lists. Equal
// values go to the lowest expert: of several lanes the lowest, of a lane's the occurrences in order.
template <int S, int K>
__device__ __forceinline__ void choose(const float (&c)[S], int k, float &mine, int &expert) {
  const int lane = threadIdx.x & 31;
  float v[S];
#pragma unroll
  for (int s = 0; s < S; ++s) v[s] = c[s];
  best_in_lane<S, K>(v);
  mine = -INFINITY;
  int owner = 0;
  constexpr bool kShort = K < S;  // lists of K >= k: picks beyond k are not used
  constexpr int kTimes = kShort ? K : 4;
#pragma unroll (kTimes)
  for (int r = 0; r < (kShort ? K : k); ++r) {
    const float best = warp_max_nan(v[0]);
    const int from = __ffs(__ballot_sync(kAll, v[0] == best)) - 1;
    owner = lane == r ? from : owner;
    mine = lane == r ? best : mine;
    const bool own = lane == from;
#pragma unroll
    for (int i = 0; i + 1 < K; ++i) v[i] = own ? v[i + 1] : v[i];
    v[K - 1] = own ? -INFINITY : v[K - 1];
  }
  const float before = __shfl_up_sync(kAll, mine, 1);
  const int by = __shfl_up_sync(kAll, owner, 1);
  const bool again = lane > 0 && mine == before && owner == by && mine > -INFINITY;
  const unsigned repeats = __ballot_sync(kAll, again);
  int nth = 0;  // which of its lane's equal values this one is
  if (repeats)
    for (int r = lane; repeats >> r & 1u; --r) ++nth;
  expert = -1;
#pragma unroll
  for (int s = 0; s < S; ++s)
    if (__shfl_sync(kAll, c[s], owner) == mine && nth-- == 0) expert = owner * S + s;
  if (mine == -INFINITY) expert = -1;
}

template <int S, int K>
__global__ void __launch_bounds__(kThreads, S > 8 ? 1 : 5) route_warp_kernel(RouteArgs A) {
  extern __shared__ int hist[];
  __shared__ int later[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, e0 = lane * S;
  float *shared_c = (float *)(hist + A.E) + warp * shared_stride(A.E);
  if (lane == 0) later[warp] = 0;
  __syncwarp();
  begin_load(A, hist);
  float bias[S];
  load_bias(A, e0, bias);
  for (long long row = (long long)blockIdx.x * kWarps + warp; row < A.rows;
       row += (long long)gridDim.x * kWarps) {
    float c[S], mine;
    load_logits(A, row, e0, A.E, c);
    const Query q = score_query<S, 32>(A, [&](int s) { return bias[s]; }, c);
    apply_groups<S, 32>(A, c, shared_c, e0, A.E, lane);
    int e[1], place[1] = {lane};
    choose<S, K>(c, A.k, mine, e[0]);
    if (lane >= A.k) e[0] = -1;
    const float x[1] = {e[0] < 0 ? -INFINITY : A.by_logits ? mine : logit_at(A, row, e[0])};
    write_chosen<1, 32>(A, q, row, true, e, place, x, hist, later + warp);
  }
  route_later(A, later + warp, 1, hist);
  end_load(A, hist);
}

__global__ void clear_load_kernel(int *load, int E) {
  pdl_wait();
  pdl_trigger();
  for (int e = threadIdx.x; e < E; e += blockDim.x) load[e] = 0;
}

// ---- a query's logits -----------------------------------------------------------------
// The S logits of a lane as they are stored.
template <class T, int S>
struct Raw {
  static constexpr int kWords = S * (int)sizeof(T) / 4;
  alignas(kWords < 4 ? 4 * kWords : 16) uint32_t w[kWords];
  __device__ __forceinline__ T at(int s) const {
    T t;
    if constexpr (sizeof(T) == 4) {
      t = __uint_as_float(w[s]);
    } else {
      const unsigned short h = (unsigned short)(s % 2 ? w[s / 2] >> 16 : w[s / 2] & 0xffffu);
      memcpy(&t, &h, 2);
    }
    return t;
  }
  // vec: rows on boundaries of a lane's bytes (16 at most) and E a multiple of S
  __device__ __forceinline__ void load(const T *x, int E, bool vec) {
    const int e0 = (threadIdx.x & 31) * S;
    if (vec) {
      if (e0 < E && BOUTE_INB(e0 + S - 1, E)) {
        if constexpr (kWords >= 4) {
#pragma unroll
          for (int i = 0; i < kWords / 4; ++i) ((uint4 *)w)[i] = ((const uint4 *)(x + e0))[i];
        } else if constexpr (kWords == 2) {
          *(uint2 *)w = *(const uint2 *)(x + e0);
        } else {
          w[0] = *(const uint32_t *)(x + e0);
        }
        return;
      }
#pragma unroll
      for (int i = 0; i < kWords; ++i) w[i] = none();
    } else {
      T t[S];
#pragma unroll
      for (int s = 0; s < S; ++s) t[s] = e0 + s < E ? x[e0 + s] : from_float<T>(-INFINITY);
      memcpy(w, t, sizeof(w));
    }
  }
  static __device__ __forceinline__ uint32_t none() {  // words of -inf
    T t[2] = {from_float<T>(-INFINITY), from_float<T>(-INFINITY)};
    uint32_t v;
    memcpy(&v, t, 4);
    return v;
  }
};

// ---- gradient ----------------------------------------------------------------------------
struct RouteGradArgs {
  long long rows, ld, ldd;
  int E, mode, k, renorm, vec;
  float factor;
  const int *idx;
  const float *g_weight;
};

// A warp's: n elements from p on are 0, by 16-byte vectors between the ends.
template <class T>
__device__ __forceinline__ void clear_run(T *p, int n, int lane) {
  constexpr int kOf = 16 / sizeof(T);
  const int head = min(n, (int)((16 - (uintptr_t)p % 16) % 16 / sizeof(T)));
  const int whole = (n - head) / kOf, tail = head + whole * kOf;
  uint4 *v = (uint4 *)(p + head);
  for (int i = lane; i < whole; i += 32)
    if (BOUTE_INB(head + (i + 1) * kOf - 1, n)) v[i] = make_uint4(0u, 0u, 0u, 0u);
  if (lane < head) p[lane] = from_float<T>(0.f);
  if (tail + lane < n) p[tail + lane] = from_float<T>(0.f);
}
// A warp's: go(x) for each of n elements from p on, 16-byte vectors between the ends.
template <class T, class Go>
__device__ __forceinline__ void for_run(const T *p, int n, int lane, Go go) {
  constexpr int kOf = 16 / sizeof(T);
  const int head = min(n, (int)((16 - (uintptr_t)p % 16) % 16 / sizeof(T)));
  const int whole = (n - head) / kOf, tail = head + whole * kOf;
  if (lane < head) go(to_float(p[lane]));
  if (tail + lane < n) go(to_float(p[tail + lane]));
  const uint4 *v = (const uint4 *)(p + head);
#pragma unroll 4
  for (int i = lane; i < whole; i += 32) {
    if (!BOUTE_INB(head + (i + 1) * kOf - 1, n)) continue;
    const uint4 w = v[i];
    T t[kOf];
    memcpy(t, &w, 16);
#pragma unroll
    for (int j = 0; j < kOf; ++j) go(to_float(t[j]));
  }
}
// The gradient where it is 0 but for the chosen experts: logistic scores, and a renormalised
// softmax (SOFT), of which the chosen logits count, and the whole row only for whether a score is 0
// (below 2^-149; its weight is 0 then, and so is its gradient). A query costs its row's bytes twice
// then: 131072 rows of 160 fp32, k = 6: 29.7 us; logistic, of which the chosen alone are read, 26.4.
//   w_i = factor s_i / S:  dx_i = factor s_i / S (g_i - sum_j g_j s_j / S) [ (1 - s_i): logistic ].
// 32 / team queries to a warp: the chosen logits are gathered, the rows cleared, the gradients put
// in.
template <class T, bool SOFT>
__global__ void __launch_bounds__(kThreads, SOFT ? 6 : 0)
    route_grad_chosen_kernel(const T *logits, RouteGradArgs A, T *dlogits, int team) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, r = lane % team, per = 32 / team;
  const long long step = (long long)gridDim.x * kWarps * per;
  for (long long row0 = ((long long)blockIdx.x * kWarps + (threadIdx.x >> 5)) * per; row0 < A.rows;
       row0 += step) {
    const long long row = row0 + lane / team;
    const int n = (int)min((long long)per, A.rows - row0);
    int e = -1;
    float x = -INFINITY, g = 0.f, most = -INFINITY;
    if (row < A.rows && r < A.k) {
      e = A.idx[row * A.k + r];
      if (e >= A.E) e = -1;
      if (SOFT || e >= 0) g = A.factor * A.g_weight[row * A.k + r];
      if (!SOFT && e >= 0) x = to_float(logits[row * A.ld + e]);
    }
    if constexpr (SOFT) {  // the largest logit of the warp's rows, all of whose loads come first
      auto larger = [&](float y) { most = max_nan(most, y); };
      if (A.ld == A.E) {
        for_run(logits + row0 * A.ld, n * A.E, lane, larger);
      } else {
        for (int i = 0; i < n; ++i) for_run(logits + (row0 + i) * A.ld, A.E, lane, larger);
      }
      if (e >= 0) x = to_float(logits[row * A.ld + e]);
      else g = 0.f;
    }
    float d = 0.f;
    if constexpr (SOFT) {
      // a score is 0 only if the largest logit of the warp's rows is far above the least chosen one
      most = warp_max_nan(most);
      const float below = team_max<32>(e >= 0 ? most - x : -INFINITY);
      bool held = e >= 0;
      if (!(below * kLog2e <= -kLeastLog2 - 10.f) || isnan(most)) {  // (a sum of 1024 at most)
        float own_m = -INFINITY, own_sum = 1.f;  // of this lane's row
        for (int i = 0; i < n; ++i) {
          float m = -INFINITY, sum = 0.f;
          const T *at = logits + (row0 + i) * A.ld;
          for (int j = lane; j < A.E; j += 32) m = max_nan(m, to_float(at[j]));
          m = warp_max_nan(m);
          for (int j = lane; j < A.E; j += 32) sum += exp2_fast((to_float(at[j]) - m) * kLog2e);
          sum = team_sum<32>(sum);
          if (lane / team == i) own_m = m, own_sum = sum;
        }
        held = e >= 0 && (x - own_m) * kLog2e - __log2f(own_sum) >= kLeastLog2;
      }
      const float top = team_max(held ? x : -INFINITY, team);
      const float v = held ? exp2_fast((x - top) * kLog2e) : 0.f;
      const float S = team_sum(v, team), w = S > 0.f ? v / S : 0.f;
      d = w * (g - team_sum(w * g, team));
    } else if (A.renorm) {
      float v = e >= 0 ? logistic(x) : 0.f, S = team_sum(v, team);
      if (__any_sync(kAll, e >= 0 && v < kFewBits)) {  // tiny scores, as in write_chosen
        const float tiny = team_max(e >= 0 && v < kFewBits ? 1.f : 0.f, team);
        const float top = team_max(e >= 0 ? x : -INFINITY, team);
        const float over = e >= 0 && x * kLog2e >= kLeastLog2
                               ? exp2_fast((x - top) * kLog2e) / (1.f + exp2_fast(x * kLog2e))
                               : 0.f;
        const float all = team_sum(over, team);
        if (tiny > 0.f && S < kSmallSum) v = over, S = all;
      }
      const float w = S > 0.f ? v / S : 0.f;
      const float q = exp2_fast(-fabsf(x) * kLog2e);  // 1 - s without the difference
      d = w * (g - team_sum(w * g, team)) * (x >= 0.f ? q : 1.f) / (1.f + q);
    } else if (e >= 0) {
      const float q = exp2_gradual(-fabsf(x) * kLog2e);
      d = g * q / ((1.f + q) * (1.f + q));
    }
    __syncwarp();  // (in place: every chosen logit has been read)
    // (131072 rows of 160 fp32 with a pitch: element by element 29 us, looking for each row's ends
    // 31; of 61 bf16 without one: 13.2 element by element, 6.7 looking for the run's ends)
    if (A.vec && A.ldd == A.E) {  // the rows are one run of 16-byte vectors
      uint4 *p = (uint4 *)(dlogits + row0 * A.E);
      const int vectors = BOUTE_INB((uintptr_t)p % 16, 1) ? n * A.E / (16 / (int)sizeof(T)) : 0;
      for (int i = lane; i < vectors; i += 32) p[i] = make_uint4(0u, 0u, 0u, 0u);
    } else if (A.ldd == A.E) {
      clear_run(dlogits + row0 * A.E, n * A.E, lane);
    } else {
      for (int i = 0; i < n; ++i)
        for (int j = lane; j < A.E; j += 32)
          dlogits[(row0 + i) * A.ldd + j] = from_float<T>(0.f);
    }
    __syncwarp();
    if (e >= 0 && BOUTE_INB(e, A.E) && BOUTE_INB(row, A.rows))
      dlogits[row * A.ldd + e] = from_float<T>(d);
  }
}

// A softmax whose weights are not renormalised: dx_j = s_j (ds_j - sum_i ds_i s_i), a warp per
// query.
template <class T, int S>
__global__ void __launch_bounds__(kThreads)
    route_grad_softmax_kernel(const T *logits, RouteGradArgs A, T *dlogits) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, E = A.E, k = A.k;
  const long long step = (long long)gridDim.x * kWarps;
  for (long long row = (long long)blockIdx.x * kWarps + (threadIdx.x >> 5); row < A.rows;
       row += step) {
    Raw<T, S> raw;
    raw.load(logits + row * A.ld, E, A.vec);
    float x[S], m = -INFINITY, sum = 0.f;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      x[s] = to_float(raw.at(s));
      m = max_nan(m, x[s]);
    }
    m = warp_max_nan(m);
    int e = lane < k ? A.idx[row * k + lane] : -1;
    if (e >= E) e = -1;
    const bool any = __any_sync(kAll, e >= 0) && m > -INFINITY;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      x[s] = any ? exp2_fast((x[s] - m) * kLog2e) : 0.f;
      sum += x[s];
    }
    const float inv = any ? __fdividef(1.f, warp_sum(sum)) : 0.f;
    float v = 0.f, ds = 0.f;
    if (e >= 0 && any) {
      v = exp2_fast((to_float(logits[row * A.ld + e]) - m) * kLog2e) * inv;
      ds = A.factor * A.g_weight[row * k + lane];
    }
    const float dot = any ? warp_sum(ds * v) : 0.f;
    __syncwarp();  // (in place: every chosen logit has been read)
    T out[S];
#pragma unroll
    for (int s = 0; s < S; ++s) out[s] = from_float<T>(-x[s] * inv * dot);
    T *dx = dlogits + row * A.ldd + lane * S;
    constexpr int kWords = Raw<T, S>::kWords;
    uint32_t w[kWords];
    memcpy(w, out, sizeof(w));
    if (A.vec) {
      if (lane * S < E && BOUTE_INB(lane * S + S - 1, E)) {
        if constexpr (kWords >= 4) {
#pragma unroll
          for (int i = 0; i < kWords / 4; ++i) ((uint4 *)dx)[i] = ((uint4 *)w)[i];
        } else if constexpr (kWords == 2) {
          *(uint2 *)dx = *(uint2 *)w;
        } else {
          *(uint32_t *)dx = w[0];
        }
      }
    } else {
#pragma unroll
      for (int s = 0; s < S; ++s)
        if (lane * S + s < E) dx[s] = out[s];
    }
    __syncwarp();
    if (e >= 0 && BOUTE_INB(e, E)) dlogits[row * A.ldd + e] = from_float<T>(v * (ds - dot));
  }
}

}  // namespace

BOUTE_BOUNDS_READER(route)

}  // namespace boute

using namespace boute;

// Experts of a lane: the fewest, a power of two, of which 32 lanes hold E.
template <class Go>
static int with_slots(int E, Go go) {
  if (E <= 64) return go(std::integral_constant<int, 2>{});
  if (E <= 128) return go(std::integral_constant<int, 4>{});
  if (E <= 256) return go(std::integral_constant<int, 8>{});
  if (E <= 512) return go(std::integral_constant<int, 16>{});
  return go(std::integral_constant<int, 32>{});
}
static int power_of_two(int k) {  // at least k
  int p = 1;
  while (p < k) p *= 2;
  return p;
}
// Whether a lane's S logits are vectors of up to 16 bytes on their boundaries in every row.
static bool vectors(const void *p, long long ld, int E, int S, size_t bytes) {
  const size_t b = std::min<size_t>(16, S * bytes);
  return (uintptr_t)p % b == 0 && ld * bytes % b == 0 && E % S == 0;
}

static bool shape_ok(const void *logits, int dtype, long long T, int E, long long ld, int mode,
                     int k, float factor) {
  return dtype_known(dtype) && T >= 0 && E >= 1 && ld >= E && k >= 1 && k <= E &&
         (mode == BOUTE_ROUTE_SOFTMAX || mode == BOUTE_ROUTE_SIGMOID) && isfinite(factor) &&
         (T == 0 || array_ok(logits, dtype_bytes(dtype)));
}
static int limits_ok(long long T, int E, int k) {
  if (E > BOUTE_MAX_EXPERTS || k > BOUTE_MAX_CHOICES || T * k >= (1ll << 31) || T >= (1ll << 31))
    return BOUTE_ERR_UNSUPPORTED;
  return device_ok();
}

extern "C" int boute_route(const void *logits, int dtype, long long T, int E, long long ld,
                           const float *bias, int mode, int G, int keep, int group_top, int k,
                           int renorm, float factor, int *idx, float *weight, int *load,
                           void *stream) {
  BOUTE_TRACE();
  if (!shape_ok(logits, dtype, T, E, ld, mode, k, factor) || G < 1 || E % G != 0 || keep < 1 ||
      keep > G || (group_top != 1 && group_top != 2) || (long long)k > (long long)keep * (E / G) ||
      !optional_ok(bias, 4) || !optional_ok(load, 4) ||
      (T > 0 && (!array_ok(idx, 4) || !array_ok(weight, 4))))
    return BOUTE_ERR_INVALID_ARG;
  if (G > BOUTE_MAX_GROUPS) return BOUTE_ERR_UNSUPPORTED;
  if (int r = limits_ok(T, E, k)) return r;
  const cudaStream_t s = (cudaStream_t)stream;
  if (T == 0) {
    if (load && cudaMemsetAsync(load, 0, E * sizeof(int), s) != cudaSuccess)
      return last_launch_status();
    return BOUTE_OK;
  }
  RouteArgs A = {};
  A.logits = logits, A.dtype = dtype, A.rows = T, A.ld = ld, A.bias = bias, A.E = E, A.mode = mode;
  A.G = G, A.keep = keep, A.group_top = group_top, A.k = k, A.renorm = renorm;
  A.factor = factor, A.idx = idx, A.load = load, A.weight = weight;
  const bool groups = keep < G;
  // (the sum of two scores has no counterpart among the logits)
  A.by_logits = !bias && !(groups && group_top == 2);
  const size_t bytes = dtype_bytes(dtype);
  A.vec = (uintptr_t)logits % 16 == 0 && ld * bytes % 16 == 0 && E * bytes % 16 == 0;
  // queries: of a warp; blocks: of an SM; S: experts of a lane. (At most 38 KB of shared memory.)
  auto run = [&](auto kernel, int queries, int blocks, int S) {
    A.group_lanes = E / G % S == 0 ? E / G / S : 0;
    const size_t smem =
        (size_t)E * 4 +
        (groups && !A.group_lanes ? (size_t)kWarps * queries * shared_stride(E) * 4 : 0);
    const long long all = (T + kWarps * queries - 1) / (kWarps * queries);
    // a few queries whose load is wanted: one block, which writes it itself
    const unsigned grid =
        load && all <= 2 ? 1u : (unsigned)std::min<long long>(all, (long long)blocks * num_sms());
    if (load && grid > 1)
      if (int r = launch_cluster(clear_load_kernel, 1, 256, 1, 0, s, load, E)) return r;
    return launch_cluster(kernel, grid, kThreads, 1, smem, s, A);
  };
  // Teams for pairs, and for other values where the queries give most SMs a block or two; and where
  // one block of them takes all queries, which then needs no launch to clear the load (of 64 fp32,
  // 32 queries: 2.5 us on the device with one launch or two, 64: 3.8 and 2.5, but a launch takes the
  // host 2). (us by
  // team and by warp: 131072 x 256 bf16 with bias, k = 4: 37, 60, in 8 groups, k = 8: 63, 107; 131072
  // x 64, 8 groups, k = 4: 29, 66; 256 experts, 8 groups, k = 8, of 300, 2000, 4099 and 10000
  // queries: 7.2, 4.1; 7.3, 5.7; 7.4, 8.4; 10.6, 13.9; 64 experts, k = 4, of 300, 2000 and 4099: 3.8,
  // 3.0; 3.9, 3.9; 4.0, 5.2.)
  using std::integral_constant;
  const bool pairs = A.by_logits && !groups && dtype != BOUTE_F32;
  auto team = [&](auto experts) {
    constexpr int S = decltype(experts)::value;
    auto teams = [&](auto list) {
      constexpr int K = decltype(list)::value;
      if (pairs)
        return dtype == BOUTE_F16 ? run(route_pairs_kernel<S, K, true>, 4, 4, S)
                                  : run(route_pairs_kernel<S, K, false>, 4, 4, S);
      // the lanes' shares of E: equal ones where they are whole vectors, unless only shares of S
      // leave each with experts of one group
      const int equal = E % (8 * (16 / (int)bytes)) == 0 ? E / 8 : S, per = E / G;
      A.own = groups && per % equal != 0 && per % S == 0 ? S : equal;
      return run(route_bound_kernel<S, K>, 4, S > 16 ? 4 : 5, A.own);
    };
    return k <= 4 ? teams(integral_constant<int, 4>{}) : teams(integral_constant<int, 8>{});
  };
  const bool one_block = load && T <= 2 * 4 * kWarps;
  if (E <= 256 && k <= 8 &&
      (pairs || one_block || T >= (E <= 128 ? 16ll : 24ll) * num_sms())) {
    if (E <= 64) return team(integral_constant<int, 8>{});
    if (E <= 128) return team(integral_constant<int, 16>{});
    return team(integral_constant<int, 32>{});
  }
  if (E <= 64) return run(route_warp_kernel<2, 2>, 1, 5, 2);
  if (E <= 128) return run(route_warp_kernel<4, 4>, 1, 5, 4);
  if (E <= 256)
    return k <= 4 ? run(route_warp_kernel<8, 4>, 1, 5, 8) : run(route_warp_kernel<8, 8>, 1, 5, 8);
  // (lists as short as the choice allows: 131072 x 512 bf16, k = 4: 95 us, whole lists 218)
  if (E <= 512)
    return k <= 4   ? run(route_warp_kernel<16, 4>, 1, 4, 16)
           : k <= 8 ? run(route_warp_kernel<16, 8>, 1, 4, 16)
                    : run(route_warp_kernel<16, 16>, 1, 4, 16);
  return k <= 8 ? run(route_warp_kernel<32, 8>, 1, 4, 32) : run(route_warp_kernel<32, 32>, 1, 4, 32);
}

extern "C" int boute_route_grad(const void *logits, int dtype, long long T, int E, long long ld,
                                int mode, int k, int renorm, float factor, const int *idx,
                                const float *g_weight, void *dlogits, long long ldd,
                                void *stream) {
  BOUTE_TRACE();
  if (!shape_ok(logits, dtype, T, E, ld, mode, k, factor) || ldd < E ||
      (dlogits == logits && ldd != ld) ||
      (T > 0 && (!array_ok(idx, 4) || !array_ok(g_weight, 4) ||
                 !array_ok(dlogits, dtype_bytes(dtype)))))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = limits_ok(T, E, k)) return r;
  if (T == 0) return BOUTE_OK;
  RouteGradArgs A = {T, ld, ldd, E, mode, k, renorm, 0, factor, idx, g_weight};
  const cudaStream_t s = (cudaStream_t)stream;
  return with_dtype(dtype, [&](auto tag) {
    using X = decltype(tag);
    if (mode == BOUTE_ROUTE_SIGMOID || renorm) {
      int team = power_of_two(k);
      // (a softmax's warp reads its rows at once: with 32 rows of 160 fp32, k = 1, 37.9 us, with 4 28.9)
      if (mode == BOUTE_ROUTE_SOFTMAX)
        while (team < 32 && 32 / team * E * sizeof(X) > 4096) team *= 2;
      A.vec = (uintptr_t)dlogits % 16 == 0 && (size_t)E * sizeof(X) % 16 == 0;
      const long long all = (T + kWarps * (32 / team) - 1) / (kWarps * (32 / team));
      const unsigned grid = (unsigned)std::min<long long>(all, (mode == BOUTE_ROUTE_SOFTMAX ? 6ll : 8ll) * num_sms());
      return launch_cluster(mode == BOUTE_ROUTE_SOFTMAX ? route_grad_chosen_kernel<X, true>
                                                        : route_grad_chosen_kernel<X, false>,
                            grid, kThreads, 1, 0, s, (const X *)logits, A, (X *)dlogits, team);
    }
    return with_slots(E, [&](auto slots) {
      constexpr int S = decltype(slots)::value;
      A.vec = vectors(logits, ld, E, S, sizeof(X)) && vectors(dlogits, ldd, E, S, sizeof(X));
      const unsigned grid =
          (unsigned)std::min<long long>((T + kWarps - 1) / kWarps, 8ll * num_sms());
      return launch_cluster(route_grad_softmax_kernel<X, S>, grid, kThreads, 1, 0, s,
                            (const X *)logits, A, (X *)dlogits);
    });
  });
}
