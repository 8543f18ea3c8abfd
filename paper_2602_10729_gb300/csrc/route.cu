// Routing of queries to experts: scores, the choice within the best groups,
// the weights and the load; and the gradient of the weights.
//
// A warp per query, lane l with the S experts l S .. l S + S - 1 (S a power of two,
// 32 S >= E), so that the lowest lane has the lowest indices. Each lane sorts the best
// of its values; k rounds then take the largest head of the 32 lists (one reduction
// each). Without a bias the logits themselves are compared, which have the order of the
// scores: only the chosen scores are computed then, and a softmax's sum only where the
// weights are not renormalised. 16-bit logits are compared as keys of their order bits
// with the expert's index below.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kWarps = 8, kThreads = 32 * kWarps;
constexpr float kLog2e = 1.4426950408889634f;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
__device__ __forceinline__ float exp2_fast(float y) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
// The warp's maximum in one instruction (a NaN wins; keys: unsigned).
__device__ __forceinline__ float warp_max(float v) {
  float r;
  asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ unsigned warp_max(unsigned v) { return __reduce_max_sync(kAll, v); }

__device__ __forceinline__ float logistic(float x) {  // (0 where exp(-x) overflows)
  float r;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(1.f + exp2_fast(-x * kLog2e)));
  return r;
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
      if (e0 < E) {
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

// ---- choosing --------------------------------------------------------------------------
__device__ __forceinline__ float key_none(float) { return -INFINITY; }
__device__ __forceinline__ unsigned key_none(unsigned) { return 0u; }

// Two values, and four or more by Batcher's odd-even merge sort, in descending order.
template <int L, class K>
__device__ __forceinline__ void sort_desc(K *v) {
#pragma unroll
  for (int p = 1; p < L; p *= 2)
#pragma unroll
    for (int q = p; q > 0; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < L; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (i + j + q < L && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
            const K a = v[i + j], b = v[i + j + q];
            v[i + j] = max(a, b);
            v[i + j + q] = min(a, b);
          }
}
// The L largest of c's S in descending order: runs of L are sorted, then joined two by two (the
// larger of each and the other's reverse form a bitonic run).
template <int S, int L, class K>
__device__ __forceinline__ void best_of(const K (&c)[S], K (&best)[L]) {
  K v[S];
#pragma unroll
  for (int s = 0; s < S; ++s) v[s] = c[s];
#pragma unroll
  for (int s = 0; s < S; s += L) sort_desc<L>(v + s);
#pragma unroll
  for (int o = L; o < S; o *= 2)
#pragma unroll
    for (int s = 0; s < S; s += 2 * o) {
#pragma unroll
      for (int i = 0; i < L; ++i) v[s + i] = max(v[s + i], v[s + o + L - 1 - i]);
#pragma unroll
      for (int q = L / 2; q > 0; q /= 2)
#pragma unroll
        for (int i = 0; i < L; ++i)
          if (!(i & q)) {
            const K a = v[s + i], b = v[s + i + q];
            v[s + i] = max(a, b);
            v[s + i + q] = min(a, b);
          }
    }
#pragma unroll
  for (int i = 0; i < L; ++i) best[i] = v[i];
}

// The k largest of the lanes' values, lane r with the r-th: its value and its expert (-1: none).
// v: each lane's L largest in descending order, L >= min(k, S). Keys (unsigned) are unique and
// carry the expert; equal floats go to the lowest expert: of several lanes the lowest, of one
// lane's the occurrences in order.
template <int S, int L, class K>
__device__ __forceinline__ void choose(const K (&c)[S], K (&v)[L], int k, K &mine, int &expert) {
  constexpr bool kKeys = std::is_same<K, unsigned>::value;
  const int lane = threadIdx.x & 31;
  mine = key_none(K{});
  int owner = 0;
#pragma unroll (L <= 4 ? L : 1)
  for (int r = 0; r < (L <= 4 && L < S ? L : k); ++r) {  // (picks beyond k are not used)
    const K best = warp_max(v[0]);
    bool own = v[0] == best;
    if constexpr (!kKeys) {
      const int from = __ffs(__ballot_sync(kAll, own)) - 1;
      owner = lane == r ? from : owner;
      own = lane == from;
    }
    mine = lane == r ? best : mine;
#pragma unroll
    for (int i = 0; i + 1 < L; ++i) v[i] = own ? v[i + 1] : v[i];
    v[L - 1] = own ? key_none(K{}) : v[L - 1];
  }
  if constexpr (kKeys) {
    expert = mine ? (int)(0xffffu - (mine & 0xffffu)) : -1;
  } else {
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
}

// The two largest of two pairs a >= b.
__device__ __forceinline__ void join_two(float &a, float &b, float a2, float b2) {
  b = fmaxf(fminf(a, a2), fmaxf(b, b2));
  a = fmaxf(a, a2);
}

// ---- groups ----------------------------------------------------------------------------
// Whether the lane's groups stay: a bit for each lane number g * width of a kept group g, 2^q =
// width lanes to a group. a, b: the two largest c of this lane's share of its group.
__device__ __forceinline__ unsigned keep_groups(float a, float b, int width, int keep,
                                                int group_top) {
  for (int o = 1; o < width; o *= 2)
    join_two(a, b, __shfl_xor_sync(kAll, a, o), __shfl_xor_sync(kAll, b, o));
  float score = group_top == 2 && b > -INFINITY ? a + b : a;
  const int lane = threadIdx.x & 31;
  unsigned kept = 0u;
  for (int r = 0; r < keep; ++r) {
    const float best = warp_max(score);
    if (best == -INFINITY) break;
    const int at = __ffs(__ballot_sync(kAll, score == best)) - 1;  // its group's first lane
    kept |= 1u << at;
    if ((lane ^ at) < width) score = -INFINITY;
  }
  return kept;
}

// Over teams of lanes (a power of two).
__device__ __forceinline__ float team_sum(float v, int team) {
  for (int o = team / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

// Pairs of 16-bit logits with -0 as +0 (and NaNs as one).
__device__ __forceinline__ uint32_t plus_zero(uint32_t w, __half) {
  uint32_t r;
  asm("add.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0u));
  return r;
}
__device__ __forceinline__ uint32_t plus_zero(uint32_t w, __nv_bfloat16) {
  uint32_t r;
  asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(w), "r"(0u));
  return r;
}

struct RouteArgs {
  long long rows, ld;
  const float *bias;
  int E, mode, G, keep, group_top, k, renorm, by_logits, vec;
  int team;   // lanes that hold the choices, a power of two
  int width;  // lanes to a group when its score is formed
  int whole;  // a lane's experts are of one group
  float factor;
  int *idx, *load;
  float *weight;
};

// K: unsigned for 16-bit logits compared as they are, float else (by_logits: the logits, else the
// scores with their bias). L: the lanes' lists.
template <int S, class K>
constexpr int kBlocks = S > 8 ? 1 : std::is_same<K, unsigned>::value ? 6 : 5;  // an SM's, at least
template <class T, int S, class K, int L>
__global__ void __launch_bounds__(kThreads, kBlocks<S, K>)
    route_kernel(const T *logits, RouteArgs A) {
  extern __shared__ int hist[];  // the block's load; then, with groups, c of each warp's query
  __shared__ float2 lanes_two[kWarps][32];
  constexpr bool kKeys = std::is_same<K, unsigned>::value;
  const bool groups = A.keep < A.G;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = A.E, k = A.k;
  const bool soft = A.mode == BOUTE_ROUTE_SOFTMAX;
  float *shared_c = (float *)(hist + E) + warp * E;
  float2 *pairs = lanes_two[warp];
  // (behind clear_load_kernel, which has waited for what came before, only the load waits)
  if (!A.load || gridDim.x == 1) pdl_wait();
  pdl_trigger();
  if (A.load) {
    for (int e = threadIdx.x; e < E; e += kThreads) hist[e] = 0;
    __syncthreads();
  }
  float bias[kKeys ? 1 : S];
  unsigned below[kKeys ? S / 2 : 1];  // pairs of the experts' complements
  if constexpr (kKeys) {
#pragma unroll
    for (int i = 0; i < S / 2; ++i)
      below[i] = (0xffffu - (lane * S + 2 * i)) | (0xffffu - (lane * S + 2 * i + 1)) << 16;
  } else {
#pragma unroll
    for (int s = 0; s < S; ++s)
      bias[s] = A.bias && lane * S + s < E ? fmaxf(A.bias[lane * S + s], -INFINITY) : 0.f;  // (NaN)
  }
  // the group whose share this lane takes, its first position there, its experts' (first) group
  const int per = E / A.G, g = lane / A.width, i0 = lane % A.width, of0 = lane * S / per;
  const long long step = (long long)gridDim.x * kWarps;
  long long row = (long long)blockIdx.x * kWarps + warp;
  Raw<T, S> next;
  if (row < A.rows) next.load(logits + row * A.ld, E, A.vec);
  for (; row < A.rows; row += step) {
    const Raw<T, S> raw = next;
    if (row + step < A.rows) next.load(logits + (row + step) * A.ld, E, A.vec);
    K c[S], v[L], mine;
    float m = -INFINITY, inv_sum = 1.f;  // of the softmax
    bool bad;
    int e;
    if constexpr (kKeys) {
      // order bits of pairs of logits, each over its expert's complement; a NaN is largest, +inf
      // next, -inf (and what is beyond E) smallest
      constexpr unsigned kInf = std::is_same<T, __half>::value ? 0xfc00u : 0xff80u;
#pragma unroll
      for (int i = 0; i < S / 2; ++i) {
        const uint32_t w = plus_zero(raw.w[i], T{});
        const uint32_t o = w ^ (((w >> 15 & 0x00010001u) * 0x7fffu) | 0x80008000u);
        c[2 * i] = __byte_perm(o, below[i], 0x1054);
        c[2 * i + 1] = __byte_perm(o, below[i], 0x3276);
      }
      best_of(c, v);
      if (soft && !A.renorm) {
        float x[S];
#pragma unroll
        for (int s = 0; s < S; ++s) m = max_nan(m, x[s] = to_float(raw.at(s)));
        m = warp_max(m);
        inv_sum = 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) inv_sum += exp2_fast((x[s] - m) * kLog2e);
        inv_sum = __fdividef(1.f, warp_sum(inv_sum));
      }
      choose(c, v, k, mine, e);
      const unsigned top = __shfl_sync(kAll, mine, 0) >> 16;
      bad = top > kInf || (soft && top == kInf);
      if (bad || mine >> 16 <= (0xffffu ^ kInf)) e = -1;
    } else {
      float x[S];
#pragma unroll
      for (int s = 0; s < S; ++s) {
        x[s] = to_float(raw.at(s));
        m = max_nan(m, x[s]);
      }
      m = warp_max(m);
      bad = isnan(m) || (soft && m == INFINITY);
      if (soft && (!A.by_logits || !A.renorm)) {
        float sum = 0.f;
#pragma unroll
        for (int s = 0; s < S; ++s) sum += exp2_fast((x[s] - m) * kLog2e);
        inv_sum = __fdividef(1.f, warp_sum(sum));
      }
      if (A.by_logits) {
#pragma unroll
        for (int s = 0; s < S; ++s) c[s] = x[s];
      } else if (soft) {
#pragma unroll
        for (int s = 0; s < S; ++s) c[s] = exp2_fast((x[s] - m) * kLog2e) * inv_sum + bias[s];
      } else {
#pragma unroll
        for (int s = 0; s < S; ++s) c[s] = logistic(x[s]) + bias[s];
      }
#pragma unroll
      for (int s = 0; s < S; ++s) c[s] = x[s] > -INFINITY && !bad ? c[s] : -INFINITY;
      if (groups) {
        float a = -INFINITY, b = -INFINITY;
        if (A.whole) {  // a lane's experts are of one group: the lanes' two largest will do
          float first = c[0], second = -INFINITY;
#pragma unroll
          for (int s = 1; s < S; ++s) join_two(first, second, c[s], -INFINITY);
          pairs[lane] = make_float2(first, second);
          __syncwarp();
          if (g < A.G)
            for (int i = i0; i < per / S; i += A.width) {
              const float2 v = pairs[g * per / S + i];
              join_two(a, b, v.x, v.y);
            }
        } else {
#pragma unroll
          for (int s = 0; s < S; ++s)
            if (lane * S + s < E) shared_c[lane * S + s] = c[s];
          __syncwarp();
          if (g < A.G)
            for (int i = i0; i < per; i += A.width)
              join_two(a, b, shared_c[g * per + i], -INFINITY);
        }
        const unsigned kept = keep_groups(a, b, A.width, A.keep, A.group_top);
        __syncwarp();
        if (A.whole) {
          const bool in = of0 < A.G && (kept >> (of0 * A.width) & 1u);
#pragma unroll
          for (int s = 0; s < S; ++s) c[s] = in ? c[s] : -INFINITY;
        } else {
          // (the lane's experts are neighbours: one division, then steps)
          int of = of0, left = (of + 1) * per - lane * S;
#pragma unroll
          for (int s = 0; s < S; ++s) {
            if (left-- == 0) {
              ++of;
              left = per - 1;
            }
            if (of >= A.G || !(kept >> (of * A.width) & 1u)) c[s] = -INFINITY;
          }
        }
      }
      best_of(c, v);
      choose(c, v, k, mine, e);
    }
    if (lane >= k) e = -1;
    // the chosen scores
    float w = 0.f;
    if (kKeys || A.by_logits) {
      float x;
      if constexpr (kKeys) {
        const unsigned o = mine >> 16, u = o & 0x8000u ? o ^ 0x8000u : o ^ 0xffffu;
        const unsigned short h = (unsigned short)u;
        T t;
        memcpy(&t, &h, 2);
        x = to_float(t);
      } else {
        x = mine;
      }
      if (soft && A.renorm) m = __shfl_sync(kAll, x, 0);
      if (e >= 0) w = !soft ? logistic(x) : exp2_fast((x - m) * kLog2e) * inv_sum;
    } else if (e >= 0) {
      const float x = to_float(logits[row * A.ld + e]);
      w = !soft ? logistic(x) : exp2_fast((x - m) * kLog2e) * inv_sum;
    }
    if (A.renorm) {
      const float sum = team_sum(w, A.team);
      w = sum > 0.f ? __fdividef(w, sum) : 0.f;
    }
    if (lane < k) {
      A.idx[row * k + lane] = e;
      A.weight[row * k + lane] = bad ? NAN : A.factor * w;
      if (A.load && e >= 0 && BOUTE_INB(e, E)) atomicAdd(hist + e, 1);
    }
  }
  if (A.load) {
    __syncthreads();
    pdl_wait();  // (until the load has been cleared)
    for (int e = threadIdx.x; e < E; e += kThreads)
      if (gridDim.x == 1) A.load[e] = hist[e];
      else if (hist[e]) atomicAdd(A.load + e, hist[e]);
  }
}

__global__ void clear_load_kernel(int *load, int E) {
  pdl_wait();
  pdl_trigger();
  for (int e = threadIdx.x; e < E; e += blockDim.x) load[e] = 0;
}

// ---- gradient ----------------------------------------------------------------------------
struct RouteGradArgs {
  long long rows, ld, ldd;
  int E, mode, k, renorm, vec;
  float factor;
  const int *idx;
  const float *g_weight;
};

// The gradient where it is 0 but for the chosen experts: logistic scores, and a renormalised
// softmax, of which only the chosen logits count:
//   w_i = factor s_i / S:  dx_i = factor s_i / S (g_i - sum_j g_j s_j / S) [ (1 - s_i): logistic ].
// 32 / team queries to a warp: the chosen logits are gathered, the rows cleared, the gradients put
// in.
template <class T>
__global__ void __launch_bounds__(kThreads)
    route_grad_chosen_kernel(const T *logits, RouteGradArgs A, T *dlogits, int team) {
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, r = lane % team, per = 32 / team;
  const bool soft = A.mode == BOUTE_ROUTE_SOFTMAX;
  const long long step = (long long)gridDim.x * kWarps * per;
  for (long long row0 = ((long long)blockIdx.x * kWarps + (threadIdx.x >> 5)) * per; row0 < A.rows;
       row0 += step) {
    const long long row = row0 + lane / team;
    const int n = (int)min((long long)per, A.rows - row0);
    int e = -1;
    float x = -INFINITY, g = 0.f;
    if (row < A.rows && r < A.k) {
      e = A.idx[row * A.k + r];
      if (e >= A.E) e = -1;
      if (e >= 0) {
        x = to_float(logits[row * A.ld + e]);
        g = A.factor * A.g_weight[row * A.k + r];
      }
    }
    float d = 0.f;
    if (soft) {
      float m = x;
      for (int o = team / 2; o > 0; o >>= 1) m = max_nan(m, __shfl_xor_sync(kAll, m, o));
      const float v = e >= 0 && x > -INFINITY ? exp2_fast((x - m) * kLog2e) : 0.f;
      const float S = team_sum(v, team), w = S > 0.f ? v / S : 0.f;
      d = w * (g - team_sum(w * g, team));
    } else if (A.renorm) {
      const float v = e >= 0 ? logistic(x) : 0.f, S = team_sum(v, team);
      const float w = S > 0.f ? v / S : 0.f;
      const float q = exp2_fast(-fabsf(x) * kLog2e);  // 1 - s without the difference
      d = w * (g - team_sum(w * g, team)) * (x >= 0.f ? q : 1.f) / (1.f + q);
    } else if (e >= 0) {
      const float q = exp2_fast(-fabsf(x) * kLog2e);
      d = g * q / ((1.f + q) * (1.f + q));
    }
    __syncwarp();  // (in place: every chosen logit has been read)
    if (A.vec && A.ldd == A.E) {  // the rows are one run of 16-byte vectors
      uint4 *p = (uint4 *)(dlogits + row0 * A.E);
      const int vectors = n * A.E / (16 / (int)sizeof(T));
      for (int i = lane; i < vectors; i += 32) p[i] = make_uint4(0u, 0u, 0u, 0u);
    } else {
      for (int i = 0; i < n; ++i)
        for (int j = lane; j < A.E; j += 32)
          dlogits[(row0 + i) * A.ldd + j] = from_float<T>(0.f);
    }
    __syncwarp();
    if (e >= 0) dlogits[row * A.ldd + e] = from_float<T>(d);
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
    m = warp_max(m);
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
      if (lane * S < E) {
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
    if (e >= 0) dlogits[row * A.ldd + e] = from_float<T>(v * (ds - dot));
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
  const bool groups = keep < G;
  // (the sum of two scores has no counterpart among the logits)
  const bool by_logits = !bias && !(groups && group_top == 2);
  RouteArgs A = {};
  A.rows = T, A.ld = ld, A.bias = bias, A.E = E, A.mode = mode, A.G = G, A.keep = keep;
  A.group_top = group_top, A.k = k, A.renorm = renorm, A.by_logits = by_logits;
  A.factor = factor, A.idx = idx, A.load = load, A.weight = weight;
  A.team = power_of_two(k);
  A.width = 32 / power_of_two(G);
  return with_dtype(dtype, [&](auto tag) {
    using X = decltype(tag);
    return with_slots(E, [&](auto slots) {
      constexpr int S = decltype(slots)::value;
      A.vec = vectors(logits, ld, E, S, sizeof(X));
      A.whole = E / G % S == 0;
      const size_t smem = (size_t)E * 4 * (groups && !A.whole ? 1 + kWarps : 1);
      const long long all = (T + kWarps - 1) / kWarps;
      auto go = [&](auto key, auto list) {
        using K = decltype(key);
        // a few queries whose load is wanted: one block, which writes it itself
        const unsigned grid =
            load && all <= 4 ? 1u : (unsigned)std::min<long long>(all, (S > 8 ? 4ll : kBlocks<S, K>) *
                                                                           num_sms());
        if (load && grid > 1) {
          if (int r = launch_cluster(clear_load_kernel, 1, 256, 1, 0, s, load, E)) return r;
        }
        auto kernel = route_kernel<X, S, K, decltype(list)::value>;
        return launch_cluster(kernel, grid, kThreads, 1, smem, s, (const X *)logits, A);
      };
      // (lists of the k best at least; shorter ones take fewer steps)
      constexpr int kShort = S < 4 ? S : 4;
      if constexpr (sizeof(X) == 2 && S <= 8)
        if (by_logits && !groups)
          return k <= kShort ? go(0u, std::integral_constant<int, kShort>{})
                             : go(0u, std::integral_constant<int, S>{});
      return k <= kShort ? go(0.f, std::integral_constant<int, kShort>{})
                         : go(0.f, std::integral_constant<int, S>{});
    });
  });
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
      const int team = power_of_two(k);
      A.vec = (uintptr_t)dlogits % 16 == 0 && (size_t)E * sizeof(X) % 16 == 0;
      const long long all = (T + kWarps * (32 / team) - 1) / (kWarps * (32 / team));
      const unsigned grid = (unsigned)std::min<long long>(all, 8ll * num_sms());
      return launch_cluster(route_grad_chosen_kernel<X>, grid, kThreads, 1, 0, s, (const X *)logits, A,
                            (X *)dlogits, team);
    }
    return with_slots(E, [&](auto slots) {
      constexpr int S = decltype(slots)::value;
      A.vec = vectors(logits, ld, E, S, sizeof(X)) && vectors(dlogits, ldd, E, S, sizeof(X));
      const unsigned grid = (unsigned)std::min<long long>((T + kWarps - 1) / kWarps, 8ll * num_sms());
      return launch_cluster(route_grad_softmax_kernel<X, S>, grid, kThreads, 1, 0, s,
                            (const X *)logits, A, (X *)dlogits);
    });
  });
}
