// Routing of queries to experts: scores, the choice within the best groups,
// the weights and the load; and the gradient of the weights.
//
// A warp per query, lane l with the S experts l S .. l S + S - 1 (S a power of two,
// 32 S >= E), so that the lowest lane has the lowest indices. Each lane sorts
// its S values; k rounds then take the largest head of the 32 lists (one
// reduction each). Without a bias the logits themselves are compared, which have
// the order of the scores: only the chosen scores are computed then, and a softmax's
// sum only where the weights are not renormalised. 16-bit logits carry their
// expert's index in the key's lower half.
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

__device__ __forceinline__ float logistic(float x) {  // (0 where exp(-x) overflows, as in fp32)
  return __fdividef(1.f, 1.f + fminf(exp2_fast(-x * kLog2e), 3e38f));
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

// v in descending order (Batcher's odd-even merge sort).
template <int S, class K>
__device__ __forceinline__ void sort_desc(K (&v)[S]) {
#pragma unroll
  for (int p = 1; p < S; p *= 2)
#pragma unroll
    for (int q = p; q > 0; q /= 2)
#pragma unroll
      for (int j = q % p; j + q < S; j += 2 * q)
#pragma unroll
        for (int i = 0; i < q; ++i)
          if (i + j + q < S && (i + j) / (2 * p) == (i + j + q) / (2 * p)) {
            const K a = v[i + j], b = v[i + j + q];
            v[i + j] = max(a, b);
            v[i + j + q] = min(a, b);
          }
}

// The k largest of the lanes' values, lane r with the r-th: its value and its expert (-1: none).
// Keys are unique and carry the expert; equal floats go to the lowest expert: of several lanes
// the lowest, of one lane's the occurrences in order.
template <int S>
__device__ __forceinline__ void choose(const unsigned (&c)[S], int k, unsigned &mine, int &expert) {
  const int lane = threadIdx.x & 31;
  unsigned v[S];
#pragma unroll
  for (int s = 0; s < S; ++s) v[s] = c[s];
  sort_desc(v);
  mine = 0u;
  for (int r = 0; r < k; ++r) {
    const unsigned b = warp_max(v[0]);
    if (lane == r) mine = b;
    if (v[0] == b) {
#pragma unroll
      for (int s = 0; s + 1 < S; ++s) v[s] = v[s + 1];
      v[S - 1] = 0u;
    }
  }
  expert = mine ? (int)(0xffffu - (mine & 0xffffu)) : -1;
}
template <int S>
__device__ __forceinline__ void choose(const float (&c)[S], int k, float &mine, int &expert) {
  const int lane = threadIdx.x & 31;
  float v[S];
#pragma unroll
  for (int s = 0; s < S; ++s) v[s] = c[s];
  sort_desc(v);
  mine = -INFINITY;
  int owner = 0;
  for (int r = 0; r < k; ++r) {
    const float b = warp_max(v[0]);
    if (b == -INFINITY) break;
    const int from = __ffs(__ballot_sync(kAll, v[0] == b)) - 1;
    if (lane == r) {
      mine = b;
      owner = from;
    }
    if (lane == from) {
#pragma unroll
      for (int s = 0; s + 1 < S; ++s) v[s] = v[s + 1];
      v[S - 1] = -INFINITY;
    }
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

// Bits of the `keep` groups with the largest scores, from the queries' c in shared memory; 2^q
// lanes to a group.
__device__ __forceinline__ unsigned keep_groups(const float *c, int G, int per, int keep,
                                                int group_top) {
  const int lane = threadIdx.x & 31;
  int width = 32;
  while (width * G > 32) width /= 2;
  const int g = lane / width;
  float a = -INFINITY, b = -INFINITY;  // the two largest
  if (g < G)
    for (int i = lane % width; i < per; i += width) {
      const float v = c[g * per + i];
      b = fmaxf(b, fminf(a, v));
      a = fmaxf(a, v);
    }
  for (int o = 1; o < width; o *= 2) {
    const float a2 = __shfl_xor_sync(kAll, a, o), b2 = __shfl_xor_sync(kAll, b, o);
    b = fmaxf(fminf(a, a2), fmaxf(b, b2));
    a = fmaxf(a, a2);
  }
  const float mine = group_top == 2 && b > -INFINITY ? a + b : a;
  int rank = 0;
  for (int h = 0; h < G; ++h) {
    const float other = __shfl_sync(kAll, mine, h * width);
    rank += other > mine || (other == mine && h < g);
  }
  const unsigned in = __ballot_sync(kAll, g < G && rank < keep && mine > -INFINITY);
  unsigned kept = 0u;
  for (int h = 0; h < G; ++h) kept |= (in >> (h * width) & 1u) << h;
  return kept;
}

struct RouteArgs {
  long long rows, ld;
  const float *bias;
  int E, mode, G, keep, group_top, k, renorm, by_logits, vec;
  float factor;
  int *idx, *load;
  float *weight;
};

// K: unsigned for 16-bit logits compared as they are, float else (by_logits: the logits, else the
// scores with their bias).
template <class T, int S, class K>
__global__ void __launch_bounds__(kThreads) route_kernel(const T *logits, RouteArgs A) {
  extern __shared__ int hist[];  // the block's load; then, with groups, c of each warp's query
  constexpr bool kKeys = std::is_same<K, unsigned>::value;
  const bool by_logits = kKeys || A.by_logits, groups = A.keep < A.G;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, E = A.E, k = A.k;
  const bool soft = A.mode == BOUTE_ROUTE_SOFTMAX;
  float *shared_c = (float *)(hist + E) + warp * E;
  if (A.load) {
    for (int e = threadIdx.x; e < E; e += kThreads) hist[e] = 0;
    __syncthreads();
  }
  float bias[kKeys ? 1 : S];
  if constexpr (!kKeys)
#pragma unroll
    for (int s = 0; s < S; ++s)
      bias[s] = A.bias && lane * S + s < E ? A.bias[lane * S + s] : 0.f;
  const long long step = (long long)gridDim.x * kWarps;
  long long row = (long long)blockIdx.x * kWarps + warp;
  Raw<T, S> next;
  if (row < A.rows) next.load(logits + row * A.ld, E, A.vec);
  for (; row < A.rows; row += step) {
    const Raw<T, S> raw = next;
    if (row + step < A.rows) next.load(logits + (row + step) * A.ld, E, A.vec);
    float x[S], m = -INFINITY;
#pragma unroll
    for (int s = 0; s < S; ++s) {
      x[s] = to_float(raw.at(s));
      m = max_nan(m, x[s]);
    }
    m = warp_max(m);
    const bool bad = isnan(m) || (soft && m == INFINITY);
    float inv_sum = 0.f;  // of the softmax
    if (soft && (!by_logits || !A.renorm)) {
      float sum = 0.f;
#pragma unroll
      for (int s = 0; s < S; ++s) sum += exp2_fast((x[s] - m) * kLog2e);
      inv_sum = __fdividef(1.f, warp_sum(sum));
    }
    K c[S];
#pragma unroll
    for (int s = 0; s < S; ++s) {
      if constexpr (kKeys) {  // upper half of order bits, expert
        unsigned u = __float_as_uint(x[s] == 0.f ? 0.f : x[s]);
        if constexpr (std::is_same<T, __half>::value) {  // (fp16 as its own bits)
          const __half h = x[s] == 0.f ? __float2half_rn(0.f) : raw.at(s);
          unsigned short q;
          memcpy(&q, &h, 2);
          u = (unsigned)q << 16;
        }
        u = (u & 0x80000000u) ? ~u : (u | 0x80000000u);
        c[s] = x[s] > -INFINITY && !bad ? (u & 0xffff0000u) | (0xffffu - (lane * S + s)) : 0u;
      } else if (by_logits) {
        c[s] = bad ? -INFINITY : x[s];
      } else {
        const float v = soft ? exp2_fast((x[s] - m) * kLog2e) * inv_sum : logistic(x[s]);
        // (fmaxf: no NaN of the bias)
        c[s] = x[s] > -INFINITY && !bad ? fmaxf(v + bias[s], -INFINITY) : -INFINITY;
      }
    }
    if (groups) {
      const int per = E / A.G;
#pragma unroll
      for (int s = 0; s < S; ++s)
        if (lane * S + s < E) {
          if constexpr (kKeys) shared_c[lane * S + s] = bad ? -INFINITY : x[s];
          else shared_c[lane * S + s] = c[s];
        }
      __syncwarp();
      const unsigned kept = keep_groups(shared_c, A.G, per, A.keep, A.group_top);
      __syncwarp();
      // (the lane's experts are neighbours: one division, then steps)
      int g = lane * S / per, left = (g + 1) * per - lane * S;
#pragma unroll
      for (int s = 0; s < S; ++s) {
        if (left-- == 0) {
          ++g;
          left = per - 1;
        }
        if (!(kept >> (g & 31) & 1u)) c[s] = key_none(K{});
      }
    }
    K mine;
    int e;
    choose(c, k, mine, e);
    // the chosen scores
    float v = 0.f;
    if (e >= 0) {
      const float xe = to_float(logits[row * A.ld + e]);
      v = !soft ? logistic(xe) : exp2_fast((xe - m) * kLog2e) * (inv_sum > 0.f ? inv_sum : 1.f);
    }
    if (A.renorm) {
      const float sum = warp_sum(v);
      v = sum > 0.f ? v / sum : 0.f;
    }
    if (lane < k) {
      A.idx[row * k + lane] = e;
      A.weight[row * k + lane] = bad ? NAN : A.factor * v;
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

// ds for this lane's choice of its query, in teams of `team` lanes (a power of two >= k) with a
// query each: v the chosen score (or anything proportional to it, with renorm), g its gradient.
__device__ __forceinline__ float team_sum(float v, int team) {
  for (int o = team / 2; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}

// The gradient where it is 0 but for the chosen experts: logistic scores, and a renormalised
// softmax, of which only the chosen logits count:
//   w_i = factor s_i / S:  dx_i = factor s_i / S (g_i - sum_j g_j s_j / S) [ (1 - s_i): logistic ].
// 32 / team queries to a warp: the chosen logits are gathered, the rows cleared, the gradients put
// in.
template <class T>
__global__ void __launch_bounds__(kThreads)
    route_grad_chosen_kernel(const T *logits, RouteGradArgs A, T *dlogits, int team) {
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
  RouteArgs A = {T,         ld, bias,   E,   mode, G,   keep, group_top, k, renorm,
                 by_logits, 0,  factor, idx, load, weight};
  return with_dtype(dtype, [&](auto tag) {
    using X = decltype(tag);
    return with_slots(E, [&](auto slots) {
      constexpr int S = decltype(slots)::value;
      A.vec = vectors(logits, ld, E, S, sizeof(X));
      const size_t smem = (size_t)E * 4 * (groups ? 1 + kWarps : 1);
      const long long all = (T + kWarps - 1) / kWarps;
      // a few queries: one block, which writes the load itself
      const unsigned grid = all <= 4 ? 1u : (unsigned)std::min<long long>(all, 4ll * num_sms());
      if (load && grid > 1) {
        clear_load_kernel<<<1, 256, 0, s>>>(load, E);
        count_launch();
      }
      auto go = [&](auto key) {
        auto kernel = route_kernel<X, S, decltype(key)>;
        if (load && grid > 1)
          launch_pdl(kernel, dim3(grid), dim3(kThreads), smem, s, (const X *)logits, A);
        else
          kernel<<<grid, kThreads, smem, s>>>((const X *)logits, A);
        count_launch();
        return last_launch_status();
      };
      if constexpr (sizeof(X) == 2 && S <= 8)
        if (A.by_logits) return go(0u);
      return go(0.f);
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
      int team = 1;
      while (team < k) team *= 2;
      A.vec = (uintptr_t)dlogits % 16 == 0 && (size_t)E * sizeof(X) % 16 == 0;
      const long long all = (T + kWarps * (32 / team) - 1) / (kWarps * (32 / team));
      const unsigned grid = (unsigned)std::min<long long>(all, 8ll * num_sms());
      route_grad_chosen_kernel<X><<<grid, kThreads, 0, s>>>((const X *)logits, A, (X *)dlogits,
                                                            team);
      count_launch();
      return last_launch_status();
    }
    return with_slots(E, [&](auto slots) {
      constexpr int S = decltype(slots)::value;
      A.vec = vectors(logits, ld, E, S, sizeof(X)) && vectors(dlogits, ldd, E, S, sizeof(X));
      const unsigned grid = (unsigned)std::min<long long>((T + kWarps - 1) / kWarps, 8ll * num_sms());
      route_grad_softmax_kernel<X, S><<<grid, kThreads, 0, s>>>((const X *)logits, A,
                                                                (X *)dlogits);
      count_launch();
      return last_launch_status();
    });
  });
}
