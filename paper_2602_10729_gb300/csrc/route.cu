// Routing of queries to experts: scores, the choice within the best groups,
// the weights and the load; and the gradient of the weights.
#include <math.h>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kWarps = 4;
constexpr unsigned kAll = 0xffffffffu;

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(kAll, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
__device__ __forceinline__ unsigned long long warp_max64(unsigned long long v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    const unsigned long long y = shfl_xor64(v, o);
    v = y > v ? y : v;
  }
  return v;
}

// exp(x - m) / sum, or the logistic function with its IEEE quotient.
__device__ __forceinline__ float score(float x, int mode, float m, float sum) {
  return mode == BOUTE_ROUTE_SIGMOID ? 1.f / (1.f + expf(-x)) : expf(x - m) / sum;
}

// The softmax's maximum and sum of a row (0 and 1 where there is nothing); bad: the row holds a
// NaN, or +inf with softmax.
template <class T>
__device__ __forceinline__ void row_stats(const T *x, int E, int mode, float &m, float &sum,
                                          bool &bad) {
  const int lane = threadIdx.x & 31;
  m = -INFINITY;
  sum = 0.f;
  bool b = false;
  for (int e = lane; e < E; e += 32) {
    const float v = to_float(x[e]);
    b |= isnan(v) || (mode == BOUTE_ROUTE_SOFTMAX && v == INFINITY);
    m = fmaxf(m, v);
  }
  bad = __any_sync(kAll, b);
  m = warp_max(m);
  if (mode == BOUTE_ROUTE_SIGMOID || bad || m == -INFINITY) {
    m = 0.f;
    sum = 1.f;
    return;
  }
  for (int e = lane; e < E; e += 32) sum += expf(to_float(x[e]) - m);
  sum = warp_sum(sum);
}

// A warp per query; its experts' c in shared memory.
template <class T>
__global__ void __launch_bounds__(32 * kWarps)
    route_kernel(const T *logits, long long rows, int E, long long ld, const float *bias,
                 int mode, int G, int keep, int group_top, int k, int renorm, float factor,
                 int *idx, float *weight, int *load) {
  extern __shared__ float smem[];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long row = (long long)blockIdx.x * kWarps + warp;
  if (row >= rows) return;
  float *c = smem + warp * E;
  const T *x = logits + row * ld;
  float m, sum;
  bool bad;
  row_stats(x, E, mode, m, sum, bad);
  for (int e = lane; e < E; e += 32) {
    const float v = to_float(x[e]);
    float ce = score(v, mode, m, sum);
    if (bias) ce += bias[e];
    c[e] = bad || v == -INFINITY || isnan(ce) ? -INFINITY : ce;
  }
  __syncwarp();
  // the groups that stay, a bit each
  const int per = E / G;
  unsigned kept = kAll;
  if (keep < G) {
    float a = -INFINITY, b = -INFINITY;
    for (int e = lane * per; lane < G && e < (lane + 1) * per; ++e) {
      const float v = c[e];
      if (v > a) b = a, a = v;
      else if (v > b) b = v;
    }
    const float g = group_top == 2 && b > -INFINITY ? a + b : a;
    unsigned long long key = lane < G && g > -INFINITY ? make_key(g, lane) : 0ull;
    kept = 0u;
    for (int r = 0; r < keep; ++r) {
      const unsigned long long best = warp_max64(key);
      if (best == 0ull) break;
      kept |= 1u << key_index(best);
      if (key == best) key = 0ull;
    }
  }
  unsigned long long last = ~0ull;
  float S = 0.f, mine = 0.f;
  int chosen = -1;
  for (int r = 0; r < k; ++r) {
    unsigned long long best = 0ull;
    for (int e = lane; e < E; e += 32) {
      const unsigned long long key = make_key(c[e], e);
      if (c[e] > -INFINITY && (kept >> (e / per) & 1u) && key < last && key > best) best = key;
    }
    best = warp_max64(best);
    if (best == 0ull) break;
    const int e = key_index(best);
    const float s = score(to_float(x[e]), mode, m, sum);
    S += s;
    if (lane == r) chosen = e, mine = s;
    last = best;
  }
  if (lane < k) {
    if (renorm) mine = S > 0.f ? mine / S : 0.f;
    idx[row * k + lane] = chosen;
    weight[row * k + lane] = bad ? NAN : factor * mine;
    if (load && chosen >= 0 && BOUTE_INB(chosen, E)) atomicAdd(load + chosen, 1);
  }
}

template <class T>
__global__ void __launch_bounds__(32 * kWarps)
    route_grad_kernel(const T *logits, long long rows, int E, long long ld, int mode, int k,
                      int renorm, float factor, const int *idx, const float *g_weight, T *dlogits,
                      long long ldd) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long row = (long long)blockIdx.x * kWarps + warp;
  if (row >= rows) return;
  const T *x = logits + row * ld;
  T *dx = dlogits + row * ldd;
  float m, sum;
  bool bad;
  row_stats(x, E, mode, m, sum, bad);
  int chosen = lane < k ? idx[row * k + lane] : -1;
  if (chosen >= E) chosen = -1;
  const bool on = chosen >= 0;
  const bool any = __any_sync(kAll, on);
  const float s = on ? score(to_float(x[chosen]), mode, m, sum) : 0.f;
  float ds = on ? factor * g_weight[row * k + lane] : 0.f;
  if (renorm) {
    const float S = warp_sum(s), gs = warp_sum(ds * s);
    ds = on && S > 0.f ? (ds - gs / S) / S : 0.f;
  }
  const float dot = mode == BOUTE_ROUTE_SOFTMAX ? warp_sum(ds * s) : 0.f;
  for (int e0 = 0; e0 < E; e0 += 32) {
    const int e = e0 + lane;
    float d = 0.f;
    for (int r = 0; r < k; ++r) {
      const int i = __shfl_sync(kAll, chosen, r);
      const float v = __shfl_sync(kAll, ds, r);
      if (i == e) d += v;
    }
    if (e >= E) continue;
    const float v = to_float(x[e]);
    float out = 0.f;
    if (any && mode == BOUTE_ROUTE_SOFTMAX) out = score(v, mode, m, sum) * (d - dot);
    if (any && mode == BOUTE_ROUTE_SIGMOID && d != 0.f) {
      const float q = expf(-fabsf(v));  // s (1 - s) without the difference
      out = d * q / ((1.f + q) * (1.f + q));
    }
    dx[e] = from_float<T>(out);
  }
}

}  // namespace

BOUTE_BOUNDS_READER(route)

}  // namespace boute

using namespace boute;

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
  if (load && cudaMemsetAsync(load, 0, E * sizeof(int), s) != cudaSuccess)
    return last_launch_status();
  if (T == 0) return BOUTE_OK;
  return with_dtype(dtype, [&](auto tag) {
    using X = decltype(tag);
    route_kernel<X><<<(unsigned)((T + kWarps - 1) / kWarps), 32 * kWarps,
                      kWarps * E * sizeof(float), s>>>((const X *)logits, T, E, ld, bias, mode, G,
                                                       keep, group_top, k, renorm, factor, idx,
                                                       weight, load);
    count_launch();
    return last_launch_status();
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
  return with_dtype(dtype, [&](auto tag) {
    using X = decltype(tag);
    route_grad_kernel<X><<<(unsigned)((T + kWarps - 1) / kWarps), 32 * kWarps, 0,
                           (cudaStream_t)stream>>>((const X *)logits, T, E, ld, mode, k, renorm,
                                                   factor, idx, g_weight, (X *)dlogits, ldd);
    count_launch();
    return last_launch_status();
  });
}
