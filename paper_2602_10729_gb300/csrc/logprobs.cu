// Log-probabilities of given tokens, with the entropy and the top alternatives
// of every position, and the gradient with respect to the logits.
//
// With z = scale x, m = max z, s = sum exp(z - m) and u = sum (z - m) exp(z - m):
//   lse = m + ln s,  logprob = z_t - m - ln s,  entropy = ln s - u / s.
#include <math.h>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kThreads = 512;
constexpr float kLowest = -200.f;  // exp(kLowest) = 0 in fp32

__device__ __forceinline__ float warp_max(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
  return v;
}
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// A row per block, three passes: maximum, sums, and one pass per alternative.
template <class T>
__global__ void __launch_bounds__(kThreads)
    token_logprobs_kernel(const T *logits, int V, long long ld, const long long *targets,
                          float scale, int k, float *logprob, float *entropy, float *lse,
                          long long *top_idx, float *top_logprob) {
  __shared__ float red[kThreads / 32][2];
  __shared__ unsigned long long best[kThreads / 32];
  __shared__ float stat[3];
  const long long row = blockIdx.x;
  const T *x = logits + row * ld;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  float m = -INFINITY;
  bool bad = false;
  for (int j = tid; j < V; j += kThreads) {
    const float z = __fmul_rn(to_float(x[j]), scale);
    bad |= !(z < INFINITY);
    m = fmaxf(m, z);
  }
  m = warp_max(m);
  bad = __syncthreads_or(bad);
  if (lane == 0) red[warp][0] = m;
  __syncthreads();
  if (warp == 0) {
    m = warp_max(lane < kThreads / 32 ? red[lane][0] : -INFINITY);
    if (lane == 0) stat[0] = m;
  }
  __syncthreads();
  m = stat[0];
  float s = 0.f, u = 0.f;
  if (!bad && m > -INFINITY)
    for (int j = tid; j < V; j += kThreads) {
      const float d = fmaxf(__fmul_rn(to_float(x[j]), scale) - m, kLowest);
      const float e = expf(d);
      s += e;
      u = fmaf(d, e, u);
    }
  s = warp_sum(s);
  u = warp_sum(u);
  if (lane == 0) red[warp][0] = s, red[warp][1] = u;
  __syncthreads();
  if (tid == 0) {
    s = u = 0.f;
    for (int w = 0; w < kThreads / 32; ++w) s += red[w][0], u += red[w][1];
    const bool empty = m == -INFINITY;
    const float ls = empty ? 0.f : logf(s);
    const long long t = targets[row];
    float lp = 0.f;
    if (t >= V) lp = NAN;
    else if (t >= 0 && BOUTE_INB(t, V))
      lp = empty ? -INFINITY : __fmul_rn(to_float(x[t]), scale) - m - ls;
    lse[row] = bad ? NAN : m + ls;
    logprob[row] = bad && t >= 0 ? NAN : lp;
    entropy[row] = bad ? NAN : empty ? 0.f : ls - u / s;
    stat[1] = ls;
  }
  __syncthreads();
  const float ls = stat[1];
  unsigned long long last = ~0ull;
  for (int r = 0; r < k; ++r) {
    unsigned long long b = 0ull;
    for (int j = tid; j < V; j += kThreads) {
      const float z = __fmul_rn(to_float(x[j]), scale);
      const unsigned long long key = make_key(z, (unsigned)j);
      if (z > -INFINITY && key < last && key > b) b = key;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      const unsigned long long y = shfl_xor64(b, o);
      b = y > b ? y : b;
    }
    if (lane == 0) best[warp] = b;
    __syncthreads();
    for (int w = 0; w < kThreads / 32; ++w) b = best[w] > b ? best[w] : b;
    __syncthreads();
    if (tid == 0) {
      const unsigned j = key_index(b);
      const bool none = b == 0ull || bad;
      top_idx[row * k + r] = none ? -1 : (long long)j;
      top_logprob[row * k + r] =
          bad ? NAN : none ? -INFINITY : __fmul_rn(to_float(x[j]), scale) - m - ls;
    }
    last = b;
  }
}

// Beyond this |lse| its rounding (2^-24 of it) would show in p: rows whose mask is the type's
// lowest value throughout have an lse that has lost ln s, and take m and ln s from the row.
constexpr float kLargeLse = 1024.f;

template <class T>
__global__ void __launch_bounds__(kThreads)
    token_logprobs_grad_kernel(const T *logits, int V, long long ld, const long long *targets,
                               float scale, const float *lse, const float *entropy,
                               const float *g_logprob, const float *g_entropy, T *dlogits,
                               long long ldd) {
  __shared__ float red[kThreads / 32];
  const long long row = blockIdx.x;
  const T *x = logits + row * ld;
  T *dx = dlogits + row * ldd;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const long long t = targets[row];
  const float l = lse[row];
  const float g = t < 0 ? 0.f : t >= V ? NAN : g_logprob[row];
  const float gh = g_entropy ? g_entropy[row] : 0.f, H = g_entropy ? entropy[row] : 0.f;
  float m = l, ls = 0.f;  // lse = m + ls
  if (fabsf(l) > kLargeLse && isfinite(l)) {
    m = -INFINITY;
    for (int j = tid; j < V; j += kThreads) m = fmaxf(m, __fmul_rn(to_float(x[j]), scale));
    m = warp_max(m);
    if (lane == 0) red[warp] = m;
    __syncthreads();
    for (int w = 0; w < kThreads / 32; ++w) m = fmaxf(m, red[w]);
    __syncthreads();
    float s = 0.f;
    for (int j = tid; j < V; j += kThreads)
      s += expf(fmaxf(__fmul_rn(to_float(x[j]), scale) - m, kLowest));
    s = warp_sum(s);
    if (lane == 0) red[warp] = s;
    __syncthreads();
    s = 0.f;
    for (int w = 0; w < kThreads / 32; ++w) s += red[w];
    ls = logf(s);
  }
  for (int j = tid; j < V; j += kThreads) {
    const float lp = fmaxf(fmaf(to_float(x[j]), scale, -m) - ls, kLowest);
    const float p = expf(lp);
    float d = -p * (g + gh * (lp + H));
    if (j == t) d += g;
    dx[j] = from_float<T>(l == -INFINITY && t < V ? 0.f : l != l ? NAN : d * scale);
  }
}

}  // namespace

BOUTE_BOUNDS_READER(logprobs)

}  // namespace boute

using namespace boute;

static bool logits_ok(const void *logits, int dtype, long long T, int V, long long ld,
                      const long long *targets, float scale) {
  return dtype_known(dtype) && T >= 0 && V >= 1 && ld >= V && scale > 0.f && isfinite(scale) &&
         (T == 0 || (array_ok(logits, dtype_bytes(dtype)) && array_ok(targets, 8)));
}

extern "C" int boute_token_logprobs(const void *logits, int dtype, long long T, int V,
                                    long long ld, const long long *targets, float scale, int k,
                                    float *logprob, float *entropy, float *lse,
                                    long long *top_idx, float *top_logprob, void *stream) {
  BOUTE_TRACE();
  if (!logits_ok(logits, dtype, T, V, ld, targets, scale) || k < 0 || k > V ||
      (T > 0 && (!array_ok(logprob, 4) || !array_ok(entropy, 4) || !array_ok(lse, 4) ||
                 (k > 0 && (!array_ok(top_idx, 8) || !array_ok(top_logprob, 4))))))
    return BOUTE_ERR_INVALID_ARG;
  if (T >= (1ll << 31) || V > BOUTE_MAX_VOCAB || k > BOUTE_MAX_ALTERNATIVES)
    return BOUTE_ERR_UNSUPPORTED;
  if (int r = device_ok()) return r;
  if (T == 0) return BOUTE_OK;
  return with_dtype(dtype, [&](auto tag) {
    using E = decltype(tag);
    token_logprobs_kernel<E><<<(unsigned)T, kThreads, 0, (cudaStream_t)stream>>>(
        (const E *)logits, V, ld, targets, scale, k, logprob, entropy, lse, top_idx, top_logprob);
    count_launch();
    return last_launch_status();
  });
}

extern "C" int boute_token_logprobs_grad(const void *logits, int dtype, long long T, int V,
                                         long long ld, const long long *targets, float scale,
                                         const float *lse, const float *entropy,
                                         const float *g_logprob, const float *g_entropy,
                                         void *dlogits, long long ldd, void *stream) {
  BOUTE_TRACE();
  if (!logits_ok(logits, dtype, T, V, ld, targets, scale) || ldd < V ||
      (T > 0 && (!array_ok(dlogits, dtype_bytes(dtype)) || !array_ok(lse, 4) ||
                 !array_ok(g_logprob, 4) || !optional_ok(g_entropy, 4) ||
                 (g_entropy && !array_ok(entropy, 4)))) ||
      (dlogits == logits && ldd != ld))
    return BOUTE_ERR_INVALID_ARG;
  if (T >= (1ll << 31) || V > BOUTE_MAX_VOCAB) return BOUTE_ERR_UNSUPPORTED;
  if (int r = device_ok()) return r;
  if (T == 0) return BOUTE_OK;
  return with_dtype(dtype, [&](auto tag) {
    using E = decltype(tag);
    token_logprobs_grad_kernel<E><<<(unsigned)T, kThreads, 0, (cudaStream_t)stream>>>(
        (const E *)logits, V, ld, targets, scale, lse, entropy, g_logprob, g_entropy,
        (E *)dlogits, ldd);
    count_launch();
    return last_launch_status();
  });
}
