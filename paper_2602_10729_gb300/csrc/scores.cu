// The scores of answers (mean and lowest log-probability, mean and highest
// entropy of the positions that hold a token) and their gradient.
#include <math.h>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kThreads = 256;

// Order-preserving bits of a float, -0 as +0, a NaN above every number.
__device__ __forceinline__ unsigned order_bits(float v) {
  if (isnan(v)) return 0xffffffffu;
  if (v == 0.f) v = 0.f;
  const unsigned u = __float_as_uint(v);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// An answer's positions within [0, T].
__device__ __forceinline__ void answer_range(const long long *offsets, long long q, long long T,
                                             long long &a, long long &b) {
  a = offsets[q];
  b = offsets[q + 1];
  a = a < 0 ? 0 : a > T ? T : a;
  b = b < a ? a : b > T ? T : b;
}

// What an answer's scores are made of. lo, hi: order_bits of -logprob and of the entropy with
// the complement of the position below, so that a maximum is the extreme's first position.
struct Part {
  float lp, ent;
  int n;
  unsigned long long lo, hi;
};

__device__ __forceinline__ Part block_join(Part p, Part *red) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) {
    p.lp += __shfl_xor_sync(0xffffffffu, p.lp, o);
    p.ent += __shfl_xor_sync(0xffffffffu, p.ent, o);
    p.n += __shfl_xor_sync(0xffffffffu, p.n, o);
    p.lo = max(p.lo, shfl_xor64(p.lo, o));
    p.hi = max(p.hi, shfl_xor64(p.hi, o));
  }
  if (lane == 0) red[warp] = p;
  __syncthreads();
  p = red[0];
  for (int w = 1; w < kThreads / 32; ++w) {
    p.lp += red[w].lp;
    p.ent += red[w].ent;
    p.n += red[w].n;
    p.lo = max(p.lo, red[w].lo);
    p.hi = max(p.hi, red[w].hi);
  }
  return p;
}

// (positions from the answer's first; an answer of 2^31 positions at most)
__device__ __forceinline__ Part answer_parts(const float *logprob, const float *entropy,
                                             const long long *targets, long long a, long long b,
                                             Part *red) {
  Part p = {0.f, 0.f, 0, 0ull, 0ull};
  for (long long t = a + threadIdx.x; t < b; t += kThreads) {
    if (targets && targets[t] < 0) continue;
    const float l = logprob[t], h = entropy[t];
    const unsigned at = 0xffffffffu - (unsigned)(t - a);
    p.lp += l;
    p.ent += h;
    p.n += 1;
    p.lo = max(p.lo, ((unsigned long long)order_bits(-l) << 32) | at);
    p.hi = max(p.hi, ((unsigned long long)order_bits(h) << 32) | at);
  }
  return block_join(p, red);
}

__device__ __forceinline__ long long position(unsigned long long key, long long a) {
  return a + (long long)(0xffffffffu - (unsigned)key);
}

__global__ void __launch_bounds__(kThreads)
    answer_scores_kernel(const float *logprob, const float *entropy, const long long *targets,
                         const long long *offsets, long long T, float *scores, int *counts) {
  __shared__ Part red[kThreads / 32];
  const long long q = blockIdx.x;
  long long a, b;
  answer_range(offsets, q, T, a, b);
  const Part p = answer_parts(logprob, entropy, targets, a, b, red);
  if (threadIdx.x == 0) {
    counts[q] = p.n;
    scores[4 * q] = p.n ? p.lp / p.n : 0.f;
    scores[4 * q + 1] = p.n ? logprob[position(p.lo, a)] : 0.f;
    scores[4 * q + 2] = p.n ? p.ent / p.n : 0.f;
    scores[4 * q + 3] = p.n ? entropy[position(p.hi, a)] : 0.f;
  }
}

__global__ void __launch_bounds__(kThreads)
    answer_scores_grad_kernel(const float *logprob, const float *entropy,
                              const long long *targets, const long long *offsets, long long T,
                              long long Q, const float *g_scores, float *g_logprob,
                              float *g_entropy) {
  __shared__ Part red[kThreads / 32];
  const long long q = blockIdx.x;
  long long a, b;
  answer_range(offsets, q, T, a, b);
  const Part p = answer_parts(logprob, entropy, targets, a, b, red);
  const float n = p.n ? (float)p.n : 1.f;
  const float *g = g_scores + 4 * q;
  const float g0 = g[0] / n, g2 = g[2] / n;
  for (long long t = a + threadIdx.x; t < b; t += kThreads) {
    const bool on = !targets || targets[t] >= 0;
    g_logprob[t] = on ? g0 + (t == position(p.lo, a) ? g[1] : 0.f) : 0.f;
    g_entropy[t] = on ? g2 + (t == position(p.hi, a) ? g[3] : 0.f) : 0.f;
  }
  // positions before the first answer and after the last
  const long long end = q == Q - 1 ? T : b, from = q == 0 ? 0 : a;
  for (long long t = from + threadIdx.x; t < end; t += kThreads)
    if (t < a || t >= b) g_logprob[t] = g_entropy[t] = 0.f;
}

}  // namespace

BOUTE_BOUNDS_READER(scores)

}  // namespace boute

using namespace boute;

static int sizes_ok(long long T, long long Q, const float *logprob, const float *entropy,
                    const long long *targets, const long long *offsets) {
  if (T < 0 || Q < 0 || (Q > 0 && !array_ok(offsets, 8)) ||
      (T > 0 && (!array_ok(logprob, 4) || !array_ok(entropy, 4))) || !optional_ok(targets, 8))
    return BOUTE_ERR_INVALID_ARG;
  return T >= (1ll << 31) || Q >= (1ll << 31) ? BOUTE_ERR_UNSUPPORTED : device_ok();
}

extern "C" int boute_answer_scores(const float *logprob, const float *entropy,
                                   const long long *targets, const long long *offsets,
                                   long long T, long long Q, float *scores, int *counts,
                                   void *stream) {
  BOUTE_TRACE();
  if (Q > 0 && (!array_ok(scores, 4) || !array_ok(counts, 4))) return BOUTE_ERR_INVALID_ARG;
  if (int r = sizes_ok(T, Q, logprob, entropy, targets, offsets)) return r;
  if (Q == 0) return BOUTE_OK;
  answer_scores_kernel<<<(unsigned)Q, kThreads, 0, (cudaStream_t)stream>>>(
      logprob, entropy, targets, offsets, T, scores, counts);
  count_launch();
  return last_launch_status();
}

extern "C" int boute_answer_scores_grad(const float *logprob, const float *entropy,
                                        const long long *targets, const long long *offsets,
                                        long long T, long long Q, const float *g_scores,
                                        float *g_logprob, float *g_entropy, void *stream) {
  BOUTE_TRACE();
  if ((Q > 0 && !array_ok(g_scores, 4)) ||
      (T > 0 && (!array_ok(g_logprob, 4) || !array_ok(g_entropy, 4))))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = sizes_ok(T, Q, logprob, entropy, targets, offsets)) return r;
  if (T == 0) return BOUTE_OK;
  if (Q == 0) {
    if (cudaMemsetAsync(g_logprob, 0, T * sizeof(float), (cudaStream_t)stream) != cudaSuccess ||
        cudaMemsetAsync(g_entropy, 0, T * sizeof(float), (cudaStream_t)stream) != cudaSuccess)
      return last_launch_status();
    return BOUTE_OK;
  }
  answer_scores_grad_kernel<<<(unsigned)Q, kThreads, 0, (cudaStream_t)stream>>>(
      logprob, entropy, targets, offsets, T, Q, g_scores, g_logprob, g_entropy);
  count_launch();
  return last_launch_status();
}
