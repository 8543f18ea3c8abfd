// The scores of answers (mean and lowest log-probability, mean and highest
// entropy of the positions that hold a token) and their gradient.
#include <math.h>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kCluster = 8;
constexpr int kTeamLane = 32;  // positions a lane of a team takes at most
constexpr int kUnroll = 4;

// Order-preserving bits of a float, -0 as +0, a NaN above every number.
__device__ __forceinline__ unsigned order_bits(float v) {
  if (isnan(v)) return 0xffffffffu;
  if (v == 0.f) v = 0.f;
  const unsigned u = __float_as_uint(v);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}

// What an answer's scores are made of. lo, hi: order_bits of -logprob and of the entropy with
// the complement of the position below, so that a maximum is the extreme's first position.
struct Part {
  unsigned long long lo, hi;
  float lp, ent;
  int n, pad;
};

__device__ __forceinline__ void add(Part &p, const Part &o) {
  p.lp += o.lp;
  p.ent += o.ent;
  p.n += o.n;
  p.lo = max(p.lo, o.lo);
  p.hi = max(p.hi, o.hi);
}

struct Answers {
  const float *logprob, *entropy;
  const long long *targets, *offsets;
  long long T, Q;

  // an answer's positions within [0, T]
  __device__ __forceinline__ void range(long long q, long long &a, long long &b) const {
    a = offsets[q];
    b = offsets[q + 1];
    a = a < 0 ? 0 : a > T ? T : a;
    b = b < a ? a : b > T ? T : b;
  }
  // Thread i of `by` over the positions [a, b) (2^31 at most).
  __device__ __forceinline__ Part part(long long a, long long b, int i, int by) const {
    Part p = {0ull, 0ull, 0.f, 0.f, 0, 0};
    for (long long t0 = a + i; t0 < b; t0 += kUnroll * by) {
      float l[kUnroll], h[kUnroll];
      bool on[kUnroll];
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const long long t = t0 + u * by;
        on[u] = t < b;
        if (!on[u]) continue;
        l[u] = logprob[t];
        h[u] = entropy[t];
        if (targets) on[u] = targets[t] >= 0;
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (!on[u]) continue;
        const unsigned at = 0xffffffffu - (unsigned)(t0 + u * by - a);
        p.lp += l[u];
        p.ent += h[u];
        p.n += 1;
        p.lo = max(p.lo, ((unsigned long long)order_bits(-l[u]) << 32) | at);
        p.hi = max(p.hi, ((unsigned long long)order_bits(h[u]) << 32) | at);
      }
    }
    return p;
  }
};

__device__ __forceinline__ long long position(unsigned long long key, long long a) {
  return a + (long long)(0xffffffffu - (unsigned)key);
}

__device__ __forceinline__ Part warp_join(Part p) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    add(p, {shfl_xor64(p.lo, o), shfl_xor64(p.hi, o), __shfl_xor_sync(kAll, p.lp, o),
            __shfl_xor_sync(kAll, p.ent, o), __shfl_xor_sync(kAll, p.n, o), 0});
  return p;
}
// Of the whole block, in every thread; red (kWarps Parts) may be used again after a barrier.
__device__ __forceinline__ Part block_join(Part p, Part *red) {
  p = warp_join(p);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = p;
  __syncthreads();
  p = red[0];
  for (int w = 1; w < kWarps; ++w) add(p, red[w]);
  return p;
}
// Of the whole cluster, in every thread; a cluster barrier before the next call.
__device__ __forceinline__ Part cluster_join(Part p, int rank, Part *red, Part *parts) {
  p = block_join(p, red);
  if (threadIdx.x < kCluster) {
    const uint32_t to = peer(&parts[rank], threadIdx.x);
    store_peer(to, p.lo);
    store_peer(to + 8, p.hi);
    store_peer(to + 16, p.lp);
    store_peer(to + 20, p.ent);
    store_peer(to + 24, __int_as_float(p.n));
  }
  cluster_sync();
  p = parts[0];
  for (int r = 1; r < kCluster; ++r) add(p, parts[r]);
  return p;
}

// A cluster of 8 blocks takes `per` answers: one by all its threads (per = 1), one a block (8), or
// one a warp (64); answers too long for such a team (ragged lengths) by the whole cluster
// afterwards. emit(q, a, b, p, i, by): thread i of `by` writes its share of answer q's results.
template <class Emit>
__device__ __forceinline__ void for_answers(const Answers &A, int per, Emit emit) {
  __shared__ Part red[kWarps], parts[kCluster];
  const int rank = blockIdx.x % kCluster, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const long long q0 = (long long)(blockIdx.x / kCluster) * per;
  const long long most = (long long)kTeamLane * (per == 64 ? 32 : kThreads);
  long long a, b;
  if (per == 64) {
    const long long q = q0 + rank * kWarps + warp;
    if (q < A.Q) {
      A.range(q, a, b);
      if (b - a <= most) emit(q, a, b, warp_join(A.part(a, b, lane, 32)), lane, 32);
    }
  } else if (per == kCluster) {
    const long long q = q0 + rank;
    if (q < A.Q) {
      A.range(q, a, b);
      if (b - a <= most) {
        const Part p = block_join(A.part(a, b, threadIdx.x, kThreads), red);
        emit(q, a, b, p, (int)threadIdx.x, kThreads);
      }
    }
  }
  __syncthreads();
  for (int j0 = 0; j0 < per; j0 += 32) {
    long long n = 0;
    if (j0 + lane < per && q0 + j0 + lane < A.Q) {
      A.range(q0 + j0 + lane, a, b);
      n = b - a;
    }
    // (the same in all of the cluster's warps)
    unsigned left = __ballot_sync(kAll, per == 1 ? lane == 0 : n > most);
    while (left) {
      const long long q = q0 + j0 + __ffs(left) - 1;
      left &= left - 1;
      A.range(q, a, b);
      const int i = rank * kThreads + threadIdx.x, by = kCluster * kThreads;
      emit(q, a, b, cluster_join(A.part(a, b, i, by), rank, red, parts), i, by);
      cluster_sync();
    }
  }
}

__global__ void __launch_bounds__(kThreads)
    answer_scores_kernel(Answers A, int per, float *scores, int *counts) {
  for_answers(A, per, [&](long long q, long long a, long long b, const Part &p, int i, int by) {
    if (i != 0) return;
    counts[q] = p.n;
    const float n = (float)p.n;
    scores[4 * q] = p.n ? p.lp / n : 0.f;
    scores[4 * q + 1] = p.n ? A.logprob[position(p.lo, a)] : 0.f;
    scores[4 * q + 2] = p.n ? p.ent / n : 0.f;
    scores[4 * q + 3] = p.n ? A.entropy[position(p.hi, a)] : 0.f;
  });
}

__global__ void __launch_bounds__(kThreads)
    answer_scores_grad_kernel(Answers A, int per, const float *g_scores, float *g_logprob,
                              float *g_entropy) {
  for_answers(A, per, [&](long long q, long long a, long long b, const Part &p, int i, int by) {
    const float n = p.n ? (float)p.n : 1.f;
    const float *g = g_scores + 4 * q;
    const float g0 = g[0] / n, g1 = g[1], g2 = g[2] / n, g3 = g[3];
    const long long lo = position(p.lo, a), hi = position(p.hi, a);
#pragma unroll 4
    for (long long t = a + i; t < b; t += by) {
      const bool on = !A.targets || A.targets[t] >= 0;
      g_logprob[t] = on ? g0 + (t == lo ? g1 : 0.f) : 0.f;
      g_entropy[t] = on ? g2 + (t == hi ? g3 : 0.f) : 0.f;
    }
  });
  // positions before the first answer and after the last
  const long long before = min(max(A.offsets[0], 0ll), A.T);
  const long long after = min(max(A.offsets[A.Q], 0ll), A.T);
  const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
  const long long by = (long long)gridDim.x * kThreads;
  for (long long t = i; t < before; t += by) g_logprob[t] = g_entropy[t] = 0.f;
  for (long long t = after + i; t < A.T; t += by) g_logprob[t] = g_entropy[t] = 0.f;
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
  return T >= (1ll << 31) || Q > BOUTE_MAX_ANSWERS ? BOUTE_ERR_UNSUPPORTED : device_ok();
}

// Answers of a cluster: as many at a time as leave a lane 16 positions of the mean answer or
// fewer, while there are clusters enough for two blocks an SM.
template <class... KArgs, class... Args>
static int launch_answers(void (*kernel)(Answers, int, KArgs...), const Answers &A,
                          cudaStream_t s, Args... args) {
  const int sms = num_sms();
  int per = kCluster * kWarps;
  while (per > 1 && (A.T / A.Q > 16 * kCluster * kThreads / per ||
                     A.Q * kCluster < 2ll * sms * per))
    per /= 8;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)((A.Q + per - 1) / per * kCluster));
  cfg.blockDim = dim3(kThreads);
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = kCluster;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  cudaLaunchKernelEx(&cfg, kernel, A, per, static_cast<KArgs>(args)...);
  count_launch();
  return last_launch_status();
}

extern "C" int boute_answer_scores(const float *logprob, const float *entropy,
                                   const long long *targets, const long long *offsets,
                                   long long T, long long Q, float *scores, int *counts,
                                   void *stream) {
  BOUTE_TRACE();
  if (Q > 0 && (!array_ok(scores, 4) || !array_ok(counts, 4))) return BOUTE_ERR_INVALID_ARG;
  if (int r = sizes_ok(T, Q, logprob, entropy, targets, offsets)) return r;
  if (Q == 0) return BOUTE_OK;
  return launch_answers(answer_scores_kernel, {logprob, entropy, targets, offsets, T, Q},
                        (cudaStream_t)stream, scores, counts);
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
  return launch_answers(answer_scores_grad_kernel, {logprob, entropy, targets, offsets, T, Q},
                        (cudaStream_t)stream, g_scores, g_logprob, g_entropy);
}
