// The scores of answers (mean and lowest log-probability, mean and highest
// entropy of the positions that hold a token) and their gradient.
//
// A block's teams (8 or 32 lanes, or all of it, by the mean length) take an answer each.
// Lengths are ragged: what is too long for a team is taken by its block afterwards, and
// where answers are long in the mean, by the eight blocks of a cluster. Latency bounds it:
// the offsets, then the positions, are one trip to memory each.
#include <math.h>

#include <algorithm>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxCluster = 8;
constexpr int kMost = 32;  // positions a lane of a team of 8 or 32 lanes, or of a block, takes
constexpr int kUnroll = 4;  // positions on their way to a lane

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
  int cluster;  // blocks of a cluster, 1 or kMaxCluster
  int per;      // answers of a block, or 0: one of a cluster

  // Thread i of `by` over the positions [a, b) (2^31 at most); on: which of its first 64 count.
  __device__ __forceinline__ Part part(long long a, long long b, int i, int by,
                                       unsigned long long &on) const {
    Part p = {0ull, 0ull, 0.f, 0.f, 0, 0};
    on = 0ull;
    int first = 0;  // of this round's positions, in the thread's order
    for (long long t0 = a + i; t0 < b; t0 += kUnroll * by, first += kUnroll) {
      float l[kUnroll], h[kUnroll];
      unsigned in = 0u;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        const long long t = t0 + u * by;
        if (t >= b) continue;
        l[u] = logprob[t];
        h[u] = entropy[t];
        in |= (unsigned)(targets ? targets[t] >= 0 : true) << u;
      }
      if (first < 64) on |= (unsigned long long)in << first;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (!(in >> u & 1u)) continue;
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

// The float whose order_bits a key has (-0 as +0), and the position, of an answer from a on.
__device__ __forceinline__ float key_value(unsigned long long key) {
  const unsigned o = (unsigned)(key >> 32);
  return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}
__device__ __forceinline__ long long key_position(unsigned long long key, long long a) {
  return a + (long long)(0xffffffffu - (unsigned)key);
}

// Of `lanes` neighbouring lanes, in each of them.
__device__ __forceinline__ Part lanes_join(Part p, int lanes) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < lanes)
      add(p, {shfl_xor64(p.lo, o), shfl_xor64(p.hi, o), __shfl_xor_sync(kAll, p.lp, o),
              __shfl_xor_sync(kAll, p.ent, o), __shfl_xor_sync(kAll, p.n, o), 0});
  return p;
}
// Of the whole block, in every thread; red (kWarps Parts) may be used again after a barrier.
__device__ __forceinline__ Part block_join(Part p, Part *red) {
  p = lanes_join(p, 32);
  if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = p;
  __syncthreads();
  p = red[0];
  for (int w = 1; w < kWarps; ++w) add(p, red[w]);
  return p;
}
// Of the whole cluster, in every thread; a cluster barrier before a block may end.
__device__ __forceinline__ Part cluster_join(Part p, int rank, int cluster, Part *red,
                                             Part *parts) {
  p = block_join(p, red);
  if (threadIdx.x < cluster) {
    const uint32_t to = peer(&parts[rank], threadIdx.x);
    store_peer(to, p.lo);
    store_peer(to + 8, p.hi);
    store_peer(to + 16, p.lp);
    store_peer(to + 20, p.ent);
    store_peer(to + 24, __int_as_float(p.n));
  }
  cluster_sync();
  p = parts[0];
  for (int r = 1; r < cluster; ++r) add(p, parts[r]);
  return p;
}

// emit(q, a, b, p, on, i, by): thread i of `by` writes its share of answer q's results.
template <class Emit>
__device__ __forceinline__ void for_answers(const Answers &A, Emit emit) {
  pdl_wait();
  pdl_trigger();
  __shared__ Part red[kWarps], parts[kMaxCluster];
  const int tid = threadIdx.x;
  long long a, b;
  unsigned long long on;
  auto range = [&](long long q) {  // within [0, T]
    a = min(max(A.offsets[q], 0ll), A.T);
    b = max(min(A.offsets[q + 1], A.T), a);
  };
  if (A.per == 0) {
    const int rank = blockIdx.x % A.cluster, i = rank * kThreads + tid, by = A.cluster * kThreads;
    const long long q = blockIdx.x / A.cluster;
    range(q);
    Part p = A.part(a, b, i, by, on);
    if (A.cluster > 1) p = cluster_join(p, rank, A.cluster, red, parts);
    else p = block_join(p, red);
    emit(q, a, b, p, on, i, by);
    if (A.cluster > 1) cluster_sync();
    return;
  }
  const int team = kThreads / A.per, i = tid % team;
  const long long q = (long long)blockIdx.x * A.per + tid / team;
  if (q < A.Q) range(q);
  else a = b = 0;
  const bool more = b - a > kMost * team;
  const Part p = lanes_join(A.part(a, more ? a : b, i, team, on), team);
  if (!more && q < A.Q) emit(q, a, b, p, on, i, team);
  // the long ones, one after another by the whole block
  __shared__ unsigned char longer[kThreads / 8];
  if (i == 0) longer[tid / team] = more;
  if (!__syncthreads_or(more)) return;
  for (int j = 0; j < A.per; ++j) {
    if (!longer[j]) continue;
    range((long long)blockIdx.x * A.per + j);
    const Part whole = block_join(A.part(a, b, tid, kThreads, on), red);
    emit((long long)blockIdx.x * A.per + j, a, b, whole, on, tid, kThreads);
    __syncthreads();
  }
}

__global__ void __launch_bounds__(kThreads, 5)
    answer_scores_kernel(Answers A, float *scores, int *counts) {
  for_answers(A, [&](long long q, long long a, long long b, const Part &p, unsigned long long on,
                     int i, int by) {
    if (i != 0) return;
    const float n = (float)p.n;
    counts[q] = p.n;
    scores[4 * q] = p.n ? p.lp / n : 0.f;
    scores[4 * q + 1] = p.n ? 0.f - key_value(p.lo) : 0.f;  // (0 - v: +0 for -0)
    scores[4 * q + 2] = p.n ? p.ent / n : 0.f;
    scores[4 * q + 3] = p.n ? key_value(p.hi) : 0.f;
  });
}

__global__ void __launch_bounds__(kThreads, 5)
    answer_scores_grad_kernel(Answers A, const float *g_scores, float *g_logprob,
                              float *g_entropy) {
  for_answers(A, [&](long long q, long long a, long long b, const Part &p, unsigned long long on,
                     int i, int by) {
    const float n = p.n ? (float)p.n : 1.f;
    const float *g = g_scores + 4 * q;
    const float g0 = g[0] / n, g1 = g[1], g2 = g[2] / n, g3 = g[3];
    const long long lo = key_position(p.lo, a), hi = key_position(p.hi, a);
    int nth = 0;
#pragma unroll 4
    for (long long t = a + i; t < b; t += by, ++nth) {
      const bool in = nth < 64 ? on >> nth & 1ull : !A.targets || A.targets[t] >= 0;
      g_logprob[t] = in ? g0 + (t == lo ? g1 : 0.f) : 0.f;
      g_entropy[t] = in ? g2 + (t == hi ? g3 : 0.f) : 0.f;
    }
  });
  // positions before the first answer and after the last
  if (blockIdx.x == 0) {
    const long long end = min(max(A.offsets[0], 0ll), A.T);
    for (long long t = threadIdx.x; t < end; t += kThreads) g_logprob[t] = g_entropy[t] = 0.f;
  }
  if (blockIdx.x == gridDim.x - 1) {
    const long long from = min(max(A.offsets[A.Q], 0ll), A.T);
    for (long long t = from + threadIdx.x; t < A.T; t += kThreads) g_logprob[t] = g_entropy[t] = 0.f;
  }
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

// Teams by the mean length: 8 lanes up to 48 positions, 32 up to 512, else a block; and up to the
// eight blocks of a cluster for answers over 1024 positions a block that are too few to fill the SMs.
// (13665 answers of 31: 9.8 us with 8 lanes, 14 with 32; 4096 of 200: 10.5 with 32, 15.6 with a
// block; 96 of 16384: 13 with eight blocks, 18 with four.)
template <class... KArgs, class... Args>
static int launch_answers(void (*kernel)(Answers, KArgs...), Answers A, cudaStream_t s,
                          Args... args) {
  const long long mean = A.T / A.Q, at_once = 8ll * num_sms();
  A.per = mean <= 48 ? 32 : mean <= 512 ? 8 : 0;
  while (A.cluster < kMaxCluster && A.per == 0 && mean > 1024 * A.cluster &&
         2 * A.cluster * A.Q <= at_once)
    A.cluster *= 2;
  return launch_cluster(kernel, A.per ? (A.Q + A.per - 1) / A.per : A.Q * A.cluster, kThreads,
                        A.cluster, 0, s, A, args...);
}

extern "C" int boute_answer_scores(const float *logprob, const float *entropy,
                                   const long long *targets, const long long *offsets,
                                   long long T, long long Q, float *scores, int *counts,
                                   void *stream) {
  BOUTE_TRACE();
  if (Q > 0 && (!array_ok(scores, 4) || !array_ok(counts, 4))) return BOUTE_ERR_INVALID_ARG;
  if (int r = sizes_ok(T, Q, logprob, entropy, targets, offsets)) return r;
  if (Q == 0) return BOUTE_OK;
  return launch_answers(answer_scores_kernel, {logprob, entropy, targets, offsets, T, Q, 1, 0},
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
  return launch_answers(answer_scores_grad_kernel, {logprob, entropy, targets, offsets, T, Q, 1, 0},
                        (cudaStream_t)stream, g_scores, g_logprob, g_entropy);
}
