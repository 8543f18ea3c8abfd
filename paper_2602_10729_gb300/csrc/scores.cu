// The scores of answers (mean and lowest log-probability, mean and highest
// entropy of the positions that hold a token) and their gradient.
//
// A block's teams (8 or 32 lanes, or all of it, by the mean length) take an answer each.
// Lengths are ragged: what is too long for a team is taken by its block afterwards, and
// where answers are long in the mean, by up to eight blocks of a cluster. Latency bounds
// it: the offsets, then the positions, are one trip to memory each, and the longest
// answer's rounds another each. 4096 answers of 200 positions in the mean: 7.4 us (13 MB,
// a floor of 2), their gradient 9.4; 96 of 16384: 12 to 13 and 16 to 19, as the longest
// has it (floors of 3.7 and 5.6). An answer of 2^20 takes 49 us alone and 601 among 4096
// of 200, where it is one block's. Blocks of 512 or 1024 threads: 12.5 and 23 to 30.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32, kMaxCluster = 8;
constexpr int kMost = 32;  // positions a lane of a team of 8 or 32 lanes, or of a block, takes
constexpr int kUnroll = 4;  // positions on their way to a lane

// Order bits with -0 as +0 and a NaN above every number.
__device__ __forceinline__ unsigned extreme_bits(float v) {
  return isnan(v) ? 0xffffffffu : order_bits(v == 0.f ? 0.f : v);
}

// What an answer's scores are made of. lo, hi: extreme_bits of -logprob and of the entropy with
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

// A block's threads may have any number of positions each: a chain of n equal terms can be off by n /
// 2 roundings (a million of them, by 1 %), so what an addition loses goes to the next (Kahan's sum).
__device__ __forceinline__ void add_exact(float &sum, float v, float &lost) {
  const float y = v - lost, t = sum + y;
  lost = (t - sum) - y;
  sum = t;
}

struct Answers {
  const float *logprob, *entropy;
  const long long *targets, *offsets;
  long long T, Q;
  int cluster;  // blocks that share an answer

  __device__ __forceinline__ bool counts(long long t) const { return !targets || targets[t] >= 0; }
  // Thread i of BY over the positions [a, b) of an answer from `from` on (2^31 at most); on: which
  // of its first 64 count. The extremes are compared as floats (3 instructions a position; keys of
  // their order bits took 13, which bounded long answers) unless a NaN or an infinity throughout
  // asks for the keys.
  template <int BY>
  __device__ __forceinline__ Part part(long long from, long long a, long long b, int i,
                                       unsigned long long &on) const {
    Part p = {0ull, 0ull, 0.f, 0.f, 0, 0};
    on = 0ull;
    float lo = INFINITY, hi = -INFINITY;
    int lo_at = -1, hi_at = -1, first = 0;  // of this round, in the thread's order
    float lost_lp = 0.f, lost_ent = 0.f;
    for (long long t0 = a + i; t0 < b; t0 += kUnroll * BY, first += kUnroll) {
      const float *pl = logprob + t0, *ph = entropy + t0;
      const long long *pt = targets + t0;
      const int at0 = (int)(t0 - from);
      float l[kUnroll], h[kUnroll];
      bool in[kUnroll];
      if (!BOUTE_INB(t0, T)) break;
      if (t0 + (kUnroll - 1) * BY < b) {
        if (!BOUTE_INB(t0 + (kUnroll - 1) * BY, T)) break;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          l[u] = pl[u * BY];
          h[u] = ph[u * BY];
          in[u] = targets ? pt[u * BY] >= 0 : true;
        }
      } else {
#pragma unroll
        for (int u = 0; u < kUnroll; ++u) {
          in[u] = t0 + u * BY < b && BOUTE_INB(t0 + u * BY, T);
          if (!in[u]) continue;
          l[u] = pl[u * BY];
          h[u] = ph[u * BY];
          if (targets) in[u] = pt[u * BY] >= 0;
        }
      }
      unsigned bits = 0u;
      float lp = 0.f, ent = 0.f;
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (!in[u]) continue;
        bits |= 1u << u;
        lp += l[u];
        ent += h[u];
        if (l[u] < lo) lo = l[u], lo_at = at0 + u * BY;
        if (h[u] > hi) hi = h[u], hi_at = at0 + u * BY;
      }
      if (BY == kThreads) {
        add_exact(p.lp, lp, lost_lp);
        add_exact(p.ent, ent, lost_ent);
      } else {
        p.lp += lp;
        p.ent += ent;
      }
      p.n += __popc(bits);
      if (first < 64) on |= (unsigned long long)bits << first;
    }
    if (p.n == 0) return p;
    if (lo_at >= 0 && hi_at >= 0 && !isnan(p.lp) && !isnan(p.ent)) {
      p.lo = ((unsigned long long)extreme_bits(-lo) << 32) | (0xffffffffu - (unsigned)lo_at);
      p.hi = ((unsigned long long)extreme_bits(hi) << 32) | (0xffffffffu - (unsigned)hi_at);
      return p;
    }
    p.lp = p.ent = 0.f;  // (what is lost of an infinity is a NaN)
    for (long long t = a + i; t < b; t += BY) {
      if (!counts(t)) continue;
      p.lp += logprob[t];
      p.ent += entropy[t];
      const unsigned at = 0xffffffffu - (unsigned)(t - from);
      p.lo = max(p.lo, ((unsigned long long)extreme_bits(-logprob[t]) << 32) | at);
      p.hi = max(p.hi, ((unsigned long long)extreme_bits(entropy[t]) << 32) | at);
    }
    return p;
  }
};

// The float whose extreme_bits a key has (-0 as +0), and the position; -1 without one.
__device__ __forceinline__ float key_value(unsigned long long key) {
  return from_order_bits((unsigned)(key >> 32));
}
__device__ __forceinline__ int key_position(unsigned long long key) {
  return key ? (int)(0xffffffffu - (unsigned)key) : -1;
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
// Of the whole cluster, in every thread, which have been at cluster_begin; a cluster barrier before
// a block may end.
__device__ __forceinline__ Part cluster_join(Part p, int rank, int cluster, Part *red,
                                             Part *parts) {
  p = block_join(p, red);
  cluster_runs();
  if (threadIdx.x < cluster && BOUTE_INB(rank, kMaxCluster)) {
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

// emit(q, from, p, a, b, on, i, by): thread i of `by` writes what positions [a, b) of answer q
// take, which begins at `from` and has the Part p.
template <int TEAM, class Emit>
__device__ __forceinline__ void for_answers(const Answers &A, Emit emit) {
  __shared__ Part red[kWarps], parts[kMaxCluster];
  if (TEAM == kThreads && A.cluster > 1) cluster_begin();
  pdl_wait();
  pdl_trigger();
  const int tid = threadIdx.x;
  long long a, b;
  unsigned long long on;
  auto range = [&](long long q) {  // within [0, T]
    a = min(max(A.offsets[q], 0ll), A.T);
    b = max(min(A.offsets[q + 1], A.T), a);
  };
  if constexpr (TEAM == kThreads) {
    // a stretch of the answer to each of the cluster's blocks
    const int rank = A.cluster > 1 ? blockIdx.x % A.cluster : 0;
    const long long q = blockIdx.x / A.cluster;
    range(q);
    const long long stretch = (b - a + A.cluster - 1) / A.cluster;
    const long long a1 = min(a + rank * stretch, b), b1 = min(a1 + stretch, b);
    Part p = A.part<kThreads>(a, a1, b1, tid, on);
    if (A.cluster > 1) p = cluster_join(p, rank, A.cluster, red, parts);
    else p = block_join(p, red);
    emit(q, a, p, a1, b1, on, tid, std::integral_constant<int, kThreads>{});
    if (A.cluster > 1) cluster_sync();
  } else {
    constexpr int kPer = kThreads / TEAM;
    const int i = tid % TEAM;
    const long long q0 = (long long)blockIdx.x * kPer, q = q0 + tid / TEAM;
    if (q < A.Q) range(q);
    else a = b = 0;
    const bool more = b - a > kMost * TEAM;
    const Part p = lanes_join(A.part<TEAM>(a, a, more ? a : b, i, on), TEAM);
    if (!more && q < A.Q) emit(q, a, p, a, b, on, i, std::integral_constant<int, TEAM>{});
    // the long ones, one after another by the whole block
    __shared__ unsigned char longer[kPer];
    if (i == 0) longer[tid / TEAM] = more;
    if (!__syncthreads_or(more)) return;
    for (int j = 0; j < kPer; ++j) {
      if (!longer[j]) continue;
      range(q0 + j);
      const Part whole = block_join(A.part<kThreads>(a, a, b, tid, on), red);
      emit(q0 + j, a, whole, a, b, on, tid, std::integral_constant<int, kThreads>{});
      __syncthreads();
    }
  }
}

template <int TEAM>
__global__ void __launch_bounds__(kThreads, 5)
    answer_scores_kernel(Answers A, float *scores, int *counts) {
  for_answers<TEAM>(A, [&](long long q, long long from, const Part &p, long long a, long long b,
                           unsigned long long on, int i, auto by) {
    if (i != 0 || a != from || !BOUTE_INB(q, A.Q)) return;
    const float n = (float)p.n;
    counts[q] = p.n;
    scores[4 * q] = p.n ? p.lp / n : 0.f;
    scores[4 * q + 1] = p.n ? 0.f - key_value(p.lo) : 0.f;  // (0 - v: +0 for -0)
    scores[4 * q + 2] = p.n ? p.ent / n : 0.f;
    scores[4 * q + 3] = p.n ? key_value(p.hi) : 0.f;
  });
}

template <int TEAM>
__global__ void __launch_bounds__(kThreads, 5)
    answer_scores_grad_kernel(Answers A, const float *g_scores, float *g_logprob,
                              float *g_entropy) {
  for_answers<TEAM>(A, [&](long long q, long long from, const Part &p, long long a, long long b,
                           unsigned long long on, int i, auto by) {
    constexpr int BY = decltype(by)::value;
    const float n = p.n ? (float)p.n : 1.f;
    if (!BOUTE_INB(q, A.Q)) return;
    const float *g = g_scores + 4 * q;
    const float g0 = g[0] / n, g1 = g[1], g2 = g[2] / n, g3 = g[3];
    const int lo = key_position(p.lo), hi = key_position(p.hi);  // from `from` on
    int first = 0;
    for (long long t0 = a + i; t0 < b; t0 += kUnroll * BY, first += kUnroll) {
      float *pl = g_logprob + t0, *ph = g_entropy + t0;
      const int at0 = (int)(t0 - from), left = (int)min(b - t0, (long long)kUnroll * BY);
      unsigned bits = (unsigned)(on >> first);
      if (first >= 64) {
        bits = 0u;
#pragma unroll
        for (int u = 0; u < kUnroll; ++u)
          if (u * BY < left) bits |= (unsigned)A.counts(t0 + u * BY) << u;
      }
#pragma unroll
      for (int u = 0; u < kUnroll; ++u) {
        if (u * BY >= left || !BOUTE_INB(t0 + u * BY, A.T)) break;
        const bool in = bits >> u & 1u;
        pl[u * BY] = in ? g0 + (at0 + u * BY == lo ? g1 : 0.f) : 0.f;
        ph[u * BY] = in ? g2 + (at0 + u * BY == hi ? g3 : 0.f) : 0.f;
      }
    }
  });
  // positions before the first answer and after the last
  if (blockIdx.x == 0) {
    const long long end = min(max(A.offsets[0], 0ll), A.T);
    for (long long t = threadIdx.x; t < end; t += kThreads) g_logprob[t] = g_entropy[t] = 0.f;
  }
  if (blockIdx.x == gridDim.x - 1) {
    const long long from = min(max(A.offsets[A.Q], 0ll), A.T);
    for (long long t = from + threadIdx.x; t < A.T; t += kThreads)
      g_logprob[t] = g_entropy[t] = 0.f;
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
  return T > BOUTE_MAX_POSITIONS || Q > BOUTE_MAX_ANSWERS ? BOUTE_ERR_UNSUPPORTED : device_ok();
}

// Teams by the mean length: 8 lanes up to 24 positions, 32 up to 512, else a block; and up to the
// eight blocks of a cluster for answers over 1024 positions a block that are too few to fill the
// SMs. (13665 answers of 31: 6.3 us with 32 lanes, 8.0 with 8; 2245 of 682: 11.7 with a block, 14.1
// with 32 lanes.)
template <class Go>
static int with_team(long long T, long long Q, Go go) {
  const long long mean = T / Q, at_once = 8ll * num_sms();
  if (mean <= 24) return go(std::integral_constant<int, 8>{}, (Q + 31) / 32, 1);
  if (mean <= 512) return go(std::integral_constant<int, 32>{}, (Q + 7) / 8, 1);
  int cluster = 1;
  while (cluster < kMaxCluster && mean > 1024 * cluster && 2 * cluster * Q <= at_once) cluster *= 2;
  return go(std::integral_constant<int, kThreads>{}, Q * cluster, cluster);
}

extern "C" int boute_answer_scores(const float *logprob, const float *entropy,
                                   const long long *targets, const long long *offsets,
                                   long long T, long long Q, float *scores, int *counts,
                                   void *stream) {
  BOUTE_TRACE();
  if (Q > 0 && (!array_ok(scores, 4) || !array_ok(counts, 4))) return BOUTE_ERR_INVALID_ARG;
  if (int r = sizes_ok(T, Q, logprob, entropy, targets, offsets)) return r;
  if (Q == 0) return BOUTE_OK;
  return with_team(T, Q, [&](auto team, long long blocks, int cluster) {
    return launch_cluster(answer_scores_kernel<decltype(team)::value>, blocks, kThreads, cluster, 0,
                          (cudaStream_t)stream,
                          Answers{logprob, entropy, targets, offsets, T, Q, cluster}, scores,
                          counts);
  });
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
  return with_team(T, Q, [&](auto team, long long blocks, int cluster) {
    return launch_cluster(answer_scores_grad_kernel<decltype(team)::value>, blocks, kThreads,
                          cluster, 0, (cudaStream_t)stream,
                          Answers{logprob, entropy, targets, offsets, T, Q, cluster}, g_scores,
                          g_logprob, g_entropy);
  });
}
