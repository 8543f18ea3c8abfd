// Log-probabilities of given tokens, with the entropy and the top alternatives
// of every position, and the gradient with respect to the logits.
//
// With z = scale x, m = max z, s = sum exp(z - m) and u = sum (z - m) exp(z - m):
//   lse = m + ln s,  logprob = z_t - m - ln s,  entropy = ln s - u / s.
// One pass over a row: each warp keeps a running maximum and s and u relative to
// it, and every lane notes the two of the 64-byte parts of the row it saw whose maxima
// are largest. The k-th largest of the lanes' own maxima is reached by k logits at least,
// and by few others; the noted parts that reach it are read again, and what reaches it
// there is ranked. (A lane with a third such part reads all of its parts again.) A row is
// a block's, or a cluster's when there are few rows. Shared memory is left to the L1
// cache, through which the loads in flight pass: with 16 KB a block for the parts
// themselves, reads were 10 % slower.
//
// Memory bounds the large calls: 8192 rows of 131072 bf16 logits, k = 20: 339 us
// (6.3 TB/s, 0.93 of the copy rate; k = 0: 306 us, 1.04; 4096 rows of fp32: 327); their
// gradient, which writes as much as it reads, 640 us (0.99; fp32 655). Rows that do not
// fill whole waves of blocks pay for the last one: 2039 rows of 50021 fp16, k = 8: 43 us
// (0.70). What follows a row's loads
// (joining, the bound, the second look, the ranks) is 4 us of latency, which bounds the
// small calls: one row of 50021, k = 5: 5.2 us; 64 of 131072 fp32, k = 20: 10.8.
#include <float.h>
#include <math.h>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kThreads = 256, kWarps = 4;  // a block's most; its warps when rows are many
constexpr int kMaxCluster = 8;
constexpr int kTops = 256;  // maxima from which the alternatives' bound is taken
constexpr int kList = 256;  // candidates ranked at once, 32 a warp at least
constexpr float kLowest = -200.f;  // exp(kLowest) = 2^kLowest = 0 in fp32
constexpr float kLn2 = 0.6931471805599453f;

// ---- a row in pieces -----------------------------------------------------------------
// A piece is 2 KB of a row, of which a lane holds four 16-byte vectors 512 bytes apart. Piece q
// holds the logits [q SPAN - off, (q + 1) SPAN - off) of a row whose first logit lies `off` logits
// after a 16-byte boundary, so that every vector starts on one.
template <class T>
struct Piece {
  static constexpr int E = 16 / sizeof(T), N = 4 * E, SPAN = 32 * N;
  uint4 v[4];
  // of a lane's j-th logit, within the piece
  static __device__ __forceinline__ int index(int j, int lane = threadIdx.x & 31) {
    return (j / E * 32 + lane) * E + j % E;
  }
  static __host__ __device__ int count(int off, int V) { return (off + V + SPAN - 1) / SPAN; }
};

// A whole piece of a row y of V logits from its logit `first` on, read once (its lines need not stay
// in L1).
template <class T>
__device__ __forceinline__ Piece<T> load_whole(const T *y, int V, long long first) {
  Piece<T> r;
  if (!BOUTE_INB(first, V) || !BOUTE_INB(first + Piece<T>::SPAN - 1, V)) {
    memset(r.v, 0, sizeof(r.v));
    return r;
  }
  const uint4 *p = (const uint4 *)(y + first) + (threadIdx.x & 31);
#pragma unroll
  for (int i = 0; i < 4; ++i)
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(r.v[i].x), "=r"(r.v[i].y), "=r"(r.v[i].z), "=r"(r.v[i].w)
                 : "l"(p + 32 * i)
                 : "memory");
  return r;
}
// The piece of a row y of V logits from its logit `first` on, `shift` bytes after a 16-byte
// boundary: -inf outside the row, of which nothing is read. (lane: whose part)
template <class T>
__device__ __forceinline__ Piece<T> load_piece(const T *y, int V, int first, int shift,
                                               int lane = threadIdx.x & 31) {
  constexpr int E = Piece<T>::E;
  Piece<T> r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j0 = first + Piece<T>::index(i * E, lane);
    if (shift == 0 && j0 >= 0 && j0 + E <= V) {
      r.v[i] = *(const uint4 *)(y + j0);
    } else if (j0 >= E && j0 + 2 * E <= V) {  // two vectors, of which these 16 bytes
      const char *p = (const char *)(y + j0) - shift;
      const uint4 a = *(const uint4 *)p, b = *(const uint4 *)(p + 16);
      uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      if (shift & 8)
#pragma unroll
        for (int q = 0; q < 6; ++q) w[q] = w[q + 2];
      if (shift & 4)
#pragma unroll
        for (int q = 0; q < 5; ++q) w[q] = w[q + 1];
      const int bits = 8 * (shift & 3);
      r.v[i] = {__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits)};
    } else {
      T t[E];
#pragma unroll
      for (int e = 0; e < E; ++e)
        t[e] = j0 + e >= 0 && j0 + e < V ? y[j0 + e] : from_float<T>(-INFINITY);
      memcpy(&r.v[i], t, 16);
    }
  }
  return r;
}
// The piece of the row y from its logit `first` (on a boundary) on; nothing outside is written.
template <class T>
__device__ __forceinline__ void store_piece(T *y, int V, int first, const Piece<T> &r) {
  constexpr int E = Piece<T>::E;
  if (first >= 0 && first + Piece<T>::SPAN <= V) {
    if (!BOUTE_INB((uintptr_t)(y + first) % 16, 1)) return;  // (a boundary)
    uint4 *p = (uint4 *)(y + first) + (threadIdx.x & 31);
#pragma unroll
    for (int i = 0; i < 4; ++i) p[32 * i] = r.v[i];
    return;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int j0 = first + Piece<T>::index(i * E);
    T t[E];
    memcpy(t, &r.v[i], 16);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (j0 + e >= 0 && j0 + e < V) y[j0 + e] = t[e];
  }
}

// Logits 2 j and 2 j + 1 of a lane's piece as a pair of floats, and back (one rounding).
__device__ __forceinline__ uint32_t word(const uint4 (&v)[4], int j) {
  const uint4 a = v[j / 4];
  return j % 4 == 0 ? a.x : j % 4 == 1 ? a.y : j % 4 == 2 ? a.z : a.w;
}
__device__ __forceinline__ void set_word(uint4 (&v)[4], int j, uint32_t w) {
  uint4 &a = v[j / 4];
  (j % 4 == 0 ? a.x : j % 4 == 1 ? a.y : j % 4 == 2 ? a.z : a.w) = w;
}
__device__ __forceinline__ void pair(const Piece<float> &p, int j, float &a, float &b) {
  a = __uint_as_float(word(p.v, 2 * j));
  b = __uint_as_float(word(p.v, 2 * j + 1));
}
__device__ __forceinline__ void pair(const Piece<__nv_bfloat16> &p, int j, float &a, float &b) {
  a = __uint_as_float(word(p.v, j) << 16);
  b = __uint_as_float(word(p.v, j) & 0xffff0000u);
}
__device__ __forceinline__ void pair(const Piece<__half> &p, int j, float &a, float &b) {
  unpack_f16x2(word(p.v, j), a, b);
}
__device__ __forceinline__ void set_pair(Piece<float> &p, int j, float a, float b) {
  set_word(p.v, 2 * j, __float_as_uint(a));
  set_word(p.v, 2 * j + 1, __float_as_uint(b));
}
__device__ __forceinline__ void set_pair(Piece<__nv_bfloat16> &p, int j, float a, float b) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  set_word(p.v, j, r);
}
__device__ __forceinline__ void set_pair(Piece<__half> &p, int j, float a, float b) {
  set_word(p.v, j, pack_f16x2(a, b));
}

// A lane's largest logit of a piece, NaN if it holds one.
__device__ __forceinline__ float lane_max(const Piece<float> &p) {
  float m = __uint_as_float(word(p.v, 15));
#pragma unroll
  for (int j = 0; j < 14; j += 2)
    m = max_nan(m, __uint_as_float(word(p.v, j)), __uint_as_float(word(p.v, j + 1)));
  return max_nan(m, __uint_as_float(word(p.v, 14)));
}
template <class H2, class T>
__device__ __forceinline__ float lane_max16(const Piece<T> &p) {
  H2 h[16];
  memcpy(h, p.v, 64);
#pragma unroll
  for (int o = 8; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < o; ++i) h[i] = __hmax2_nan(h[i], h[i + o]);
  return max_nan(to_float(h[0].x), to_float(h[0].y));
}
__device__ __forceinline__ float lane_max(const Piece<__half> &p) { return lane_max16<__half2>(p); }
__device__ __forceinline__ float lane_max(const Piece<__nv_bfloat16> &p) {
  return lane_max16<__nv_bfloat162>(p);
}

// ---- sums ----------------------------------------------------------------------------
// s = sum 2^y and u = sum y 2^y with y = (x - m) c, c = scale log2 e (x - m is exact where it
// matters: rows at the type's lowest value throughout have x - m = 0); m = -inf: nothing yet.
struct Sums {
  float m, s, u;
  // s and u relative to a larger (or equal) m
  __device__ __forceinline__ void move(float to, float c) {
    if (m == -INFINITY) s = u = 0.f;  // (also when `to` is)
    else {
      const float d = fmaxf((m - to) * c, kLowest), f = exp2_fast(d);
      u = (u + d * s) * f;
      s *= f;
    }
    m = to;
  }
};

__device__ __forceinline__ Sums join(Sums a, Sums b, float c) {
  const float m = fmaxf(a.m, b.m);
  a.move(m, c);
  b.move(m, c);
  return {m, a.s + b.s, a.u + b.u};
}

// A piece's pairs of partial sums (which join the running ones once: a lane's terms, some hundreds of
// a long row, added one after another would round at the running sum's size each time); CLAMP: with logits so far below m that (x - m) c
// overflows (-inf, masks of the type's lowest value), whose y 2^y is else a NaN.
template <bool CLAMP, class T>
__device__ __forceinline__ void sum_piece(const Piece<T> &p, float m, float c,
                                          unsigned long long &s2, unsigned long long &u2) {
  const unsigned long long m2 = f2_dup(m), c2 = f2_dup(c);
  s2 = u2 = 0ull;
#pragma unroll
  for (int j = 0; j < Piece<T>::N / 2; ++j) {
    float a, b;
    pair(p, j, a, b);
    unsigned long long y = f2_mul(f2_sub(f2_pack(a, b), m2), c2);
    f2_split(y, a, b);
    if (CLAMP) {
      a = fmaxf(a, kLowest);
      b = fmaxf(b, kLowest);
      y = f2_pack(a, b);
    }
    const unsigned long long e = f2_pack(exp2_fast(a), exp2_fast(b));
    s2 = f2_add(s2, e);
    u2 = f2_fma(y, e, u2);
  }
}

// ---- alternatives --------------------------------------------------------------------
// An upper half of order bits, which stands for a lower bound, that k of n floats reach (n a
// multiple of 32, at most kTops), close to the largest such one: built two bits at a time until
// exactly k reach it; by one warp. That of -inf where fewer than k are above it.
__device__ __forceinline__ unsigned kth_bound(const float *v, int n, int k) {
  const int lane = threadIdx.x & 31;
  unsigned o[kTops / 32], t = 0u;
#pragma unroll
  for (int i = 0; i < kTops / 32; ++i) o[i] = 32 * i < n ? order_bits(v[32 * i + lane]) >> 16 : 0u;
  for (int b = 14; b >= 0; b -= 2) {
    unsigned c = 0u;  // the counts at or above three trials, ten bits each
#pragma unroll
    for (int i = 0; i < kTops / 32; ++i) {
      c += o[i] >= (t | 1u << b) ? 1u : 0u;
      c += o[i] >= (t | 2u << b) ? 1u << 10 : 0u;
      c += o[i] >= (t | 3u << b) ? 1u << 20 : 0u;
    }
    c = __reduce_add_sync(kAll, c);
    const int c1 = c & 1023u, c2 = c >> 10 & 1023u, c3 = c >> 20;
    t |= (c3 >= k ? 3u : c2 >= k ? 2u : c1 >= k ? 1u : 0u) << b;
    if (c3 == k || c2 == k || c1 == k) break;
  }
  return max(t, order_bits(-INFINITY) >> 16);
}
// A warp's best 32 keys, fed with those above a bound that rises with the k-th of them.
struct WarpBest {
  WarpTopBatch batch;
  unsigned long long bound = 0ull;
  __device__ __forceinline__ void feed(bool in, unsigned long long key, int k, int lane) {
    unsigned rest = __ballot_sync(kAll, in && key > bound);
    while (rest) {
      const unsigned long long b = shfl64(key, __ffs(rest) - 1);
      rest &= rest - 1;
      if (b <= bound) continue;
      batch.add(b, lane);
      if (batch.count == 0) bound = shfl64(batch.top, k - 1);
    }
  }
};

// A row per cluster of CS blocks; piece q is warp (q mod CS W)'s.
template <class T>
__global__ void __launch_bounds__(kThreads, 4)
    token_logprobs_kernel(const T *logits, int V, long long ld, const long long *targets,
                          float scale, int k, int CS, float *logprob, float *entropy, float *lse,
                          long long *top_idx, float *top_logprob) {
  constexpr int N = Piece<T>::N, SPAN = Piece<T>::SPAN;
  __shared__ unsigned long long list[kList];  // (the leader's) candidates' keys
  __shared__ float tops[kTops], lanes[kThreads];
  __shared__ Sums wsum[kThreads / 32];
  __shared__ float csum[kMaxCluster][3];
  __shared__ float stat[2];  // m (NaN: no distribution) and ln s
  __shared__ unsigned bound;
  __shared__ int nlist;
  if (CS > 1) cluster_begin();
  pdl_wait();
  pdl_trigger();
  const int NT = blockDim.x, W = NT / 32, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = CS > 1 ? blockIdx.x % CS : 0;
  const long long row = blockIdx.x / CS;
  const T *x = logits + row * ld;
  const int off = (int)((uintptr_t)x % 16 / sizeof(T));
  const float c = fminf(scale * kLog2e, FLT_MAX);
  long long t = -1;
  float xt = 0.f;
  if (tid == 0) nlist = 0;
  if (tid == NT - 32 && rank == 0) {  // (of the warp that writes the row's statistics)
    t = targets[row];
    if (t >= 0 && t < V) xt = to_float(x[t]);
  }

  const int Q = Piece<T>::count(off, V), step = CS * W, first = rank * W + warp;
  const int whole0 = off ? 1 : 0, whole1 = (off + V) / SPAN;  // pieces within the row
  float m = -INFINITY;
  unsigned long long s2 = 0ull, u2 = 0ull;  // pairs of partial sums
  bool clamp = false;
  // the three largest maxima of this lane's parts, and the pieces of the first two
  float top = -INFINITY, second = -INFINITY, third = -INFINITY;
  int q1 = -1, q2 = -1;
  for (int q = first; q < Q; q += step) {
    const bool whole = q >= whole0 && q < whole1;
    const Piece<T> p = whole ? load_whole(x, V, (long long)q * SPAN - off)
                             : load_piece(x, V, q * SPAN - off, 0);
    const float l = lane_max(p);
    if (k > 0) {
      q2 = l > top ? q1 : l > second ? q : q2;
      q1 = l > top ? q : q1;
      third = fmaxf(third, fminf(second, l));
      second = fmaxf(second, fminf(top, l));
      top = fmaxf(top, l);
    }
    const float g = warp_max_nan(l);
    if (!(g <= m)) {  // (NaN too: it stays in m)
      Sums a, b;
      a.m = b.m = m;
      f2_split(s2, a.s, b.s);
      f2_split(u2, a.u, b.u);
      a.move(g, c);
      b.move(g, c);
      s2 = f2_pack(a.s, b.s);
      u2 = f2_pack(a.u, b.u);
      m = max_nan(m, g);
    }
    unsigned long long s = 0ull, u = 0ull;
    if (whole && !clamp) {
      sum_piece<false>(p, m, c, s, u);
      float a, b;
      f2_split(u, a, b);
      clamp = __any_sync(kAll, isnan(a + b));
    }
    if (!whole || clamp) {
      if (!(m > -INFINITY)) continue;
      sum_piece<true>(p, m, c, s, u);
    }
    s2 = f2_add(s2, s);
    u2 = f2_add(u2, u);
  }
  {
    float a, b;
    f2_split(s2, a, b);
    const float s = warp_sum(a + b);
    f2_split(u2, a, b);
    const float u = warp_sum(a + b);
    if (lane == 0) wsum[warp] = {m, s, u};
  }
  (CS > 1 ? lanes : tops)[tid] = top;
  __syncthreads();
  if (CS > 1) {
    cluster_runs();
    if (tid == 0 && BOUTE_INB(rank, kMaxCluster)) {
      Sums a = wsum[0];
      for (int w = 1; w < W; ++w) {
        if (isnan(wsum[w].m)) a.m = NAN;
        a = isnan(a.m) ? a : join(a, wsum[w], c);
      }
      store_peer(peer(&csum[rank][0], 0), a.m);
      store_peer(peer(&csum[rank][1], 0), a.s);
      store_peer(peer(&csum[rank][2], 0), a.u);
    }
    // the blocks' lane maxima to all blocks, kTops / CS of each: of lanes with the same number
    // in warps this far apart
    const int mine = kTops / CS;
    if (k > 0 && tid < mine) {
      float t = -INFINITY;
      for (int i = tid; i < NT; i += mine) t = max_nan(t, lanes[i]);
      for (int b = 0; b < CS; ++b)
        if (BOUTE_INB(rank * mine + tid, kTops)) store_peer(peer(&tops[rank * mine + tid], b), t);
    }
    cluster_sync();
  }
  if (rank == 0 && warp == W - 1) {  // (the bound is another warp's)
    const int n = CS > 1 ? CS : W;
    Sums a = {-INFINITY, 0.f, 0.f};
    if (lane < n) a = CS > 1 ? Sums{csum[lane][0], csum[lane][1], csum[lane][2]} : wsum[lane];
    bool bad = __any_sync(kAll, isnan(a.m));
#pragma unroll
    for (int o = kMaxCluster / 2; o > 0; o >>= 1)
      a = join(a, {__shfl_xor_sync(kAll, a.m, o), __shfl_xor_sync(kAll, a.s, o),
                   __shfl_xor_sync(kAll, a.u, o)}, c);
    const float M = __fmul_rn(a.m, scale);
    const bool empty = M == -INFINITY;  // (scaled values that underflow the type are masked too)
    bad |= M == INFINITY;
    const float ls = empty ? 0.f : logf(a.s);
    if (lane == 0) {
      float lp = 0.f;
      if (t >= V || (bad && t >= 0)) lp = NAN;
      else if (t >= 0) lp = empty ? -INFINITY : __fmul_rn(xt, scale) - M - ls;
      lse[row] = bad ? NAN : M + ls;
      logprob[row] = lp;
      entropy[row] = bad ? NAN : empty ? 0.f : ls - kLn2 * (a.u / a.s);
      stat[0] = bad ? NAN : M;
      stat[1] = ls;
    }
  }
  float zt = -INFINITY;
  if (k > 0) {
    // a bound that k lanes reach
    if (warp == 0) bound = kth_bound(tops, CS > 1 ? kTops : NT, k);
    __syncthreads();
    if (bound > order_bits(-INFINITY) >> 16) zt = __fmul_rn(from_order_bits(bound << 16), scale);
    bool full = false;
    // a part's logits that reach the bound, into the list
    auto take_from = [&](const Piece<T> &p, int q, int of) {
      unsigned hit = 0u;
#pragma unroll
      for (int j = 0; j < N; j += 2) {
        float a, b;
        pair(p, j / 2, a, b);
        hit |= (__fmul_rn(a, scale) >= zt ? 1u : 0u) << j;
        hit |= (__fmul_rn(b, scale) >= zt ? 1u : 0u) << (j + 1);
      }
      while (hit) {
        const int j = __ffs(hit) - 1;
        hit &= hit - 1;
        const int index = q * SPAN - off + Piece<T>::index(j, of);
        if (index < 0 || index >= V) continue;  // (-inf beyond the row, with a bound of -inf)
        if (!BOUTE_INB(q, Q)) continue;  // (a piece of this row)
        const float z = __fmul_rn(to_float(x[index]), scale);
        if (z == -INFINITY) continue;
        const int to = add_peer(peer(&nlist, 0), 1);
        if (to < kList) store_peer(peer(list, 0) + 8u * to, make_key(z, (unsigned)index));
        else full = true, hit = 0u;
      }
    };
    auto reaches = [&](float v) { return v > -INFINITY && __fmul_rn(v, scale) >= zt; };
    const bool r1 = reaches(top), r2 = reaches(second);
    Piece<T> p1, p2;
    if (r1) p1 = load_piece(x, V, q1 * SPAN - off, 0);
    if (r2) p2 = load_piece(x, V, q2 * SPAN - off, 0);
    if (r1) take_from(p1, q1, lane);
    if (r2) take_from(p2, q2, lane);
    // a lane with a third: its other parts, a piece to each lane
    unsigned more = __ballot_sync(kAll, reaches(third));
    while (more) {
      const int of = __ffs(more) - 1;
      more &= more - 1;
      const int skip1 = __shfl_sync(kAll, q1, of), skip2 = __shfl_sync(kAll, q2, of);
      for (int q = first + lane * step; q < Q && !full; q += 32 * step) {
        if (q == skip1 || q == skip2) continue;
        const Piece<T> p = load_piece(x, V, q * SPAN - off, 0, of);
        if (reaches(lane_max(p))) take_from(p, q, of);
      }
    }
    if (CS > 1) cluster_sync();
    else __syncthreads();
  }
  if (rank != 0) return;
  if (k > 0) {
    const float M = stat[0], ls = stat[1];
    const bool bad = isnan(M), empty = M == -INFINITY;
    int n = bad || empty ? 0 : nlist;
    if (n > kList) {  // (many equal logits, or most of the largest in few lanes)
      __syncthreads();
      if (tid == 0) nlist = 0;
      __syncthreads();
      WarpBest best;
      for (int q = warp; q < Q; q += W) {
        const Piece<T> p = load_piece(x, V, q * SPAN - off, 0);
        if (!__any_sync(kAll, __fmul_rn(lane_max(p), scale) >= zt)) continue;
#pragma unroll
        for (int j = 0; j < N; j += 2) {
          float z[2];
          pair(p, j / 2, z[0], z[1]);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            z[e] = __fmul_rn(z[e], scale);
            best.feed(z[e] >= zt && z[e] > -INFINITY,
                      make_key(z[e], (unsigned)(q * SPAN - off + Piece<T>::index(j + e))), k, lane);
          }
        }
      }
      best.batch.flush(lane);
      if (lane < k && best.batch.top != 0ull) {
        const int at = atomicAdd(&nlist, 1);
        if (BOUTE_INB(at, kList)) list[at] = best.batch.top;
      }
      __syncthreads();
      n = nlist;
    }
    for (int i = tid; i < n; i += NT) {
      const unsigned long long key = list[i];
      int place = 0;
      for (int j = 0; j < n; ++j) place += list[j] > key;
      if (place < k && BOUTE_INB(key_index(key), V)) {
        top_idx[row * k + place] = (long long)key_index(key);
        top_logprob[row * k + place] = from_order_bits((unsigned)(key >> 32)) - M - ls;
      }
    }
    for (int i = n + tid; i < k; i += NT) {
      top_idx[row * k + i] = -1;
      top_logprob[row * k + i] = bad ? NAN : -INFINITY;
    }
  }
}

// Beyond this |lse| its rounding (2^-24 of it) would show in p: rows whose mask is the type's
// lowest value throughout have an lse that has lost ln s, and take the largest logit and ln s from
// the row. The product of that logit and the scale has a rounding of the same size, so lp is then
// (x - max x) scale - ln s: the difference comes first, as in the sums.
constexpr float kLargeLse = 1024.f;

// With lp_j = z_j - lse and p_j = exp(lp_j):
//   dlogits_j = p_j (A + B lp_j) + scale g [j = t],  A = -scale (g + gh H),  B = -scale gh.
// A row per cluster of CS blocks; pieces as in the forward pass, but of the gradient's row (the
// logits' row may start elsewhere against a 16-byte boundary).
template <class T>
__global__ void __launch_bounds__(kThreads, 4)
    token_logprobs_grad_kernel(const T *logits, int V, long long ld, const long long *targets,
                               float scale, const float *lse, const float *entropy,
                               const float *g_logprob, const float *g_entropy, T *dlogits,
                               long long ldd, int CS) {
  constexpr int N = Piece<T>::N, SPAN = Piece<T>::SPAN;
  __shared__ Sums wsum[kThreads / 32];
  __shared__ float csum[kMaxCluster][3];
  pdl_wait();
  pdl_trigger();
  const int W = blockDim.x / 32, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rank = CS > 1 ? blockIdx.x % CS : 0;
  const long long row = blockIdx.x / CS;
  const T *x = logits + row * ld;
  T *dx = dlogits + row * ldd;
  const int off = (int)((uintptr_t)dx % 16 / sizeof(T));
  const int shift = (int)(((uintptr_t)x - off * sizeof(T)) % 16);  // of a piece's first logit
  const int Q = Piece<T>::count(off, V), step = CS * W, first = rank * W + warp;
  const int whole0 = off ? 1 : 0, whole1 = (off + V) / SPAN;
  auto load = [&](int q) {
    return shift == 0 && q >= whole0 && q < whole1
               ? load_whole(x, V, (long long)q * SPAN - off)
               : load_piece(x, V, q * SPAN - off, shift);
  };
  const long long t = targets[row];
  const float l = lse[row];
  float g = t < 0 ? 0.f : t >= V ? NAN : g_logprob[row];
  float gh = g_entropy ? g_entropy[row] : 0.f, H = g_entropy ? entropy[row] : 0.f;
  if (l == -INFINITY && t < V) g = gh = H = 0.f;
  if (isnan(l)) g = NAN;
  float m = 0.f, ls = l == -INFINITY ? 0.f : l;  // lp = (x - m) scale - ls
  if (fabsf(l) > kLargeLse && isfinite(l)) {
    if (CS > 1) cluster_begin();  // (l is the row's: all of its blocks are here, or none)
    const float c = fminf(scale * kLog2e, FLT_MAX);
    Sums a = {-INFINITY, 0.f, 0.f};
    for (int q = first; q < Q; q += step) {
      const Piece<T> p = load(q);
      const float top = fmaxf(a.m, lane_max(p));
      a.move(top, c);
      unsigned long long s2 = 0ull, u2 = 0ull;
      if (top > -INFINITY) sum_piece<true>(p, top, c, s2, u2);
      float s, t2;
      f2_split(s2, s, t2);
      a.s += s + t2;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1)
      a = join(a, {__shfl_xor_sync(kAll, a.m, o), __shfl_xor_sync(kAll, a.s, o), 0.f}, c);
    if (lane == 0) wsum[warp] = a;
    __syncthreads();
    a = wsum[0];
    for (int w = 1; w < W; ++w) a = join(a, wsum[w], c);
    if (CS > 1) {
      // (every block has read its part of the row before any writes: in place)
      cluster_runs();
      if (threadIdx.x < CS && BOUTE_INB(rank, kMaxCluster)) {
        store_peer(peer(&csum[rank][0], threadIdx.x), a.m);
        store_peer(peer(&csum[rank][1], threadIdx.x), a.s);
      }
      cluster_sync();
      a = {csum[0][0], csum[0][1], 0.f};
      for (int b = 1; b < CS; ++b) a = join(a, {csum[b][0], csum[b][1], 0.f}, c);
    }
    m = a.m;
    ls = logf(a.s);
  }
  const float A = -scale * (g + gh * H), B = -scale * gh, extra = scale * g;
  const unsigned long long A2 = f2_dup(A), B2 = f2_dup(B), c2 = f2_dup(scale), m2 = f2_dup(m),
                           ls2 = f2_dup(-ls), e2 = f2_dup(kLog2e);
  for (int q = first; q < Q; q += step) {
    Piece<T> p = load(q);
    const int at0 = q * SPAN - off;
    const bool target = t >= at0 && t < at0 + SPAN;
#pragma unroll
    for (int j = 0; j < N / 2; ++j) {
      float a, b;
      pair(p, j, a, b);
      f2_split(f2_fma(f2_sub(f2_pack(a, b), m2), c2, ls2), a, b);
      const unsigned long long lp = f2_pack(fmaxf(a, kLowest), fmaxf(b, kLowest));
      f2_split(f2_mul(lp, e2), a, b);
      const unsigned long long e = f2_pack(exp2_fast(a), exp2_fast(b));
      f2_split(f2_mul(e, f2_fma(B2, lp, A2)), a, b);
      if (target) {
        const int d = (int)(t - at0) - Piece<T>::index(2 * j);
        a += d == 0 ? extra : 0.f;
        b += d == 1 ? extra : 0.f;
      }
      set_pair(p, j, a, b);
    }
    store_piece(dx, V, at0, p);
  }
}

}  // namespace

BOUTE_BOUNDS_READER(logprobs)

}  // namespace boute

using namespace boute;

// How a row's pieces are spread: a warp per piece, up to kWarps to a block, and the blocks of a
// cluster while the rows alone leave the SMs without work and every warp gets a piece; with rows
// so few that all their warps run at once, twice the warps.
// (us by the most blocks an SM that clusters may make of rows, 4, 8 or 16: 600 x 131072 bf16,
// k = 8: 36, 31, 41; 256 x 131072, k = 20: 23, 19, 24. Warps to a block, 2, 4 or 8: 2039 x 50021
// fp16, k = 8: 44, 43, 46; 2500 x 32000 bf16, k = 5: 42, 38, 41.)
struct Spread {
  int W, CS;
  template <class P>
  Spread(long long T, int V, P) {
    const int Q = P::count(P::E - 1, V), sms = num_sms();
    W = Q < kWarps ? Q : kWarps;
    CS = 1;
    while (CS < kMaxCluster && 2 * CS * T <= 8 * sms && 2 * CS * W <= Q) CS *= 2;
    if (CS == kMaxCluster && 2 * W * CS * T <= 32 * sms && CS * W < Q) W *= 2;
  }
  // Many short rows: what follows a row's loads takes as long as they do, and rows of one warp (of
  // two, where many alternatives are ranked) have more of it going on at once. (us by 1, 2 and 4
  // warps: 9000 x 8000 bf16, k = 4: 40, 44, 54, k = 20: 62, 58, 64, k = 0: 28, 29, 30; 20000 x
  // 32000, k = 4: 220, 218, 235, k = 0: 200, 194, 193; 5000 x 13000, k = 20: 57, 47, 46.)
  template <class P>
  void for_alternatives(long long T, int V, int k, P) {
    const int Q = P::count(P::E - 1, V), few = k <= 8 ? 1 : 2;
    if (T >= 48ll * num_sms() && Q <= (k ? 32 : 8)) W = W < few ? W : few;
  }
};

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
    Spread sp(T, V, Piece<E>{});
    sp.for_alternatives(T, V, k, Piece<E>{});
    return launch_cluster(token_logprobs_kernel<E>, T * sp.CS, 32 * sp.W, sp.CS, 0,
                          (cudaStream_t)stream, (const E *)logits, V, ld, targets, scale, k, sp.CS,
                          logprob, entropy, lse, top_idx, top_logprob);
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
    const Spread sp(T, V, Piece<E>{});
    return launch_cluster(token_logprobs_grad_kernel<E>, T * sp.CS, 32 * sp.W, sp.CS, 0,
                          (cudaStream_t)stream, (const E *)logits, V, ld, targets, scale, lse,
                          entropy, g_logprob, g_entropy, (E *)dlogits, ldd, sp.CS);
  });
}
