// Log-probabilities of given tokens, with the entropy and the top alternatives
// of every position, and the gradient with respect to the logits.
//
// With z = scale x, m = max z, s = sum exp(z - m) and u = sum (z - m) exp(z - m):
//   lse = m + ln s,  logprob = z_t - m - ln s,  entropy = ln s - u / s.
// One pass over a row: each warp keeps a running maximum and s and u relative to
// it, and leaves the maximum of every chunk of 256 logits. The k-th largest of
// the lanes' own maxima is reached by k logits at least, and by few others; only
// the chunks whose maximum reaches it are read again, and what reaches it there
// is ranked. A row is a block's, or a cluster's when there are few rows.
#include <float.h>
#include <math.h>

#include "answers.cuh"

namespace boute {

namespace {

constexpr unsigned kAll = 0xffffffffu;
constexpr int kThreads = 256;   // of a block that has as many chunks
constexpr int kChunk = 256;     // logits a warp reads at a time
constexpr int kMaxCluster = 8;
constexpr float kLowest = -200.f;  // exp(kLowest) = 2^kLowest = 0 in fp32
constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(kAll, v, o);
  return v;
}
// The warp's maximum in one instruction; a NaN anywhere wins.
__device__ __forceinline__ float warp_max_nan(float v) {
  float r;
  asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
  return r;
}
__device__ __forceinline__ float max_nan(float a, float b) {
  float r;
  asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float exp2_fast(float y) {  // (2 ulp; what is below 2^-126 is 0)
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(y));
  return r;
}

// ---- clusters (a block launched alone is a cluster of one) ---------------------------
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::
                   : "memory");
}
// Address of block r's copy of a shared variable.
__device__ __forceinline__ uint32_t peer(const void *p, int r) {
  uint32_t a;
  asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(r));
  return a;
}
__device__ __forceinline__ void store_peer(uint32_t a, float v) {
  asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(a), "f"(v) : "memory");
}
__device__ __forceinline__ void store_peer(uint32_t a, unsigned long long v) {
  asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}
__device__ __forceinline__ int add_peer(uint32_t a, int v) {
  int old;
  asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(a), "r"(v) : "memory");
  return old;
}

// ---- a row in chunks -----------------------------------------------------------------
// Chunk c holds the logits [256 c - off, 256 c - off + 256) of a row whose first logit lies
// `off` elements after a 16-byte boundary, so that every chunk starts on one. A lane holds one
// 16-byte vector of it (16-bit logits) or two (fp32).
template <class T>
struct Chunk {
  static constexpr int E = 16 / sizeof(T), VPL = kChunk / (32 * E);
  uint4 v[VPL];
  static __device__ __forceinline__ int index(int i, int e) {  // within the chunk
    return (i * 32 + (threadIdx.x & 31)) * E + e;
  }
};

template <class T>
struct Row {
  const T *x;
  int off, V;
  __device__ __forceinline__ Row(const T *row, int V_) : x(row), V(V_) {
    off = (int)((uintptr_t)row % 16 / sizeof(T));
  }
  static __host__ __device__ int chunks(int off, int V) { return (off + V + kChunk - 1) / kChunk; }
  // -inf outside the row; nothing outside the row is read
  __device__ __forceinline__ Chunk<T> load(int c) const {
    Chunk<T> r;
    const int first = c * kChunk - off;
    if (first >= 0 && first + kChunk <= V) {
#pragma unroll
      for (int i = 0; i < Chunk<T>::VPL; ++i)
        r.v[i] = *(const uint4 *)(x + first + Chunk<T>::index(i, 0));
    } else {
      T t[Chunk<T>::E];
#pragma unroll
      for (int i = 0; i < Chunk<T>::VPL; ++i) {
#pragma unroll
        for (int e = 0; e < Chunk<T>::E; ++e) {
          const int j = first + Chunk<T>::index(i, e);
          t[e] = j >= 0 && j < V ? x[j] : from_float<T>(-INFINITY);
        }
        memcpy(&r.v[i], t, 16);
      }
    }
    return r;
  }
};

// The chunk of another row y of the same length whose chunks lie elsewhere: from the logit y
// holds at `first` on, `shift` bytes after a 16-byte boundary in y.
template <class T>
__device__ __forceinline__ Chunk<T> load_shifted(const T *y, int V, int first, int shift) {
  constexpr int E = Chunk<T>::E;
  Chunk<T> r;
  if (first >= E && first + kChunk + E <= V) {
#pragma unroll
    for (int i = 0; i < Chunk<T>::VPL; ++i) {
      const char *p = (const char *)(y + first + Chunk<T>::index(i, 0)) - shift;
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
    }
  } else {
    T t[E];
#pragma unroll
    for (int i = 0; i < Chunk<T>::VPL; ++i) {
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const int j = first + Chunk<T>::index(i, e);
        t[e] = j >= 0 && j < V ? y[j] : from_float<T>(-INFINITY);
      }
      memcpy(&r.v[i], t, 16);
    }
  }
  return r;
}
// Chunk c of the row at y (off elements after a boundary); nothing outside the row is written.
template <class T>
__device__ __forceinline__ void store(T *y, int off, int V, int c, const Chunk<T> &r) {
  const int first = c * kChunk - off;
  if (first >= 0 && first + kChunk <= V) {
#pragma unroll
    for (int i = 0; i < Chunk<T>::VPL; ++i)
      *(uint4 *)(y + first + Chunk<T>::index(i, 0)) = r.v[i];
  } else {
    T t[Chunk<T>::E];
#pragma unroll
    for (int i = 0; i < Chunk<T>::VPL; ++i) {
      memcpy(t, &r.v[i], 16);
#pragma unroll
      for (int e = 0; e < Chunk<T>::E; ++e) {
        const int j = first + Chunk<T>::index(i, e);
        if (j >= 0 && j < V) y[j] = t[e];
      }
    }
  }
}

// A lane's 8 (VPL x E) logits of a chunk as floats, and back (one rounding).
__device__ __forceinline__ void unpack2(uint32_t w, float &a, float &b, __nv_bfloat16) {
  a = __uint_as_float(w << 16);
  b = __uint_as_float(w & 0xffff0000u);
}
__device__ __forceinline__ void unpack2(uint32_t w, float &a, float &b, __half) {
  unpack_f16x2(w, a, b);
}
template <class T>
__device__ __forceinline__ void values(const Chunk<T> &c, float (&x)[8]) {
#pragma unroll
  for (int i = 0; i < Chunk<T>::VPL; ++i) {
    const uint32_t w[4] = {c.v[i].x, c.v[i].y, c.v[i].z, c.v[i].w};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (sizeof(T) == 4) x[4 * i + q] = __uint_as_float(w[q]);
      else unpack2(w[q], x[2 * q], x[2 * q + 1], T{});
    }
  }
}
__device__ __forceinline__ uint32_t pack2(float a, float b, __half) { return pack_f16x2(a, b); }
__device__ __forceinline__ uint32_t pack2(float a, float b, __nv_bfloat16) {
  uint32_t r;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(b), "f"(a));
  return r;
}
template <class T>
__device__ __forceinline__ Chunk<T> chunk_of(const float (&x)[8]) {
  Chunk<T> c;
#pragma unroll
  for (int i = 0; i < Chunk<T>::VPL; ++i) {
    uint32_t w[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      if constexpr (sizeof(T) == 4) w[q] = __float_as_uint(x[4 * i + q]);
      else w[q] = pack2(x[2 * q], x[2 * q + 1], T{});
    }
    c.v[i] = {w[0], w[1], w[2], w[3]};
  }
  return c;
}
// A lane's largest logit of a chunk, NaN if it holds one.
__device__ __forceinline__ float lane_max(const Chunk<float> &c) {
  float x[8];
  values(c, x);
#pragma unroll
  for (int o = 4; o > 0; o >>= 1)
#pragma unroll
    for (int i = 0; i < o; ++i) x[i] = max_nan(x[i], x[i + o]);
  return x[0];
}
template <class H2, class T>
__device__ __forceinline__ float lane_max16(const Chunk<T> &c) {
  H2 h[4];
  memcpy(h, &c.v[0], 16);
  const H2 m = __hmax2_nan(__hmax2_nan(h[0], h[1]), __hmax2_nan(h[2], h[3]));
  return max_nan(to_float(m.x), to_float(m.y));
}
__device__ __forceinline__ float lane_max(const Chunk<__half> &c) {
  return lane_max16<__half2>(c);
}
__device__ __forceinline__ float lane_max(const Chunk<__nv_bfloat16> &c) {
  return lane_max16<__nv_bfloat162>(c);
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

// Order-preserving bits; of -inf at least, which is below every logit.
__device__ __forceinline__ unsigned order_bits(float v) {
  const unsigned u = __float_as_uint(v);
  return (u & 0x80000000u) ? ~u : (u | 0x80000000u);
}
__device__ __forceinline__ float from_order_bits(unsigned o) {
  return __uint_as_float((o & 0x80000000u) ? o & 0x7fffffffu : ~o);
}

// A value that k of the block's threads reach with theirs, close to the largest such one: built
// bit by bit until exactly k reach it. -inf where fewer than k have one.
__device__ __forceinline__ float kth_bound(float mine, int k) {
  const unsigned o = order_bits(mine);
  unsigned t = 0u;
  for (unsigned bit = 1u << 31; bit; bit >>= 1) {
    const int n = __syncthreads_count(o >= (t | bit));
    if (n >= k) t |= bit;
    if (n == k) break;
  }
  return from_order_bits(max(t, order_bits(-INFINITY)));
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

// A row per cluster of CS blocks; chunk c is warp (c mod CS W)'s, in order.
template <class T>
__global__ void __launch_bounds__(kThreads, 4)
    token_logprobs_kernel(const T *logits, int V, long long ld, const long long *targets,
                          float scale, int k, int CS, int per_warp, float *logprob,
                          float *entropy, float *lse, long long *top_idx, float *top_logprob) {
  constexpr int U = sizeof(T) == 4 ? 2 : 4;  // chunks in flight: 64 bytes a lane
  extern __shared__ unsigned long long list[];  // the leader's: CS W 32 candidates' keys
  __shared__ Sums wsum[kThreads / 32];
  __shared__ float csum[kMaxCluster][3], ctau[kMaxCluster];
  __shared__ int nlist;
  const int W = blockDim.x / 32, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int rank = CS > 1 ? blockIdx.x % CS : 0;
  const long long row = blockIdx.x / CS;
  const Row<T> r(logits + row * ld, V);
  const float c = fminf(scale * kLog2e, FLT_MAX);
  float *cmax = (float *)(list + CS * W * 32) + warp * per_warp;  // this warp's chunks' maxima
  if (tid == 0) nlist = 0;

  const int C = Row<T>::chunks(r.off, V), step = CS * W, first = rank * W + warp;
  float m = -INFINITY, top = -INFINITY;
  unsigned long long s2 = 0ull, u2 = 0ull;  // pairs of partial sums
  for (int i = 0; i < per_warp; i += U) {
    Chunk<T> v[U];
    float cm[U], g = -INFINITY;
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = r.load(first + (i + u) * step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float l = lane_max(v[u]);
      top = max_nan(top, l);
      cm[u] = warp_max_nan(l);
      g = max_nan(g, cm[u]);
    }
    if (lane == 0 && k > 0)
#pragma unroll
      for (int u = 0; u < U; ++u) cmax[i + u] = cm[u];
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
    if (m == -INFINITY) continue;
    const unsigned long long m2 = f2_dup(m), c2 = f2_dup(c);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[8];
      values(v[u], x);
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float y0, y1;
        f2_split(f2_mul(f2_sub(f2_pack(x[e], x[e + 1]), m2), c2), y0, y1);
        y0 = fmaxf(y0, kLowest);
        y1 = fmaxf(y1, kLowest);
        const unsigned long long p = f2_pack(exp2_fast(y0), exp2_fast(y1));
        s2 = f2_add(s2, p);
        u2 = f2_fma(f2_pack(y0, y1), p, u2);
      }
    }
  }
  {
    float a, b;
    f2_split(s2, a, b);
    const float s = warp_sum(a + b);
    f2_split(u2, a, b);
    const float u = warp_sum(a + b);
    if (lane == 0) wsum[warp] = {m, s, u};
  }
  float tau = -INFINITY;
  if (k > 0) tau = kth_bound(top, k);
  __syncthreads();
  if (CS > 1) {
    if (tid == 0) {
      Sums a = wsum[0];
      for (int w = 1; w < W; ++w) {
        if (isnan(wsum[w].m)) a.m = NAN;
        a = isnan(a.m) ? a : join(a, wsum[w], c);
      }
      store_peer(peer(&csum[rank][0], 0), a.m);
      store_peer(peer(&csum[rank][1], 0), a.s);
      store_peer(peer(&csum[rank][2], 0), a.u);
    }
    if (tid < CS) store_peer(peer(&ctau[rank], tid), tau);
    cluster_sync();
    for (int b = 0; b < CS; ++b) tau = fmaxf(tau, ctau[b]);
  }
  if (k > 0) {
    // the chunks that reach tau, read again
    const float zt = __fmul_rn(tau, scale);
    WarpBest best;
    for (int i0 = 0; i0 < per_warp; i0 += 32) {
      const float cm = i0 + lane < per_warp ? __fmul_rn(cmax[i0 + lane], scale) : -INFINITY;
      unsigned hit = __ballot_sync(kAll, cm >= zt && cm > -INFINITY);
      while (hit) {
        const int ch = first + (i0 + __ffs(hit) - 1) * step;
        hit &= hit - 1;
        if (ch >= C) continue;
        const Chunk<T> v = r.load(ch);
        float x[8];
        values(v, x);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = __fmul_rn(x[e], scale);
          const int j = ch * kChunk - r.off + Chunk<T>::index(e / Chunk<T>::E, e % Chunk<T>::E);
          best.feed(z >= zt && z > -INFINITY, make_key(z, (unsigned)j), k, lane);
        }
      }
    }
    best.batch.flush(lane);
    const unsigned have = __ballot_sync(kAll, lane < k && best.batch.top != 0ull);
    if (have) {
      int at = 0;
      if (lane == 0) at = add_peer(peer(&nlist, 0), __popc(have));
      at = __shfl_sync(kAll, at, 0) + lane;
      if ((have >> lane & 1u) && BOUTE_INB(at, CS * W * 32))
        store_peer(peer(list, 0) + 8u * at, best.batch.top);
    }
    if (CS > 1) cluster_sync();
    else __syncthreads();
  }
  if (rank != 0) return;
  Sums a = CS > 1 ? Sums{csum[0][0], csum[0][1], csum[0][2]} : wsum[0];
  bool bad = isnan(a.m);
  for (int w = 1; w < (CS > 1 ? CS : W); ++w) {
    const Sums b = CS > 1 ? Sums{csum[w][0], csum[w][1], csum[w][2]} : wsum[w];
    bad |= isnan(b.m);
    a = join(a, b, c);
  }
  const float M = __fmul_rn(a.m, scale);
  const bool empty = M == -INFINITY;  // (scaled values that underflow the type are masked too)
  bad |= M == INFINITY;
  const float ls = empty ? 0.f : logf(a.s);
  if (tid == 0) {
    const long long t = targets[row];
    float lp = 0.f;
    if (t >= V || (bad && t >= 0)) lp = NAN;
    else if (t >= 0 && BOUTE_INB(t, V))
      lp = empty ? -INFINITY : __fmul_rn(to_float(r.x[t]), scale) - M - ls;
    lse[row] = bad ? NAN : M + ls;
    logprob[row] = lp;
    entropy[row] = bad ? NAN : empty ? 0.f : ls - kLn2 * (a.u / a.s);
  }
  if (k > 0) {
    const int n = bad || empty ? 0 : nlist;
    for (int i = tid; i < n; i += blockDim.x) {
      const unsigned long long key = list[i];
      int place = 0;
      for (int j = 0; j < n; ++j) place += list[j] > key;
      if (place < k) {
        top_idx[row * k + place] = (long long)key_index(key);
        top_logprob[row * k + place] = from_order_bits((unsigned)(key >> 32)) - M - ls;
      }
    }
    for (int i = n + tid; i < k; i += blockDim.x) {
      top_idx[row * k + i] = -1;
      top_logprob[row * k + i] = bad ? NAN : -INFINITY;
    }
  }
}

// Beyond this |lse| its rounding (2^-24 of it) would show in p: rows whose mask is the type's
// lowest value throughout have an lse that has lost ln s, and take m and ln s from the row.
constexpr float kLargeLse = 1024.f;

// With lp_j = z_j - lse and p_j = exp(lp_j):
//   dlogits_j = p_j (A + B lp_j) + scale g [j = t],  A = -scale (g + gh H),  B = -scale gh.
// A row per cluster of CS blocks; chunks as in the forward pass, but of the gradient's row (the
// logits' row may start elsewhere against a 16-byte boundary).
template <class T>
__global__ void __launch_bounds__(kThreads, 4)
    token_logprobs_grad_kernel(const T *logits, int V, long long ld, const long long *targets,
                               float scale, const float *lse, const float *entropy,
                               const float *g_logprob, const float *g_entropy, T *dlogits,
                               long long ldd, int CS, int per_warp) {
  constexpr int U = sizeof(T) == 4 ? 2 : 4;
  __shared__ Sums wsum[kThreads / 32];
  __shared__ float csum[kMaxCluster][3];
  const int W = blockDim.x / 32, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int rank = CS > 1 ? blockIdx.x % CS : 0;
  const long long row = blockIdx.x / CS;
  const T *x = logits + row * ld;
  T *dx = dlogits + row * ldd;
  const int off = (int)((uintptr_t)dx % 16 / sizeof(T));
  const int shift = (int)(((uintptr_t)x - off * sizeof(T)) % 16);  // of a chunk's first logit
  const int C = Row<T>::chunks(off, V), step = CS * W, first = rank * W + warp;
  const long long t = targets[row];
  const float l = lse[row];
  float g = t < 0 ? 0.f : t >= V || isnan(l) ? NAN : g_logprob[row];
  float gh = g_entropy ? g_entropy[row] : 0.f, H = g_entropy ? entropy[row] : 0.f;
  if (l == -INFINITY && t < V) g = gh = H = 0.f;
  if (isnan(l)) g = NAN;
  float m = l == -INFINITY ? 0.f : l, ls = 0.f;  // lse = m + ls
  auto load = [&](int ch) {
    return shift ? load_shifted(x, V, ch * kChunk - off, shift) : [&] {
      Row<T> r(x, V);
      r.off = off;
      return r.load(ch);
    }();
  };
  if (fabsf(l) > kLargeLse && isfinite(l)) {
    const float c = fminf(scale * kLog2e, FLT_MAX);
    Sums a = {-INFINITY, 0.f, 0.f};
    for (int ch = first; ch < C; ch += step) {
      const Chunk<T> v = load(ch);
      float z[8];
      values(v, z);
      const float top = fmaxf(a.m, lane_max(v));
      a.move(top, c);
      if (top > -INFINITY)
#pragma unroll
        for (int e = 0; e < 8; ++e) a.s += exp2_fast(fmaxf((z[e] - top) * c, kLowest));
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
      if (threadIdx.x < CS) {
        store_peer(peer(&csum[rank][0], threadIdx.x), a.m);
        store_peer(peer(&csum[rank][1], threadIdx.x), a.s);
      }
      cluster_sync();
      a = {csum[0][0], csum[0][1], 0.f};
      for (int b = 1; b < CS; ++b) a = join(a, {csum[b][0], csum[b][1], 0.f}, c);
    }
    m = __fmul_rn(a.m, scale);
    ls = logf(a.s);
  }
  const float A = -scale * (g + gh * H), B = -scale * gh, hit = scale * g;
  const unsigned long long A2 = f2_dup(A), B2 = f2_dup(B), c2 = f2_dup(scale), m2 = f2_dup(-m),
                           ls2 = f2_dup(ls), e2 = f2_dup(kLog2e);
  for (int i = 0; i < per_warp; i += U) {
    Chunk<T> v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = load(first + (i + u) * step);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int ch = first + (i + u) * step;
      if (ch >= C) break;
      float z[8];
      values(v[u], z);
#pragma unroll
      for (int e = 0; e < 8; e += 2) {
        float a, b;
        f2_split(f2_sub(f2_fma(f2_pack(z[e], z[e + 1]), c2, m2), ls2), a, b);
        const unsigned long long lp = f2_pack(fmaxf(a, kLowest), fmaxf(b, kLowest));
        f2_split(f2_mul(lp, e2), a, b);
        const unsigned long long p = f2_pack(exp2_fast(a), exp2_fast(b));
        f2_split(f2_mul(p, f2_fma(B2, lp, A2)), z[e], z[e + 1]);
      }
      const long long at = t - ((long long)ch * kChunk - off);
      if (at >= 0 && at < kChunk)
#pragma unroll
        for (int e = 0; e < 8; ++e)
          z[e] += Chunk<T>::index(e / Chunk<T>::E, e % Chunk<T>::E) == at ? hit : 0.f;
      store(dx, off, V, ch, chunk_of<T>(z));
    }
  }
}

}  // namespace

BOUTE_BOUNDS_READER(logprobs)

}  // namespace boute

using namespace boute;

// How a row's chunks are spread: a warp per chunk, up to eight to a block, and the blocks of a
// cluster while the rows alone leave the SMs without work and every warp gets a few chunks.
struct Spread {
  int W, CS, per_warp;
  Spread(long long T, int V, size_t bytes) {
    const int C = ((int)(16 / bytes) - 1 + V + kChunk - 1) / kChunk;
    W = C < kThreads / 32 ? C : kThreads / 32;
    CS = 1;
    const int sms = num_sms();
    while (CS < kMaxCluster && 2 * CS * T <= 4 * sms && 4 * CS * W <= C) CS *= 2;
    per_warp = round_up((C + CS * W - 1) / (CS * W), bytes == 4 ? 2 : 4);
  }
};

template <class... KArgs, class... Args>
static int launch_rows(void (*kernel)(KArgs...), const Spread &sp, long long T, size_t smem,
                       cudaStream_t s, Args &&...args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)(T * sp.CS));
  cfg.blockDim = dim3(32 * sp.W);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = sp.CS;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = sp.CS > 1;
  cudaLaunchKernelEx(&cfg, kernel, static_cast<KArgs>(args)...);
  count_launch();
  return last_launch_status();
}

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
    const Spread sp(T, V, sizeof(E));
    const size_t smem = (size_t)sp.W * (sp.CS * 32 * 8 + sp.per_warp * 4);
    return launch_rows(token_logprobs_kernel<E>, sp, T, smem, (cudaStream_t)stream,
                       (const E *)logits, V, ld, targets, scale, k, sp.CS, sp.per_warp, logprob,
                       entropy, lse, top_idx, top_logprob);
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
    const Spread sp(T, V, sizeof(E));
    return launch_rows(token_logprobs_grad_kernel<E>, sp, T, 0, (cudaStream_t)stream,
                       (const E *)logits, V, ld, targets, scale, lse, entropy, g_logprob,
                       g_entropy, (E *)dlogits, ldd, sp.CS, sp.per_warp);
  });
}
