// Between a routing and its experts: the choices in the order of their experts, the queries'
// rows copied there, the experts' rows summed back with the routing's weights, and the gradients.
//
// Memory bounds all but the smallest calls.
#include <algorithm>
#include <type_traits>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;

// ---- the order -----------------------------------------------------------------------
// A stable counting sort by expert; a choice of no expert counts as one of expert E, whose places
// follow all others. A block has up to kChunk choices, kSteps to a lane: a warp's neighbours of equal
// expert are found by one match and counted behind the warp's earlier ones, so a choice's rank among
// its block's is known after one pass. Up to a cluster's blocks the counts are joined through shared
// memory, in one launch. More choices take three: the blocks' counts, their sums before each block,
// and the places; a block's counts lie in its own part of `place` until it writes that.
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32, kSteps = 8;
constexpr int kChunk = kSortThreads * kSteps, kMaxCluster = 8;
constexpr int kScanThreads = 1024;

struct Order {
  const int *idx;
  long long N;
  int E, blocks;
  int *offsets, *source, *place;

  // block b's choices (the chunks of more than a cluster's blocks hold E + 1 at least)
  __host__ __device__ long long first(int b) const { return (long long)b * N / blocks; }
  // an expert, or E for none
  __device__ __forceinline__ int expert(long long c) const {
    const int e = BOUTE_INB(c, N) ? idx[c] : -1;
    return (unsigned)e < (unsigned)E ? e : E;
  }
};

// hist: kSortWarps x (E + 1) counts of the warps' choices; key, rank: of each of the lane's.
__device__ __forceinline__ void count_choices(const Order &A, int b, int *hist, int (&key)[kSteps],
                                              int (&rank)[kSteps]) {
  const int E1 = A.E + 1, tid = threadIdx.x, lane = tid & 31;
  const long long from = A.first(b) + (tid / 32) * (32 * kSteps), end = A.first(b + 1);
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const long long c = from + j * 32 + lane;
    key[j] = c < end ? A.expert(c) : -1;
  }
  for (int i = tid; i < kSortWarps * E1; i += kSortThreads) hist[i] = 0;
  __syncthreads();
  int *mine = hist + (tid / 32) * E1;
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const unsigned peers = __match_any_sync(kAll, key[j]);
    const int before = __popc(peers & ((1u << lane) - 1u));
    int had = 0;
    if (key[j] >= 0 && BOUTE_INB(key[j], E1)) had = mine[key[j]];
    __syncwarp();
    if (key[j] >= 0 && before == 0) mine[key[j]] = had + __popc(peers);
    __syncwarp();
    rank[j] = had + before;
  }
  __syncthreads();
}

// Each lane's choices to their places: hist holds the first place of each warp's choices of an expert.
__device__ __forceinline__ void place_choices(const Order &A, int b, const int *hist,
                                              const int (&key)[kSteps], const int (&rank)[kSteps]) {
  const int E1 = A.E + 1, tid = threadIdx.x, lane = tid & 31;
  const long long from = A.first(b) + (tid / 32) * (32 * kSteps);
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    if (key[j] < 0) continue;
    const int c = (int)(from + j * 32 + lane), at = hist[(tid / 32) * E1 + key[j]] + rank[j];
    if (!BOUTE_INB(c, A.N) || !BOUTE_INB(at, A.N)) continue;
    A.place[c] = key[j] < A.E ? at : -1;
    A.source[at] = key[j] < A.E ? c : -1;
  }
}

// v[0 .. n) becomes the sums before each, in place; the block's threads all come.
template <int THREADS>
__device__ __forceinline__ void block_scan(int *v, int n, int *warp_sums) {
  const int tid = threadIdx.x, lane = tid & 31, per = (n + THREADS - 1) / THREADS;
  const int a = min(tid * per, n), b = min(a + per, n);
  int sum = 0;
  for (int i = a; i < b; ++i) sum += v[i];
  int up = sum;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kAll, up, o);
    if (lane >= o) up += x;
  }
  if (lane == 31) warp_sums[tid / 32] = up;
  __syncthreads();
  int before = up - sum;
  for (int w = 0; w < tid / 32; ++w) before += warp_sums[w];
  for (int i = a; i < b; ++i) {
    const int x = v[i];
    v[i] = before;
    before += x;
  }
  __syncthreads();
}

__device__ __forceinline__ int load_peer(uint32_t a) {
  int v;
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
  return v;
}

// One cluster. Shared memory: kSortWarps x (E + 1) counts, the block's counts, the experts' first places.
__global__ void __launch_bounds__(kSortThreads) expert_sort_kernel(Order A) {
  extern __shared__ int sort_smem[];
  __shared__ int warp_sums[kSortWarps];
  pdl_wait();
  pdl_trigger();
  const int E1 = A.E + 1, tid = threadIdx.x, b = blockIdx.x;
  int *hist = sort_smem, *count = hist + kSortWarps * E1, *first = count + E1;
  int key[kSteps], rank[kSteps];
  count_choices(A, b, hist, key, rank);
  for (int e = tid; e < E1; e += kSortThreads) {
    int n = 0;
    for (int w = 0; w < kSortWarps; ++w) n += hist[w * E1 + e];
    first[e] = count[e] = n;
  }
  int before_e[(BOUTE_MAX_EXPERTS + kSortThreads) / kSortThreads];  // of my experts, in lower blocks
#pragma unroll
  for (int i = 0; i < (int)(sizeof(before_e) / sizeof(int)); ++i) before_e[i] = 0;
  if (A.blocks > 1) {
    cluster_sync();
#pragma unroll
    for (int i = 0; i < (int)(sizeof(before_e) / sizeof(int)); ++i) {
      const int e = tid + i * kSortThreads;
      if (e >= E1) break;
      int all = 0;
      for (int r = 0; r < A.blocks; ++r) {
        const int n = load_peer(peer(&count[e], r));
        if (r < b) before_e[i] += n;
        all += n;
      }
      first[e] = all;
    }
  }
  __syncthreads();
  block_scan<kSortThreads>(first, E1, warp_sums);
#pragma unroll
  for (int i = 0; i < (int)(sizeof(before_e) / sizeof(int)); ++i) {
    const int e = tid + i * kSortThreads;
    if (e >= E1) break;
    if (b == 0) A.offsets[e] = first[e];
    int at = first[e] + before_e[i];
    for (int w = 0; w < kSortWarps; ++w) {
      const int n = hist[w * E1 + e];
      hist[w * E1 + e] = at;
      at += n;
    }
  }
  __syncthreads();
  place_choices(A, b, hist, key, rank);
  if (A.blocks > 1) cluster_sync();  // (the others may read this block's counts until here)
}

// The blocks' counts, each in its own part of `place`.
__global__ void __launch_bounds__(kSortThreads) expert_count_kernel(Order A) {
  __shared__ int hist[BOUTE_MAX_EXPERTS + 1];
  pdl_wait();
  pdl_trigger();
  const int E1 = A.E + 1, tid = threadIdx.x;
  const long long from = A.first(blockIdx.x), end = A.first(blockIdx.x + 1);
  int key[kSteps];
#pragma unroll
  for (int j = 0; j < kSteps; ++j) {
    const long long c = from + j * kSortThreads + tid;
    key[j] = c < end ? A.expert(c) : -1;
  }
  for (int e = tid; e < E1; e += kSortThreads) hist[e] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < kSteps; ++j)
    if (key[j] >= 0) atomicAdd(&hist[key[j]], 1);
  __syncthreads();
  for (int e = tid; e < E1; e += kSortThreads)
    if (BOUTE_INB(from + e, end)) A.place[from + e] = hist[e];
}

// One cluster: the counts become the first places of each block's choices of an expert. A block of
// the cluster has a part of the experts, a thread a run of the blocks for one of them.
__global__ void __launch_bounds__(kScanThreads) expert_scan_kernel(Order A) {
  __shared__ int runs[kScanThreads], total[BOUTE_MAX_EXPERTS / kMaxCluster + 1];
  __shared__ int first[BOUTE_MAX_EXPERTS + 1], warp_sums[kScanThreads / 32];
  pdl_wait();
  pdl_trigger();
  const int E1 = A.E + 1, tid = threadIdx.x, rank = blockIdx.x;
  const int part = (E1 + kMaxCluster - 1) / kMaxCluster;  // experts of a block
  const int e0 = rank * part, mine = max(0, min(part, E1 - e0));
  const int per = min(kScanThreads / part, 64), i = tid % part, r = tid / part;  // runs of an expert
  const int len = (A.blocks + per - 1) / per;
  const int b0 = min(r * len, A.blocks), b1 = r < per && i < mine ? min(b0 + len, A.blocks) : b0;
  int sum = 0;
#pragma unroll 4
  for (int b = b0; b < b1; ++b)
    if (BOUTE_INB(A.first(b) + e0 + i, A.N)) sum += A.place[A.first(b) + e0 + i];
  runs[tid] = sum;
  __syncthreads();
  if (tid < part) {
    int at = 0;
    for (int q = 0; q < per; ++q) {
      const int n = runs[q * part + tid];
      runs[q * part + tid] = at;
      at += n;
    }
    total[tid] = at;
  }
  cluster_sync();
  for (int e = tid; e < E1; e += kScanThreads) first[e] = load_peer(peer(&total[e % part], e / part));
  __syncthreads();
  block_scan<kScanThreads>(first, E1, warp_sums);
  if (rank == 0)
    for (int e = tid; e < E1; e += kScanThreads) A.offsets[e] = first[e];
  int at = b1 > b0 ? first[e0 + i] + runs[tid] : 0;
#pragma unroll 4
  for (int b = b0; b < b1; ++b) {
    if (!BOUTE_INB(A.first(b) + e0 + i, A.N)) continue;
    const int n = A.place[A.first(b) + e0 + i];
    A.place[A.first(b) + e0 + i] = at;
    at += n;
  }
  cluster_sync();
}

__global__ void __launch_bounds__(kSortThreads) expert_place_kernel(Order A) {
  extern __shared__ int sort_smem[];
  pdl_wait();
  pdl_trigger();
  const int E1 = A.E + 1, tid = threadIdx.x, b = blockIdx.x;
  int *hist = sort_smem;
  int key[kSteps], rank[kSteps];
  count_choices(A, b, hist, key, rank);
  for (int e = tid; e < E1; e += kSortThreads) {
    int at = BOUTE_INB(A.first(b) + e, A.N) ? A.place[A.first(b) + e] : 0;
    for (int w = 0; w < kSortWarps; ++w) {
      const int n = hist[w * E1 + e];
      hist[w * E1 + e] = at;
      at += n;
    }
  }
  __syncthreads();
  place_choices(A, b, hist, key, rank);
}

// ---- rows ----------------------------------------------------------------------------
// Rows are moved in vectors of W bytes, the widest that all the rows' addresses allow, and what
// is left of a row by single elements. A team of lanes has kUnroll vectors a lane of a row.
template <int W>
struct Vec;
template <>
struct Vec<16> { using type = uint4; };
template <>
struct Vec<8> { using type = uint2; };
template <>
struct Vec<4> { using type = uint32_t; };
template <>
struct Vec<2> { using type = uint16_t; };

struct Rows {
  long long T, R;  // queries; experts' rows
  int k, D;
  long long ldt, ldr;  // pitches of the queries' and the experts' rows, in elements
  const int *place;
  // the row of a choice, or -1
  __device__ __forceinline__ long long row(long long c) const {
    const int p = BOUTE_INB(c, T * k) ? place[c] : -1;
    return (unsigned long long)(long long)p < (unsigned long long)R ? p : -1;
  }
};

// A unit of work is a run of a row's vectors: `unit` in [0, T x parts).
template <int W, int TEAM, int U>
struct Run {
  long long t;
  int v0, vectors;  // the lane's first vector; vectors of a row
  bool last;        // the row's last run, with what no vector holds
  __device__ __forceinline__ Run(long long unit, int parts, int bytes) {
    t = unit / parts;
    const int part = (int)(unit - t * parts);
    vectors = bytes / W;
    v0 = part * (TEAM * U) + threadIdx.x % TEAM;
    last = part == parts - 1;
  }
};
template <int W, int TEAM, int U>
inline int parts_of(int bytes) {
  return std::max(1, (bytes / W + TEAM * U - 1) / (TEAM * U));
}

template <int W, int TEAM, int U>
__global__ void __launch_bounds__(kThreads)
    expert_dispatch_kernel(Rows A, int parts, int size, const char *x, char *rows) {
  using V = typename Vec<W>::type;
  pdl_wait();
  pdl_trigger();
  const long long unit = ((long long)blockIdx.x * kThreads + threadIdx.x) / TEAM;
  if (unit >= A.T * parts) return;
  const int bytes = A.D * size;
  const Run<W, TEAM, U> run(unit, parts, bytes);
  const char *from = x + run.t * A.ldt * size;
  V v[U];
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (run.v0 + u * TEAM < run.vectors) v[u] = ((const V *)from)[run.v0 + u * TEAM];
  // (what is left of the row, in halves of 4-byte elements too)
  const int rest = run.vectors * W + 2 * (threadIdx.x % TEAM);
  const bool more = run.last && rest < bytes;
  const uint16_t left = more ? *(const uint16_t *)(from + rest) : (uint16_t)0;
  for (int i = 0; i < A.k; ++i) {
    const long long p = A.row(run.t * A.k + i);
    if (p < 0) continue;
    char *to = rows + p * A.ldr * size;
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (run.v0 + u * TEAM < run.vectors) ((V *)to)[run.v0 + u * TEAM] = v[u];
    if (more) *(uint16_t *)(to + rest) = left;
  }
}

// Elements of a vector as floats, and back with one rounding.
template <class T, int W>
__device__ __forceinline__ void add_vector(float *acc, typename Vec<W>::type v, float w) {
  T e[W / sizeof(T)];
  memcpy(e, &v, W);
#pragma unroll
  for (int i = 0; i < (int)(W / sizeof(T)); ++i) acc[i] = fmaf(w, to_float(e[i]), acc[i]);
}
template <class T, int W>
__device__ __forceinline__ typename Vec<W>::type to_vector(const float *acc) {
  T e[W / sizeof(T)];
#pragma unroll
  for (int i = 0; i < (int)(W / sizeof(T)); ++i) e[i] = from_float<T>(acc[i]);
  typename Vec<W>::type v;
  memcpy(&v, e, W);
  return v;
}

// out[t] = the sum of weight x row over the query's choices, in their order; weight NULL: of 1.
template <class T, int W, int TEAM, int U>
__global__ void __launch_bounds__(kThreads)
    expert_combine_kernel(Rows A, int parts, const T *rows, const float *weight, T *out) {
  using V = typename Vec<W>::type;
  constexpr int E = W / sizeof(T), kAtOnce = 4;  // choices on their way to a lane
  pdl_wait();
  pdl_trigger();
  const long long unit = ((long long)blockIdx.x * kThreads + threadIdx.x) / TEAM;
  if (unit >= A.T * parts) return;
  const Run<W, TEAM, U> run(unit, parts, A.D * (int)sizeof(T));
  const int rest = run.vectors * E + threadIdx.x % TEAM;
  const bool more = run.last && rest < A.D;
  float acc[U][E], left = 0.f;
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int e = 0; e < E; ++e) acc[u][e] = 0.f;
  for (int i0 = 0; i0 < A.k; i0 += kAtOnce) {
    V v[kAtOnce][U];
    T one[kAtOnce];
    long long p[kAtOnce];
    float w[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const long long c = run.t * A.k + i0 + i;
      p[i] = i0 + i < A.k ? A.row(c) : -1;
      w[i] = p[i] >= 0 && weight ? weight[c] : 1.f;
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (p[i] < 0) continue;
      const T *from = rows + p[i] * A.ldr;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (run.v0 + u * TEAM < run.vectors) v[i][u] = ((const V *)from)[run.v0 + u * TEAM];
      if (more) one[i] = from[rest];
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      if (p[i] < 0) continue;
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (run.v0 + u * TEAM < run.vectors) add_vector<T, W>(acc[u], v[i][u], w[i]);
      if (more) left = fmaf(w[i], to_float(one[i]), left);
    }
  }
  T *to = out + run.t * A.ldt;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (run.v0 + u * TEAM < run.vectors)
      ((V *)to)[run.v0 + u * TEAM] = to_vector<T, W>(acc[u]);
  if (more) to[rest] = from_float<T>(left);
}

// A team per choice: g_rows[place] = weight g_out[t], g_weight = <g_out[t], rows[place]>.
template <class T, int W, int TEAM, int U>
__global__ void __launch_bounds__(kThreads)
    expert_combine_grad_kernel(Rows A, const T *g_out, const T *rows, const float *weight,
                               T *g_rows, long long ldg, float *g_weight) {
  using V = typename Vec<W>::type;
  constexpr int E = W / sizeof(T);
  __shared__ float red[kWarps];
  pdl_wait();
  pdl_trigger();
  const long long c = ((long long)blockIdx.x * kThreads + threadIdx.x) / TEAM, N = A.T * A.k;
  const long long p = c < N ? A.row(c) : -1;
  const int lane = threadIdx.x % TEAM, vectors = A.D / E;
  float dot = 0.f;
  if (p >= 0) {
    const T *go = g_out + c / A.k * A.ldt, *from = rows + p * A.ldr;
    T *to = g_rows + p * ldg;
    const float w = weight[c];
    for (int v0 = lane; v0 < vectors; v0 += TEAM * U) {
      V a[U], b[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v0 + u * TEAM < vectors) {
          a[u] = ((const V *)go)[v0 + u * TEAM];
          b[u] = ((const V *)from)[v0 + u * TEAM];
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (v0 + u * TEAM < vectors) {
          T x[E], y[E];
          memcpy(x, &a[u], W);
          memcpy(y, &b[u], W);
          float g[E];
#pragma unroll
          for (int e = 0; e < E; ++e) {
            dot = fmaf(to_float(x[e]), to_float(y[e]), dot);
            g[e] = w * to_float(x[e]);
          }
          ((V *)to)[v0 + u * TEAM] = to_vector<T, W>(g);
        }
    }
    const int rest = vectors * E + lane;
    if (rest < A.D) {
      const float x = to_float(go[rest]);
      dot = fmaf(x, to_float(from[rest]), dot);
      to[rest] = from_float<T>(w * x);
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < TEAM) dot += __shfl_xor_sync(kAll, dot, o);
  if constexpr (TEAM > 32) {
    if ((threadIdx.x & 31) == 0) red[threadIdx.x / 32] = dot;
    __syncthreads();
    dot = 0.f;
    for (int q = 0; q < TEAM / 32; ++q) dot += red[q];
  }
  if (lane == 0 && c < N && BOUTE_INB(c, N)) g_weight[c] = dot;
}

}  // namespace

BOUTE_BOUNDS_READER(experts)

}  // namespace boute

using namespace boute;

extern "C" int boute_expert_sort(const int *idx, long long T, int k, int E, int *offsets,
                                 int *source, int *place, void *stream) {
  BOUTE_TRACE();
  if (T < 0 || k < 1 || E < 1 || !array_ok(offsets, 4) ||
      (T > 0 && (!array_ok(idx, 4) || !array_ok(source, 4) || !array_ok(place, 4))))
    return BOUTE_ERR_INVALID_ARG;
  if (T > 0x7fffffff || k > BOUTE_MAX_CHOICES || T * k > 0x7fffffff || E > BOUTE_MAX_EXPERTS)
    return BOUTE_ERR_UNSUPPORTED;
  if (int r = device_ok()) return r;
  const long long N = T * k;
  const cudaStream_t s = (cudaStream_t)stream;
  Order A{idx, N, E, (int)std::max(1ll, (N + kChunk - 1) / kChunk), offsets, source, place};
  const size_t hist = (size_t)kSortWarps * (E + 1) * sizeof(int);
  auto allow = [](auto *kernel, size_t bytes) {
    return bytes <= 48 * 1024 ||
           cudaFuncSetAttribute((const void *)kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                (int)bytes) == cudaSuccess;
  };
  if (A.blocks <= kMaxCluster) {
    const size_t smem = hist + 2 * (E + 1) * sizeof(int);
    if (!allow(expert_sort_kernel, smem)) return last_launch_status();
    return launch_cluster(expert_sort_kernel, A.blocks, kSortThreads, A.blocks, smem, s, A);
  }
  if (!allow(expert_place_kernel, hist)) return last_launch_status();
  if (int r = launch_cluster(expert_count_kernel, A.blocks, kSortThreads, 1, 0, s, A)) return r;
  if (int r = launch_cluster(expert_scan_kernel, kMaxCluster, kScanThreads, kMaxCluster, 0, s, A))
    return r;
  return launch_cluster(expert_place_kernel, A.blocks, kSortThreads, 1, hist, s, A);
}

namespace {

int rows_ok(int dtype, const void *x, long long T, int D, long long ldx, const void *rows,
            long long R, long long ldr, const int *place, int k) {
  const size_t size = dtype_bytes(dtype);
  if (!dtype_known(dtype) || T < 0 || R < 0 || D < 1 || k < 1 || ldx < D || ldr < D ||
      (T > 0 && (!array_ok(x, size) || !array_ok(place, 4))) || (R > 0 && !array_ok(rows, size)))
    return BOUTE_ERR_INVALID_ARG;
  return T > 0x7fffffff || R > 0x7fffffff || k > BOUTE_MAX_CHOICES || T * k > 0x7fffffff ||
                 D > BOUTE_MAX_ROW
             ? BOUTE_ERR_UNSUPPORTED
             : device_ok();
}

// go(W): the widest vectors that all these rows allow (bits: of their addresses and pitches, in
// bytes).
template <class Go>
int with_width(uint64_t bits, int size, Go go) {
  if (bits % 16 == 0) return go(std::integral_constant<int, 16>{});
  if (bits % 8 == 0) return go(std::integral_constant<int, 8>{});
  if (bits % 4 == 0 || size == 4) return go(std::integral_constant<int, 4>{});
  return go(std::integral_constant<int, 2>{});
}

// The sum over the choices of rows, weighted or not.
int combine(const void *rows, int dtype, long long R, int D, long long ldr, const int *place,
            const float *weight, long long T, int k, void *out, long long ldo, cudaStream_t s) {
  const int size = (int)dtype_bytes(dtype);
  const Rows A{T, R, k, D, ldo, ldr, place};
  const uint64_t bits = (uintptr_t)rows | (uintptr_t)out | (uint64_t)(ldr * size) |
                        (uint64_t)(ldo * size);
  return with_dtype(dtype, [&](auto t) {
    using E = decltype(t);
    return with_width(bits, size, [&](auto w) {
      constexpr int W = decltype(w)::value;
      if constexpr (W < (int)sizeof(E)) {
        return (int)BOUTE_ERR_INVALID_ARG;
      } else {
        auto go = [&](auto team, auto u) {
          constexpr int TEAM = decltype(team)::value, U = decltype(u)::value;
          const int parts = parts_of<W, TEAM, U>(D * size);
          return launch_cluster(expert_combine_kernel<E, W, TEAM, U>,
                                (T * parts + kThreads / TEAM - 1) / (kThreads / TEAM), kThreads, 1,
                                0, s, A, parts, (const E *)rows, weight, (E *)out);
        };
        if (D * size / W <= 8) return go(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
        return go(std::integral_constant<int, 32>{}, std::integral_constant<int, 2>{});
      }
    });
  });
}

}  // namespace

extern "C" int boute_expert_dispatch(const void *x, int dtype, long long T, int D, long long ldx,
                                     const int *place, int k, void *rows, long long R,
                                     long long ldr, void *stream) {
  BOUTE_TRACE();
  if (int r = rows_ok(dtype, x, T, D, ldx, rows, R, ldr, place, k)) return r;
  if (T == 0 || R == 0) return BOUTE_OK;
  const int size = (int)dtype_bytes(dtype);
  const Rows A{T, R, k, D, ldx, ldr, place};
  const uint64_t bits = (uintptr_t)x | (uintptr_t)rows | (uint64_t)(ldx * size) |
                        (uint64_t)(ldr * size);
  return with_width(bits, size, [&](auto w) {
    constexpr int W = decltype(w)::value;
    auto go = [&](auto team, auto u) {
      constexpr int TEAM = decltype(team)::value, U = decltype(u)::value;
      const int parts = parts_of<W, TEAM, U>(D * size);
      return launch_cluster(expert_dispatch_kernel<W, TEAM, U>,
                            (T * parts + kThreads / TEAM - 1) / (kThreads / TEAM), kThreads, 1, 0,
                            (cudaStream_t)stream, A, parts, size, (const char *)x, (char *)rows);
    };
    if (D * size / W <= 8) return go(std::integral_constant<int, 8>{}, std::integral_constant<int, 1>{});
    return go(std::integral_constant<int, 32>{}, std::integral_constant<int, 4>{});
  });
}

extern "C" int boute_expert_dispatch_grad(const void *g_rows, int dtype, long long R, int D,
                                          long long ldr, const int *place, long long T, int k,
                                          void *dx, long long ldx, void *stream) {
  BOUTE_TRACE();
  if (int r = rows_ok(dtype, dx, T, D, ldx, g_rows, R, ldr, place, k)) return r;
  if (T == 0) return BOUTE_OK;
  return combine(g_rows, dtype, R, D, ldr, place, nullptr, T, k, dx, ldx, (cudaStream_t)stream);
}

extern "C" int boute_expert_combine(const void *rows, int dtype, long long R, int D, long long ldr,
                                    const int *place, const float *weight, long long T, int k,
                                    void *out, long long ldo, void *stream) {
  BOUTE_TRACE();
  if (T > 0 && !array_ok(weight, 4)) return BOUTE_ERR_INVALID_ARG;
  if (int r = rows_ok(dtype, out, T, D, ldo, rows, R, ldr, place, k)) return r;
  if (T == 0) return BOUTE_OK;
  return combine(rows, dtype, R, D, ldr, place, weight, T, k, out, ldo, (cudaStream_t)stream);
}

extern "C" int boute_expert_combine_grad(const void *g_out, int dtype, long long T, int D,
                                         long long ldo, const void *rows, long long R,
                                         long long ldr, const int *place, const float *weight,
                                         int k, void *g_rows, long long ldg, float *g_weight,
                                         void *stream) {
  BOUTE_TRACE();
  const int size = (int)dtype_bytes(dtype);
  if ((T > 0 && (!array_ok(weight, 4) || !array_ok(g_weight, 4))) || ldg < D ||
      (R > 0 && !array_ok(g_rows, size)) || (R > 0 && g_rows == rows && ldg != ldr))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = rows_ok(dtype, g_out, T, D, ldo, rows, R, ldr, place, k)) return r;
  if (T == 0) return BOUTE_OK;
  const Rows A{T, R, k, D, ldo, ldr, place};
  const uint64_t bits = (uintptr_t)g_out | (uintptr_t)rows | (uintptr_t)g_rows |
                        (uint64_t)(ldo * size) | (uint64_t)(ldr * size) | (uint64_t)(ldg * size);
  return with_dtype(dtype, [&](auto t) {
    using E = decltype(t);
    return with_width(bits, size, [&](auto w) {
      constexpr int W = decltype(w)::value;
      if constexpr (W < (int)sizeof(E)) {
        return (int)BOUTE_ERR_INVALID_ARG;
      } else {
        auto go = [&](auto team, auto u) {
          constexpr int TEAM = decltype(team)::value, U = decltype(u)::value;
          return launch_cluster(expert_combine_grad_kernel<E, W, TEAM, U>,
                                (T * k + kThreads / TEAM - 1) / (kThreads / TEAM), kThreads, 1, 0,
                                (cudaStream_t)stream, A, (const E *)g_out, (const E *)rows, weight,
                                (E *)g_rows, ldg, g_weight);
        };
        if (D * size / W <= 16) return go(std::integral_constant<int, 8>{}, std::integral_constant<int, 2>{});
        return go(std::integral_constant<int, 32>{}, std::integral_constant<int, 4>{});
      }
    });
  });
}
