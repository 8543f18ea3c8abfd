// Between a routing and its experts: the choices in the order of their experts, the queries'
// rows copied there, the experts' rows summed back with the routing's weights, and the gradients.
//
// Memory bounds all but the smallest calls: 65536 queries of 2048 bf16, k = 8, are sorted and sent
// to 256 experts in 370 us (0.97 of the copy rate) and their rows brought back in 345 (1.04); the
// gradients of 32768 x 4096 take 995 (1.04). Rows that start anywhere go at 0.8 (sent), 0.65 (back)
// and 0.6 to 0.9 (gradients) of it, short ones of those at 0.35. The order alone takes three
// launches' latencies beyond 32768 choices (131072 of 64 experts: 8.6 us, 1048576 of 256: 20, of
// which the scan of the blocks' counts is 6 and the places 10), a few queries the host's two calls
// (32 of 64 features: 11.8 us, 3.5 on the device).
#include <algorithm>
#include <type_traits>

#include "answers.cuh"

namespace boute {

namespace {

constexpr int kThreads = 256;

// ---- the order -----------------------------------------------------------------------
// A stable counting sort by expert; a choice of no expert counts as one of expert E, whose places
// follow all others. A block has STEPS choices a thread: a warp's neighbours of equal expert are
// found by ballots and counted behind the warp's earlier ones, so a choice's rank among its
// block's is known after one pass. Up to a cluster's blocks the counts are joined through shared
// memory, in one launch. More choices take three: the blocks' counts, their sums before each block,
// and the places; a block's counts lie in its own part of `place` until it writes that.
constexpr int kSortThreads = 512, kSortWarps = kSortThreads / 32;
constexpr int kMaxCluster = 8, kScanThreads = 1024, kRuns = 64;

struct Order {
  const int *idx;
  long long N;
  int E, blocks, each, more;  // N = blocks each + more
  int *offsets, *source, *place;

  // block b's choices, from here to first(b + 1) (of more than a cluster's blocks, each has E + 1
  // at least)
  __device__ __forceinline__ long long first(int b) const {
    return (long long)b * each + min(b, more);
  }
  // an expert, or E for none
  __device__ __forceinline__ int expert(long long c) const {
    const int e = BOUTE_INB(c, N) ? idx[c] : -1;
    return (unsigned)e < (unsigned)E ? e : E;
  }
};

// The lanes whose key (below 2^bits, or -1) is this lane's: a ballot for each bit. (One match
// instruction takes a turn for each different key: 19 us for the places of 1048576 choices of 256.)
__device__ __forceinline__ unsigned same_key(int key, int bits) {
  unsigned same = kAll;
  for (int i = 0; i <= bits; ++i) {
    const bool on = key >> i & 1;
    const unsigned of = __ballot_sync(kAll, on);
    same &= on ? of : ~of;
  }
  return same;
}

// hist: kSortWarps x (E + 1) counts of the warps' choices; key, rank: of each of the lane's.
template <int STEPS>
__device__ __forceinline__ void count_choices(const Order &A, int b, int *hist, int (&key)[STEPS],
                                              int (&rank)[STEPS]) {
  const int E1 = A.E + 1, tid = threadIdx.x, lane = tid & 31;
  const long long from = A.first(b) + (tid / 32) * (32 * STEPS), end = A.first(b + 1);
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    const long long c = from + j * 32 + lane;
    key[j] = c < end ? A.expert(c) : -1;
  }
  for (int i = tid; i < kSortWarps * E1; i += kSortThreads) hist[i] = 0;
  __syncthreads();
  int *mine = hist + (tid / 32) * E1;
  unsigned peers[STEPS];
  const int bits = 32 - __clz(A.E);
#pragma unroll
  for (int j = 0; j < STEPS; ++j) peers[j] = same_key(key[j], bits);
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    const int before = __popc(peers[j] & ((1u << lane) - 1u));
    int had = 0;
    if (key[j] >= 0 && BOUTE_INB(key[j], E1)) had = mine[key[j]];
    __syncwarp();
    if (key[j] >= 0 && before == 0) mine[key[j]] = had + __popc(peers[j]);
    __syncwarp();
    rank[j] = had + before;
  }
  __syncthreads();
}

// The warps' counts of an expert become the places of each warp's first, from `at` on.
__device__ __forceinline__ void warp_places(int *hist, int E1, int e, int at) {
  int n[kSortWarps];
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) n[w] = hist[w * E1 + e];
#pragma unroll
  for (int w = 0; w < kSortWarps; ++w) {
    hist[w * E1 + e] = at;
    at += n[w];
  }
}

// Each lane's choices to their places: hist holds the first place of each warp's choices of an
// expert.
template <int STEPS>
__device__ __forceinline__ void place_choices(const Order &A, int b, const int *hist,
                                              const int (&key)[STEPS], const int (&rank)[STEPS]) {
  const int E1 = A.E + 1, tid = threadIdx.x, lane = tid & 31;
  const long long from = A.first(b) + (tid / 32) * (32 * STEPS);
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    if (key[j] < 0) continue;
    const int c = (int)(from + j * 32 + lane), at = hist[(tid / 32) * E1 + key[j]] + rank[j];
    if (!BOUTE_INB(c, A.N) || !BOUTE_INB(at, A.N)) continue;
    A.place[c] = key[j] < A.E ? at : -1;
    A.source[at] = key[j] < A.E ? c : -1;
  }
}

// The sums before each of a warp's values, and their total in every lane.
__device__ __forceinline__ int warp_before(int v, int &total) {
  const int lane = threadIdx.x & 31;
  int up = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int x = __shfl_up_sync(kAll, up, o);
    if (lane >= o) up += x;
  }
  total = __shfl_sync(kAll, up, 31);
  return up - v;
}
// v[0 .. n) becomes the sums before each, in place; the block's threads all come.
template <int THREADS>
__device__ __forceinline__ void block_scan(int *v, int n, int *warp_sums) {
  const int tid = threadIdx.x, lane = tid & 31, per = (n + THREADS - 1) / THREADS;
  const int a = min(tid * per, n), b = min(a + per, n);
  int sum = 0, total;
  for (int i = a; i < b; ++i) sum += v[i];
  int before = warp_before(sum, total);
  if (lane == 31) warp_sums[tid / 32] = total;
  __syncthreads();
  const int other = lane < THREADS / 32 ? warp_sums[lane] : 0;
  before += __shfl_sync(kAll, warp_before(other, total), tid / 32);
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

// One cluster. Shared memory: kSortWarps x (E + 1) counts, the block's counts, the experts' first
// places.
template <int STEPS>
__global__ void __launch_bounds__(kSortThreads) expert_sort_kernel(Order A) {
  extern __shared__ int sort_smem[];
  __shared__ int warp_sums[kSortWarps];
  pdl_wait();
  pdl_trigger();
  const int E1 = A.E + 1, tid = threadIdx.x, b = blockIdx.x;
  int *hist = sort_smem, *count = hist + kSortWarps * E1, *first = count + E1;
  int key[STEPS], rank[STEPS];
  count_choices(A, b, hist, key, rank);
  for (int e = tid; e < E1; e += kSortThreads) {
    int n = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) n += hist[w * E1 + e];
    first[e] = count[e] = n;
  }
  constexpr int kMine = (BOUTE_MAX_EXPERTS + kSortThreads) / kSortThreads;  // a thread's experts
  int before_e[kMine];  // of them, in lower blocks
#pragma unroll
  for (int i = 0; i < kMine; ++i) before_e[i] = 0;
  if (A.blocks > 1) {
    cluster_sync();
#pragma unroll
    for (int i = 0; i < kMine; ++i) {
      const int e = tid + i * kSortThreads;
      if (e >= E1) break;
      int n[kMaxCluster], all = 0;
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r)
        n[r] = r < A.blocks ? load_peer(peer(&count[e], r)) : 0;
#pragma unroll
      for (int r = 0; r < kMaxCluster; ++r) {
        if (r < b) before_e[i] += n[r];
        all += n[r];
      }
      first[e] = all;
    }
  }
  __syncthreads();
  block_scan<kSortThreads>(first, E1, warp_sums);
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int e = tid + i * kSortThreads;
    if (e >= E1) break;
    if (b == 0) A.offsets[e] = first[e];
    warp_places(hist, E1, e, first[e] + before_e[i]);
  }
  __syncthreads();
  place_choices(A, b, hist, key, rank);
  if (A.blocks > 1) cluster_sync();  // (the others may read this block's counts until here)
}

// The blocks' counts, each in its own part of `place`.
template <int STEPS>
__global__ void __launch_bounds__(kSortThreads) expert_count_kernel(Order A) {
  __shared__ int hist[BOUTE_MAX_EXPERTS + 1];
  pdl_wait();
  pdl_trigger();
  const int E1 = A.E + 1, tid = threadIdx.x;
  const long long from = A.first(blockIdx.x), end = A.first(blockIdx.x + 1);
  int key[STEPS];
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    const long long c = from + j * kSortThreads + tid;
    key[j] = c < end ? A.expert(c) : -1;
  }
  for (int e = tid; e < E1; e += kSortThreads) hist[e] = 0;
  __syncthreads();
#pragma unroll
  for (int j = 0; j < STEPS; ++j)
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
  constexpr int kKept = 8;  // counts of a run that stay in registers
  const int E1 = A.E + 1, tid = threadIdx.x, rank = blockIdx.x;
  const int part = (E1 + kMaxCluster - 1) / kMaxCluster;  // experts of a block
  const int e0 = rank * part, mine = max(0, min(part, E1 - e0));
  const int per = min(kScanThreads / part, kRuns);  // an expert's runs
  const int i = tid % part, r = tid / part;
  const int len = (A.blocks + per - 1) / per;
  const int b0 = min(r * len, A.blocks), b1 = r < per && i < mine ? min(b0 + len, A.blocks) : b0;
  auto count = [&](int b) -> int & { return A.place[A.first(b) + e0 + i]; };
  int kept[kKept], sum = 0;
#pragma unroll
  for (int j = 0; j < kKept; ++j) {
    const int b = b0 + j;
    kept[j] = b < b1 && BOUTE_INB(A.first(b) + e0 + i, A.N) ? count(b) : 0;
    sum += kept[j];
  }
#pragma unroll 4
  for (int b = b0 + kKept; b < b1; ++b)
    if (BOUTE_INB(A.first(b) + e0 + i, A.N)) sum += count(b);
  runs[tid] = sum;
  __syncthreads();
  for (int q = tid / 32; q < part; q += kScanThreads / 32) {  // a warp per expert
    const int l = 2 * (tid & 31);
    const int x = l < per ? runs[l * part + q] : 0, y = l + 1 < per ? runs[(l + 1) * part + q] : 0;
    int all;
    const int before = warp_before(x + y, all);
    if (l < per) runs[l * part + q] = before;
    if (l + 1 < per) runs[(l + 1) * part + q] = before + x;
    if (l == 0) total[q] = all;
  }
  cluster_sync();
  for (int e = tid; e < E1; e += kScanThreads)
    first[e] = load_peer(peer(&total[e % part], e / part));
  __syncthreads();
  block_scan<kScanThreads>(first, E1, warp_sums);
  if (rank == 0)
    for (int e = tid; e < E1; e += kScanThreads) A.offsets[e] = first[e];
  int at = b1 > b0 ? first[e0 + i] + runs[tid] : 0;
#pragma unroll
  for (int j = 0; j < kKept; ++j) {
    const int b = b0 + j;
    if (b < b1 && BOUTE_INB(A.first(b) + e0 + i, A.N)) count(b) = at;
    at += kept[j];
  }
#pragma unroll 4
  for (int b = b0 + kKept; b < b1; ++b) {
    if (!BOUTE_INB(A.first(b) + e0 + i, A.N)) continue;
    const int n = count(b);
    count(b) = at;
    at += n;
  }
  cluster_sync();
}

// The choices are put in order within the block first: neighbours then write neighbouring sources
// (1048576 choices of 256: 16.8 us with each lane's own store to its place).
constexpr size_t sort_smem_bytes(int E) { return (size_t)(kSortWarps + 2) * (E + 1) * sizeof(int); }
template <int STEPS>
constexpr size_t place_smem_bytes(int E) {
  return sort_smem_bytes(E) + 2 * kSortThreads * STEPS * sizeof(int);
}
template <int STEPS>
__global__ void __launch_bounds__(kSortThreads) expert_place_kernel(Order A) {
  extern __shared__ int sort_smem[];
  __shared__ int warp_sums[kSortWarps];
  pdl_wait();
  pdl_trigger();
  const int E1 = A.E + 1, tid = threadIdx.x, lane = tid & 31, b = blockIdx.x;
  int *hist = sort_smem, *first = hist + kSortWarps * E1, *move = first + E1;
  int *choice = move + E1, *to = choice + kSortThreads * STEPS;
  const long long from = A.first(b);
  const int n = (int)(A.first(b + 1) - from);
  int key[STEPS], rank[STEPS];
  count_choices(A, b, hist, key, rank);
  for (int e = tid; e < E1; e += kSortThreads) {
    int all = 0;
#pragma unroll
    for (int w = 0; w < kSortWarps; ++w) all += hist[w * E1 + e];
    first[e] = all;
    move[e] = BOUTE_INB(from + e, A.N) ? A.place[from + e] : 0;
  }
  __syncthreads();
  block_scan<kSortThreads>(first, E1, warp_sums);
  for (int e = tid; e < E1; e += kSortThreads) {
    warp_places(hist, E1, e, first[e]);
    move[e] -= first[e];
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < STEPS; ++j) {
    if (key[j] < 0) continue;
    const int c = (int)from + (tid / 32) * (32 * STEPS) + j * 32 + lane;
    const int here = hist[(tid / 32) * E1 + key[j]] + rank[j], at = here + move[key[j]];
    if (!BOUTE_INB(c, A.N) || !BOUTE_INB(here, n)) continue;
    A.place[c] = key[j] < A.E ? at : -1;
    choice[here] = key[j] < A.E ? c : -1;
    to[here] = at;
  }
  __syncthreads();
  for (int i = tid; i < n; i += kSortThreads)
    if (BOUTE_INB(to[i], A.N)) A.source[to[i]] = choice[i];
}

// ---- rows ----------------------------------------------------------------------------
// A row is written in 16-byte words (chunks), its ends by elements. Where all rows start and end on
// 16-byte boundaries (ALIGNED) a chunk is one load; else its bytes lie across two words of the row
// that is read, which are loaded and shifted (a lane's second word is its neighbour's first, from
// L1).
struct Rows {
  long long T, R;  // queries; experts' rows
  int k, D;
  long long ldt, ldr;  // pitches of the queries' and the experts' rows, in elements
  const int *place;
  // the row of a choice, or -1
  __device__ __forceinline__ long long row(unsigned c) const {
    const int p = BOUTE_INB(c, T * k) ? place[c] : -1;
    return (unsigned long long)(long long)p < (unsigned long long)R ? p : -1;
  }
};

// How a row that is written falls into 16-byte words: the bytes before the first boundary, the
// whole words (the chunks), the bytes behind them. The bytes at the ends are the row's edges, moved
// by elements, of which there are 14 at most.
template <bool ALIGNED, int SIZE>
struct Split {
  int head, full, edges;  // (edges: elements)
  __device__ __forceinline__ Split(const char *row, int bytes) {
    head = ALIGNED ? 0 : min((int)(0u - (unsigned)(uintptr_t)row) & 15, bytes);
    full = (bytes - head) / 16;
    edges = (bytes - 16 * full) / SIZE;
  }
  // the byte of edge element i
  __device__ __forceinline__ int edge(int i) const {
    return i * SIZE + (i * SIZE < head ? 0 : 16 * full);
  }
};
template <int SIZE>
using Element = typename std::conditional<SIZE == 4, uint32_t, uint16_t>::type;

// A lane's U chunks j0, j0 + TEAM, ... of the `full` from src on: begin() issues the loads of the
// words that hold them, take() gives a chunk.
template <bool ALIGNED, int TEAM, int U>
struct Chunks {
  uint4 a[U], b[ALIGNED ? 1 : U];
  int sh;
  __device__ __forceinline__ void begin(const char *src, int j0, int full) {
    sh = ALIGNED ? 0 : (int)((uintptr_t)src & 15);
    const uint4 *word = (const uint4 *)(src - sh);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int j = j0 + u * TEAM;
      if (j >= full) continue;
      a[u] = word[j];
      if (!ALIGNED && sh) b[ALIGNED ? 0 : u] = word[j + 1];
    }
  }
  __device__ __forceinline__ uint4 take(int u) const {
    if (ALIGNED) return a[u];
    return shifted(a[u], b[ALIGNED ? 0 : u], sh);
  }
};

// A unit of work is a run of a row's chunks, of T x parts; the first has the row's edges, too.
template <int TEAM, int U>
inline int parts_of(int bytes) {
  return std::max(1, (bytes / 16 + TEAM * U - 1) / (TEAM * U));
}
// (T x parts is below 2^31: where there are several parts, one is 16 TEAM U bytes of a row)
template <int TEAM>
__device__ __forceinline__ unsigned unit_index() {
  return (unsigned)(((unsigned long long)blockIdx.x * kThreads + threadIdx.x) / TEAM);
}
// Edge elements of a lane of a team.
template <bool ALIGNED, int TEAM>
constexpr int kEdges = ALIGNED ? 0 : (14 + TEAM - 1) / TEAM;

template <bool ALIGNED, int SIZE, int TEAM, int U>
__global__ void __launch_bounds__(kThreads)
    expert_dispatch_kernel(Rows A, unsigned units, unsigned parts, const char *x, char *rows) {
  using El = Element<SIZE>;
  pdl_wait();
  pdl_trigger();
  const unsigned unit = unit_index<TEAM>();
  if (unit >= units) return;
  const unsigned t = unit / parts, c = t * A.k, part = unit - t * parts;
  const int lane = threadIdx.x % TEAM, j0 = (int)part * (TEAM * U) + lane, bytes = A.D * SIZE;
  const char *from = x + t * A.ldt * SIZE;
  Chunks<ALIGNED, TEAM, U> v;
  if constexpr (ALIGNED) v.begin(from, j0, bytes / 16);
  for (int i = 0; i < A.k; ++i) {
    const long long p = A.row(c + i);
    if (p < 0) continue;
    char *to = rows + p * A.ldr * SIZE;
    const Split<ALIGNED, SIZE> s(to, bytes);
    if constexpr (!ALIGNED) v.begin(from + s.head, j0, s.full);
    if (!ALIGNED && part == 0)
#pragma unroll
      for (int q = 0; q < kEdges<ALIGNED, TEAM>; ++q)
        if (lane + q * TEAM < s.edges) {
          const int at = s.edge(lane + q * TEAM);
          *(El *)(to + at) = *(const El *)(from + at);
        }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (j0 + u * TEAM < s.full) ((uint4 *)(to + s.head))[j0 + u * TEAM] = v.take(u);
  }
}

// A vector's elements as floats, and back with one rounding.
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
template <class T, int W>
__device__ __forceinline__ void vector_floats(typename Vec<W>::type v, float (&x)[W / sizeof(T)]) {
  if constexpr (W == 2) {
    T e;
    memcpy(&e, &v, 2);
    x[0] = to_float(e);
  } else {
    uint32_t w[W / 4];
    memcpy(w, &v, W);
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      if constexpr (sizeof(T) == 4) x[i] = __uint_as_float(w[i]);
      else unpack2(T{}, w[i], x[2 * i], x[2 * i + 1]);
    }
  }
}
template <class T, int W>
__device__ __forceinline__ typename Vec<W>::type floats_vector(const float (&x)[W / sizeof(T)]) {
  typename Vec<W>::type v;
  if constexpr (W == 2) {
    const T e = from_float<T>(x[0]);
    memcpy(&v, &e, 2);
  } else {
    uint32_t w[W / 4];
#pragma unroll
    for (int i = 0; i < W / 4; ++i) {
      if constexpr (sizeof(T) == 4) w[i] = __float_as_uint(x[i]);
      else w[i] = pack2(T{}, x[2 * i], x[2 * i + 1]);
    }
    memcpy(&v, w, W);
  }
  return v;
}
template <class T>
__device__ __forceinline__ void to_floats(uint4 v, float (&x)[16 / sizeof(T)]) {
  vector_floats<T, 16>(v, x);
}
template <class T>
__device__ __forceinline__ uint4 from_floats(const float (&x)[16 / sizeof(T)]) {
  return floats_vector<T, 16>(x);
}

// out[t] = the sum of weight x row over the query's choices, in their order; weight NULL: of 1.
template <class T, bool ALIGNED, int TEAM, int U, int AT_ONCE>
__global__ void __launch_bounds__(kThreads)
    expert_combine_kernel(Rows A, unsigned units, unsigned parts, const T *rows,
                          const float *weight, T *out) {
  constexpr int SIZE = sizeof(T), E = 16 / SIZE, EDGES = kEdges<ALIGNED, TEAM>;
  pdl_wait();
  pdl_trigger();
  const unsigned unit = unit_index<TEAM>();
  if (unit >= units) return;
  const unsigned t = unit / parts, c = t * A.k, part = unit - t * parts;
  const int lane = threadIdx.x % TEAM, j0 = (int)part * (TEAM * U) + lane, bytes = A.D * SIZE;
  char *to = (char *)(out + t * A.ldt);
  const Split<ALIGNED, SIZE> s(to, bytes);
  const int edges = part == 0 ? s.edges : 0;
  float acc[U][E], edge[EDGES + 1];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int i = 0; i < E; ++i) acc[u][i] = 0.f;
#pragma unroll
  for (int q = 0; q < EDGES; ++q) edge[q] = 0.f;
  for (int i0 = 0; i0 < A.k; i0 += AT_ONCE) {
    Chunks<ALIGNED, TEAM, U> v[AT_ONCE];
    T one[AT_ONCE][EDGES + 1];
    const char *from[AT_ONCE];
    float w[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      const long long p = i0 + i < A.k ? A.row(c + i0 + i) : -1;
      from[i] = p >= 0 ? (const char *)(rows + p * A.ldr) : nullptr;
      w[i] = p >= 0 && weight ? weight[c + i0 + i] : 1.f;
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (!from[i]) continue;
      v[i].begin(from[i] + s.head, j0, s.full);
#pragma unroll
      for (int q = 0; q < EDGES; ++q)
        if (lane + q * TEAM < edges) one[i][q] = *(const T *)(from[i] + s.edge(lane + q * TEAM));
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (!from[i]) continue;
#pragma unroll
      for (int u = 0; u < U; ++u) {
        float f[E];
        to_floats<T>(v[i].take(u), f);
#pragma unroll
        for (int q = 0; q < E; ++q) acc[u][q] = fmaf(w[i], f[q], acc[u][q]);
      }
#pragma unroll
      for (int q = 0; q < EDGES; ++q)
        if (lane + q * TEAM < edges) edge[q] = fmaf(w[i], to_float(one[i][q]), edge[q]);
    }
  }
  if (!BOUTE_INB(t, A.T)) return;
#pragma unroll
  for (int u = 0; u < U; ++u)
    if (j0 + u * TEAM < s.full) ((uint4 *)(to + s.head))[j0 + u * TEAM] = from_floats<T>(acc[u]);
#pragma unroll
  for (int q = 0; q < EDGES; ++q)
    if (lane + q * TEAM < edges) *(T *)(to + s.edge(lane + q * TEAM)) = from_float<T>(edge[q]);
}

// x y of a chunk, added to dot; w x.
template <class T>
__device__ __forceinline__ uint4 chunk_grad(uint4 x, uint4 y, float w, float &dot) {
  constexpr int E = 16 / sizeof(T);
  float f[E], r[E];
  to_floats<T>(x, f);
  to_floats<T>(y, r);
#pragma unroll
  for (int q = 0; q < E; ++q) {
    dot = fmaf(f[q], r[q], dot);
    f[q] *= w;
  }
  return from_floats<T>(f);
}
// g_rows[place] = weight g_out[t], g_weight = <g_out[t], rows[place]>: a team for each choice. In
// vectors of W bytes, to whose boundaries all rows are aligned, and the elements behind the last.
template <class T, int W, int TEAM, int U>
__global__ void __launch_bounds__(kThreads)
    expert_combine_grad_kernel(Rows A, const T *g_out, const T *rows, const float *weight,
                               T *g_rows, long long ldg, float *g_weight) {
  using V = typename Vec<W>::type;
  constexpr int E = W / sizeof(T);
  pdl_wait();
  pdl_trigger();
  const unsigned c = unit_index<TEAM>(), N = (unsigned)(A.T * A.k);
  const long long p = c < N ? A.row(c) : -1;
  const int lane = threadIdx.x % TEAM, full = A.D / E;
  float dot = 0.f;
  if (p >= 0) {
    const T *go = g_out + c / A.k * A.ldt, *from = rows + p * A.ldr;
    T *to = g_rows + p * ldg;
    const float w = weight[c];
    const int rest = full * E + lane;
    T x1, y1;
    if (rest < A.D) {
      x1 = go[rest];
      y1 = from[rest];
    }
    for (int j0 = lane; j0 < full; j0 += TEAM * U) {
      V x[U], y[U];
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j0 + u * TEAM < full) {
          x[u] = ((const V *)go)[j0 + u * TEAM];
          y[u] = ((const V *)from)[j0 + u * TEAM];
        }
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (j0 + u * TEAM < full) {
          float f[E], r[E];
          vector_floats<T, W>(x[u], f);
          vector_floats<T, W>(y[u], r);
#pragma unroll
          for (int q = 0; q < E; ++q) {
            dot = fmaf(f[q], r[q], dot);
            f[q] *= w;
          }
          ((V *)to)[j0 + u * TEAM] = floats_vector<T, W>(f);
        }
    }
    if (rest < A.D) {
      dot = fmaf(to_float(x1), to_float(y1), dot);
      to[rest] = from_float<T>(w * to_float(x1));
    }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < TEAM) dot += __shfl_xor_sync(kAll, dot, o);
  if (lane == 0 && c < N && BOUTE_INB(c, N)) g_weight[c] = dot;
}

// The same of short rows at any address, in shifted chunks.
template <class T, int TEAM>
__global__ void __launch_bounds__(kThreads)
    expert_shifted_grad_kernel(Rows A, const T *g_out, const T *rows, const float *weight,
                               T *g_rows, long long ldg, float *g_weight) {
  constexpr int EDGES = kEdges<false, TEAM>;
  pdl_wait();
  pdl_trigger();
  const unsigned c = unit_index<TEAM>(), N = (unsigned)(A.T * A.k);
  const long long p = c < N ? A.row(c) : -1;
  const int lane = threadIdx.x % TEAM, bytes = A.D * (int)sizeof(T);
  float dot = 0.f;
  if (p >= 0) {
    const char *go = (const char *)(g_out + c / A.k * A.ldt);
    const char *from = (const char *)(rows + p * A.ldr);
    char *to = (char *)(g_rows + p * ldg);
    const Split<false, sizeof(T)> s(to, bytes);
    const float w = weight[c];
    T x1[EDGES], y1[EDGES];
#pragma unroll
    for (int q = 0; q < EDGES; ++q)
      if (lane + q * TEAM < s.edges) {
        x1[q] = *(const T *)(go + s.edge(lane + q * TEAM));
        y1[q] = *(const T *)(from + s.edge(lane + q * TEAM));
      }
    for (int j = lane; j < s.full; j += TEAM) {
      Chunks<false, TEAM, 1> x, y;
      x.begin(go + s.head, j, s.full);
      y.begin(from + s.head, j, s.full);
      ((uint4 *)(to + s.head))[j] = chunk_grad<T>(x.take(0), y.take(0), w, dot);
    }
#pragma unroll
    for (int q = 0; q < EDGES; ++q)
      if (lane + q * TEAM < s.edges) {
        dot = fmaf(to_float(x1[q]), to_float(y1[q]), dot);
        *(T *)(to + s.edge(lane + q * TEAM)) = from_float<T>(w * to_float(x1[q]));
      }
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o < TEAM) dot += __shfl_xor_sync(kAll, dot, o);
  if (lane == 0 && c < N && BOUTE_INB(c, N)) g_weight[c] = dot;
}

// The same with a team for each query, which holds its gradient: aligned rows of up to TEAM x U
// chunks. (200000 x 4 rows of 64 bf16: 45 us, 345 by a warp for each choice; 50000 of 512: 71 and
// 111.)
template <class T, int TEAM, int U, int AT_ONCE>
__global__ void __launch_bounds__(kThreads)
    expert_query_grad_kernel(Rows A, const T *g_out, const T *rows, const float *weight,
                             T *g_rows, long long ldg, float *g_weight) {
  constexpr int SIZE = sizeof(T);
  pdl_wait();
  pdl_trigger();
  const unsigned t = unit_index<TEAM>();
  const bool in = t < A.T;
  const unsigned c = in ? t * A.k : 0u;
  const int lane = threadIdx.x % TEAM, bytes = A.D * SIZE, full = bytes / 16;
  const char *go = (const char *)(g_out + t * A.ldt);
  Chunks<true, TEAM, U> x;
  if (in) x.begin(go, lane, full);
  for (int i0 = 0; i0 < A.k; i0 += AT_ONCE) {
    Chunks<true, TEAM, U> y[AT_ONCE];
    long long p[AT_ONCE];
    float w[AT_ONCE], dot[AT_ONCE];
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      p[i] = in && i0 + i < A.k ? A.row(c + i0 + i) : -1;
      w[i] = p[i] >= 0 ? weight[c + i0 + i] : 0.f;
      dot[i] = 0.f;
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i)
      if (p[i] >= 0) y[i].begin((const char *)(rows + p[i] * A.ldr), lane, full);
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
      if (p[i] < 0) continue;
      char *to = (char *)(g_rows + p[i] * ldg);
#pragma unroll
      for (int u = 0; u < U; ++u)
        if (lane + u * TEAM < full)
          ((uint4 *)to)[lane + u * TEAM] = chunk_grad<T>(x.take(u), y[i].take(u), w[i], dot[i]);
    }
#pragma unroll
    for (int i = 0; i < AT_ONCE; ++i) {
#pragma unroll
      for (int o = 16; o > 0; o >>= 1)
        if (o < TEAM) dot[i] += __shfl_xor_sync(kAll, dot[i], o);
      if (lane == 0 && in && i0 + i < A.k && BOUTE_INB(c + i0 + i, A.T * A.k))
        g_weight[c + i0 + i] = dot[i];
    }
  }
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
  const long long N = T * k;
  // (the choices are read again after the outputs are written)
  if (outputs_overlap({array_of(offsets, E + 1, 4), array_of(source, N, 4), array_of(place, N, 4)},
                      {array_of(idx, N, 4)}))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = device_ok()) return r;
  const cudaStream_t s = (cudaStream_t)stream;
  Order A{idx, N, E, 0, 0, 0, offsets, source, place};
  constexpr size_t kUnasked = 47 * 1024;  // of 48 KB that kernels have, beside static arrays
  auto go = [&](auto steps) -> int {
    constexpr int STEPS = decltype(steps)::value;
    A.blocks = (int)std::max(1ll, (N + kSortThreads * STEPS - 1) / (kSortThreads * STEPS));
    A.each = (int)(N / A.blocks);
    A.more = (int)(N % A.blocks);
    if (A.blocks <= kMaxCluster) {
      const size_t smem = sort_smem_bytes(E);
      if (smem > kUnasked && raise_smem(expert_sort_kernel<STEPS>, smem) != cudaSuccess)
        return last_launch_status();
      return launch_cluster(expert_sort_kernel<STEPS>, A.blocks, kSortThreads, A.blocks, smem, s,
                            A);
    }
    const size_t smem = place_smem_bytes<STEPS>(E);
    if (smem > kUnasked && raise_smem(expert_place_kernel<STEPS>, smem) != cudaSuccess)
      return last_launch_status();
    if (int r = launch_cluster(expert_count_kernel<STEPS>, A.blocks, kSortThreads, 1, 0, s, A))
      return r;
    if (int r = launch_cluster(expert_scan_kernel, kMaxCluster, kScanThreads, kMaxCluster, 0, s, A))
      return r;
    return launch_cluster(expert_place_kernel<STEPS>, A.blocks, kSortThreads, 1, smem, s, A);
  };
  // One launch of a cluster as far as it goes (24594 choices: 6.7 us, 8.3 in three); behind it
  // small blocks that fill the SMs, but for many choices, of which the blocks' counts would be most
  // of the work (131072 of 64: 8.6 us with 2 steps, 11.6 with 8; 524288 of 256: 23.3 and 13.6), and
  // no fewer choices a block than counts.
  constexpr long long kOne = (long long)kMaxCluster * kSortThreads;
  const long long at_once = num_sms() * kSortThreads * 2ll;
  if (N <= 2 * kOne) return go(std::integral_constant<int, 2>{});
  if (N <= 4 * kOne) return go(std::integral_constant<int, 4>{});
  if (N <= 8 * kOne) return go(std::integral_constant<int, 8>{});
  if (N > 2 * at_once) return go(std::integral_constant<int, 8>{});
  return E < 900 ? go(std::integral_constant<int, 2>{}) : go(std::integral_constant<int, 4>{});
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
             : BOUTE_OK;
}

// Whether rows of these addresses, pitches and lengths (in bytes) start and end on 16-byte
// boundaries.
bool rows_aligned(uint64_t bits) { return bits % 16 == 0; }

template <int N>
using Int = std::integral_constant<int, N>;
using Yes = std::true_type;
using No = std::false_type;

// The sum over the choices of rows, weighted or not.
int combine(const void *rows, int dtype, long long R, int D, long long ldr, const int *place,
            const float *weight, long long T, int k, void *out, long long ldo, cudaStream_t s) {
  const int size = (int)dtype_bytes(dtype), bytes = D * size;
  const Rows A{T, R, k, D, ldo, ldr, place};
  const bool aligned = rows_aligned((uintptr_t)rows | (uintptr_t)out | (uint64_t)(ldr * size) |
                                    (uint64_t)(ldo * size) | (uint64_t)bytes);
  return with_dtype(dtype, [&](auto t) {
    using E = decltype(t);
    auto go = [&](auto al, auto team, auto u, auto at_once) {
      constexpr int TEAM = decltype(team)::value, U = decltype(u)::value;
      const int parts = parts_of<TEAM, U>(bytes);
      return launch_cluster(
          expert_combine_kernel<E, decltype(al)::value, TEAM, U, decltype(at_once)::value>,
          (T * parts + kThreads / TEAM - 1) / (kThreads / TEAM), kThreads, 1, 0, s, A,
          (unsigned)(T * parts), (unsigned)parts, (const E *)rows, weight, (E *)out);
    };
    // Lanes and chunks by the row, of which there should be enough on their way, and lanes that are
    // not idle (bf16, k = 4, in us): 200000 rows of 64: 27 by 8 lanes, 81 by 32; 50000 of 512: 45
    // by 32 lanes of 2 chunks, 48 by 8 of 1, 61 of 4; 32768 of 1024: 54 by 32 of 4, 57 of 2. Not
    // aligned, 200000 of 64: 42 by 8 lanes of 1 chunk, 58 of 2; 100000 of 256: 65 of 2, 79 of 1,
    // 107 by 32 lanes; 32768 of 1024: 77 by 32 lanes, 81 by 8, 104 by 32 with four choices at once.
    if (aligned) {
      if (bytes <= 512) return go(Yes{}, Int<8>{}, Int<1>{}, Int<4>{});
      return bytes < 2048 ? go(Yes{}, Int<32>{}, Int<2>{}, Int<4>{})
                          : go(Yes{}, Int<32>{}, Int<4>{}, Int<4>{});
    }
    if (bytes <= 160) return go(No{}, Int<8>{}, Int<1>{}, Int<2>{});
    return bytes <= 1024 ? go(No{}, Int<8>{}, Int<2>{}, Int<2>{})
                         : go(No{}, Int<32>{}, Int<2>{}, Int<2>{});
  });
}

}  // namespace

extern "C" int boute_expert_dispatch(const void *x, int dtype, long long T, int D, long long ldx,
                                     const int *place, int k, void *rows, long long R,
                                     long long ldr, void *stream) {
  BOUTE_TRACE();
  if (int r = rows_ok(dtype, x, T, D, ldx, rows, R, ldr, place, k)) return r;
  const int size = (int)dtype_bytes(dtype), bytes = D * size;
  if (outputs_overlap({rows_of(rows, R, D, ldr, size)},
                      {rows_of(x, T, D, ldx, size), array_of(place, T * k, 4)}))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = device_ok()) return r;
  if (T == 0 || R == 0) return BOUTE_OK;
  const Rows A{T, R, k, D, ldx, ldr, place};
  const bool aligned = rows_aligned((uintptr_t)x | (uintptr_t)rows | (uint64_t)(ldx * size) |
                                    (uint64_t)(ldr * size) | (uint64_t)bytes);
  auto go = [&](auto al, auto sz, auto team, auto u) {
    constexpr int TEAM = decltype(team)::value, U = decltype(u)::value;
    const int parts = parts_of<TEAM, U>(bytes);
    return launch_cluster(
        expert_dispatch_kernel<decltype(al)::value, decltype(sz)::value, TEAM, U>,
        (T * parts + kThreads / TEAM - 1) / (kThreads / TEAM), kThreads, 1, 0,
        (cudaStream_t)stream, A, (unsigned)(T * parts), (unsigned)parts, (const char *)x,
        (char *)rows);
  };
  auto with_size = [&](auto sz) {
    // (bf16, k = 4, in us: 400000 rows of 24: 19 by 8 lanes, 58 by 32; 32768 of 1024: 52 and 51;
    // not aligned, of 24: 50 and 179, of 1024: 65 and 58)
    if (aligned)
      return bytes <= 512 ? go(Yes{}, sz, Int<8>{}, Int<1>{}) : go(Yes{}, sz, Int<32>{}, Int<2>{});
    return bytes <= 512 ? go(No{}, sz, Int<8>{}, Int<1>{}) : go(No{}, sz, Int<32>{}, Int<2>{});
  };
  return size == 4 ? with_size(Int<4>{}) : with_size(Int<2>{});
}

extern "C" int boute_expert_dispatch_grad(const void *g_rows, int dtype, long long R, int D,
                                          long long ldr, const int *place, long long T, int k,
                                          void *dx, long long ldx, void *stream) {
  BOUTE_TRACE();
  if (int r = rows_ok(dtype, dx, T, D, ldx, g_rows, R, ldr, place, k)) return r;
  const size_t size = dtype_bytes(dtype);
  if (outputs_overlap({rows_of(dx, T, D, ldx, size)},
                      {rows_of(g_rows, R, D, ldr, size), array_of(place, T * k, 4)}))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = device_ok()) return r;
  if (T == 0) return BOUTE_OK;
  return combine(g_rows, dtype, R, D, ldr, place, nullptr, T, k, dx, ldx, (cudaStream_t)stream);
}

extern "C" int boute_expert_combine(const void *rows, int dtype, long long R, int D, long long ldr,
                                    const int *place, const float *weight, long long T, int k,
                                    void *out, long long ldo, void *stream) {
  BOUTE_TRACE();
  if (T > 0 && !array_ok(weight, 4)) return BOUTE_ERR_INVALID_ARG;
  if (int r = rows_ok(dtype, out, T, D, ldo, rows, R, ldr, place, k)) return r;
  const size_t size = dtype_bytes(dtype);
  if (outputs_overlap({rows_of(out, T, D, ldo, size)},
                      {rows_of(rows, R, D, ldr, size), array_of(place, T * k, 4),
                       array_of(weight, T * k, 4)}))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = device_ok()) return r;
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
      (R > 0 && !array_ok(g_rows, size)))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = rows_ok(dtype, g_out, T, D, ldo, rows, R, ldr, place, k)) return r;
  const Region read = rows_of(rows, R, D, ldr, size), g_read = rows_of(g_out, T, D, ldo, size);
  const Region written = rows_of(g_rows, R, D, ldg, size), g_w = array_of(g_weight, T * k, 4);
  const Region places = array_of(place, T * k, 4), weights = array_of(weight, T * k, 4);
  const bool in_place = g_rows == rows && (ldg == ldr || R <= 1);
  if (outputs_overlap({written, g_w}, {g_read, places, weights}) || overlap(g_w, read) ||
      (!in_place && overlap(written, read)))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = device_ok()) return r;
  if (T == 0) return BOUTE_OK;
  const Rows A{T, R, k, D, ldo, ldr, place};
  const int bytes = D * size;
  const uint64_t bits = (uintptr_t)g_out | (uintptr_t)rows | (uintptr_t)g_rows |
                        (uint64_t)(ldo * size) | (uint64_t)(ldr * size) | (uint64_t)(ldg * size);
  const cudaStream_t s = (cudaStream_t)stream;
  return with_dtype(dtype, [&](auto t) {
    using E = decltype(t);
    auto start = [&](auto *kernel, long long teams, int team) {
      return launch_cluster(kernel, (teams + kThreads / team - 1) / (kThreads / team), kThreads, 1,
                            0, s, A, (const E *)g_out, (const E *)rows, weight, (E *)g_rows, ldg,
                            g_weight);
    };
    if (rows_aligned(bits | (uint64_t)bytes)) {
      if (bytes <= 128) return start(expert_query_grad_kernel<E, 8, 1, 4>, T, 8);
      if (bytes <= 512) return start(expert_query_grad_kernel<E, 32, 1, 4>, T, 32);
      if (bytes <= 1024) return start(expert_query_grad_kernel<E, 32, 2, 4>, T, 32);
    }
    if (bits % 16 == 0) return start(expert_combine_grad_kernel<E, 16, 32, 4>, T * k, 32);
    // (200000 x 4 rows of 64 bf16: 84 us in vectors of 8 bytes, 97 in shifted chunks, 205 in
    // vectors of 4, 160 in elements; long rows go as fast in vectors of 4 and elements as shifted,
    // 32768 x 4 of 1024: 109 and 141 us for 153)
    if (bits % 8 == 0)
      return bytes <= 256 ? start(expert_combine_grad_kernel<E, 8, 8, 4>, T * k, 8)
                          : start(expert_combine_grad_kernel<E, 8, 32, 4>, T * k, 32);
    if (bytes <= 256) return start(expert_shifted_grad_kernel<E, 8>, T * k, 8);
    if constexpr (sizeof(E) == 4) {
      return start(expert_combine_grad_kernel<E, 4, 32, 8>, T * k, 32);
    } else {
      return bits % 4 == 0 ? start(expert_combine_grad_kernel<E, 4, 32, 8>, T * k, 32)
                           : start(expert_combine_grad_kernel<E, 2, 32, 8>, T * k, 32);
    }
  });
}
