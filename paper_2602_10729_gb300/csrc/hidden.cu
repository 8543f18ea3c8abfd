// Log-probabilities of given tokens from a model's last hidden states and its vocabulary's
// weight, without the logits, and the gradient with respect to both.
//
// With x = h . w_j (fp32, of 16-bit products), c = scale log2 e, and per token of the vocabulary's
// pieces m = max x, s = sum 2^((x - m) c), u = sum (x - m) c 2^((x - m) c):
//   lse = scale m + ln s,  logprob = scale (x_t - m) - ln s,  entropy = ln s - ln 2 u / s.
// The gradient takes the logits again, piece by piece of the vocabulary, as coefficients
//   c_tj = scale (g ([j = t] - p_j) - g_H p_j (ln p_j + H)),
// of which dh = c W and dW = c^T h are two more products.
// Where |lse| is large its rounding would be in every p: the statistics are taken once more before
// that, in a launch that ends at once where no position needs it.
//
// All products run on the tensor cores. A pair of blocks takes tiles of 256 rows x up to 256
// columns, one warp bringing operand tiles, one issuing products, and two groups of four warps
// taking the accumulators' tiles in turn, so that a tile's sums or stores go on behind the next
// one's products. The logits' pieces are as small as a tile (256 tokens), the coefficients' as
// large as 256 MB: a piece's reductions and its tail of tiles are long beside what they wait for.
//
// Many positions are bound by the tensor cores (97 % of their cycles in the statistics, 91 and 78
// in the gradient's two launches) and at that by power, which takes the clock to 1.7 GHz: 4096
// positions x 131072 tokens, 4096 elements, bf16: 2.38 to 2.52 ms from machine to machine (1.74 to
// 1.85 PFLOP/s; a library product that writes such logits 2.25 ms); the gradient with 2048 elements
// 4.1 to 4.23 ms (1.56 to 1.61). In the gradient, what operands read by columns cost is not hidden
// (without their copies the launch took 508 us for 627). Few positions are bound by reading the
// weight: one position of 50021 x 2048 takes 42 us (4.9 TB/s; 36 are the kernel's, the rest its
// start, the last tile and the join), 64 of 32768 x 4096 51, and 158 for the gradient, which reads
// the weight twice and writes as much. Between them every 256 tokens ask as many bytes of the L2 as
// it brings at the tensor cores' pace: 515 x 50021 x 1024 47 to 50 us (1.1 PFLOP/s). A weight whose
// rows are no multiples of 128 bytes is read in pieces of two lines (515 x 50021 x 1000 fp16:
// gradient 167 to 178 us, with 1024 elements 157 to 161), one of no multiples of 16 is copied first
// (64 x 32768 x 1001: 42 to 46 us, x 1000 18 to 22). Far positions cost what the statistics do (515
// x 50021 x 1000: 265 us).
#include <float.h>
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "pair_mma.cuh"

namespace boute {

namespace {

constexpr int kThreads = 320, kEpiWarps = 8, kGroup = 128;  // two warps of roles, two groups
constexpr int kMaxStages = 12;
constexpr int kABytes = 128 * kBlockK * 2;  // a block's half of a stage's rows
constexpr int kPitch = 36;  // floats of a row of a warp's 32 x 32 transposition
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kLowest = -200.f;  // 2^kLowest = 0 in fp32

// What a launch makes of its tiles. The logits come with the vocabulary in the tile's rows and the
// positions in its columns (any number of positions fills the columns of a tile), or with the
// positions in its rows (a thread has a position's logits, and no sum crosses threads).
enum Kind { kStatsCols, kStatsRows, kCoefCols, kCoefRows, kGrads };

// At the start of a call's workspace.
constexpr int kBlocks = 256;  // of a launch at most
constexpr int kBounds = BOUTE_MAX_HIDDEN / 256;
struct Header {
  // BOUTE_ERR_TIMEOUT where a wait ran out: in the gradient's launches, which clear it first; in
  // each block of the statistics' launch, which writes its own
  int late, status[kBlocks];
  // bits of the largest bound of a coefficient, of each 256 positions
  unsigned largest[kBounds];
};
// What the coefficients of a position need: p = e^lp, lp = (x - m) scale - ls, p (a + b lp), + g at
// its target j (-1 for none). m is 0 but for far positions.
struct Position {
  float ls, a, b, g;
};
struct Target {
  int j;
  float m;
};

// Whether lse's rounding (2^-24 of it) would show in p. Such positions' coefficients take the
// largest logit and ln s from the logits, which are then summed once more; with the difference
// first, the rounding of the product by the scale is no larger than lp's.
__device__ __forceinline__ bool is_far(float lse) {
  return fabsf(lse) > kLargeLse && isfinite(lse);
}

// The power of two by which the coefficients are scaled while they are 16-bit numbers: the largest
// comes to 2^14 (fp16: what is 2^-28 of that has all its bits, and 2^-39 some). For whole warps.
__device__ __forceinline__ float coef_scale(const Header *head, int bounds, bool inverse) {
  unsigned largest = 0u;
  for (int i = threadIdx.x & 31; i < bounds; i += 32) largest = max(largest, head->largest[i]);
  largest = __reduce_max_sync(kAll, largest);
  const int e = (int)(largest >> 23) - 127;  // (the largest is in [2^e, 2^(e + 1)))
  if (largest == 0u) return 1.f;
  const int k = min(max(13 - e, -126), 126);
  return exp2i(inverse ? -k : k);
}

// The statistics are of logits times k, which is 2 where scale log2 e would be infinite (of a scale
// above 2.3e38: 0 times it would be NaN).
float logits_by(float scale) { return scale * kLog2e <= FLT_MAX ? 1.f : 2.f; }
float exponents_of(float scale) { return scale / logits_by(scale) * kLog2e; }

struct Work {
  int M, N, K;              // rows, columns, reduction
  int tile_m, tile_n, nM, nN, splits;  // (tile_m: rows of a block, 128 but for few positions)
  int a_mn, b_mn, rows_first;  // operands' order; whether neighbouring units differ in their rows
  int tx_bytes;             // that a block's copies bring for a stage
  Header *head;
  int bounds;               // values of head->largest
  // statistics
  float k, c2;              // logits_by, exponents_of the scale
  float *part;              // 3 x parts x Tp: maxima, s, u
  float *picked;            // Tp: x of the targets
  const long long *targets;
  const float *lse;         // (to ask for far positions)
  long long Tp;             // (coefficients: the pitch of coef)
  // coefficients
  const Position *pos;
  const Target *tgt;
  float scale;
  uint16_t *coef;           // a piece's: tokens x positions, or positions x tokens
  int low;                  // columns on, what rounding left of each follows (0: none kept)
  int row0;                 // of the piece in the vocabulary
  // gradients
  float *sums;              // dh: splits x N x M, in fp32
  int add;                  // to what earlier pieces left there
  char *out;                // dW: M x N, pitch ldo
  long long ldo;
  int width;                // bytes that the rows' alignment allows in a store
  int boxes;                // whether `out` has a map
};
// A launch's products: one set of tiles, or dh's and behind them dW's.
struct Job {
  CUtensorMap a, b, out;  // out: where boxes are stored
  Work w;
};
struct Jobs {
  Job job[2];
  int units[2], stages, stage_bytes;
  int far;   // statistics of a pass that has far positions alone, else of none
  int part;  // blocks of the reduction that an accumulator takes (statistics in parts)
  // The pairs take the first set's units in turn; those that got one fewer (`light`, from pair
  // light_from on) take `ahead` of the second set first, then all take the rest in turn.
  int light_from, ahead;
};

struct Unit {
  int job, m, n, k0, k1, split;  // tiles; blocks of the reduction; job < 0: none
};
// The i-th unit of a pair.
template <Kind KIND>
__device__ __forceinline__ Unit unit_of(const Jobs &J, int pair, int pairs, int i) {
  int job = 0, u = pair + i * pairs;
  if (KIND == kGrads && u >= J.units[0]) {
    job = 1;
    const int had = pair < J.units[0] ? (J.units[0] - pair + pairs - 1) / pairs : 0;
    int j = i - had;
    const int lights = pairs - J.light_from, l = pair - J.light_from;
    const int heads = min(J.units[1], lights * J.ahead);
    if (l < 0) {
      u = heads + j * pairs + lights + pair;
    } else {
      const int mine = l < heads ? (heads - l + lights - 1) / lights : 0;
      u = j < mine ? j * lights + l : heads + (j - mine) * pairs + l;
    }
  }
  if (u >= J.units[job]) return {-1, 0, 0, 0, 0, 0};
  const Work &W = J.job[job].w;
  const int kb = (W.K + kBlockK - 1) / kBlockK;  // (times a split: 2^14 x 64 at most)
  Unit t{job, 0, 0, 0, kb, 0};
  if (W.splits > 1) {
    const int per = W.nM * W.nN;
    t.split = u / per;
    u -= t.split * per;
    t.k0 = t.split * kb / W.splits;
    t.k1 = (t.split + 1) * kb / W.splits;
  }
  if (W.rows_first) {
    t.n = u / W.nM;
    t.m = u - t.n * W.nM;
  } else {
    t.m = u / W.nN;
    t.n = u - t.m * W.nN;
  }
  return t;
}

// Shared memory behind the ring: what a kind needs, and from kBoxes on a box for each warp that
// stores them.
constexpr int kBoxBytes = 4096;
template <Kind KIND>
constexpr int kBoxes = KIND == kStatsCols ? kEpiWarps * 32 * kPitch * 4 + 2 * 4 * kMaxTileN * 12
                       : KIND == kCoefCols
                           ? 2 * kMaxTileN * (int)(sizeof(Position) + sizeof(Target))
                           : 0;
template <Kind KIND>
constexpr int kEpi =
    kBoxes<KIND> + (KIND == kStatsCols || KIND == kStatsRows ? 0 : kEpiWarps * kBoxBytes);

// ---- the sums of a tile ----------------------------------------------------------------
struct Stat {
  float m, s, u;
};
// Of 32 logits; c2 > 0.
__device__ __forceinline__ Stat stat_of(const float (&x)[32], float c2) {
  float m = x[0];
#pragma unroll
  for (int i = 1; i < 31; i += 2) m = max_nan(m, x[i], x[i + 1]);
  m = max_nan(m, x[31]);
  if (m == -INFINITY) return {m, 0.f, 0.f};
  const unsigned long long zero = f2_dup(0.f), less = f2_dup(-m), by = f2_dup(c2);
  unsigned long long s[2] = {zero, zero}, u[2] = {zero, zero};
#pragma unroll
  for (int i = 0; i < 32; i += 2) {
    const unsigned long long y = f2_mul(f2_add(f2_pack(x[i], x[i + 1]), less), by);
    float y0, y1;
    f2_split(y, y0, y1);
    const unsigned long long e = f2_pack(exp2_fast(y0), exp2_fast(y1));
    s[i / 2 & 1] = f2_add(s[i / 2 & 1], e);
    u[i / 2 & 1] = f2_fma(y, e, u[i / 2 & 1]);
  }
  Stat r = {m, 0.f, 0.f};
  float a, b;
  f2_split(f2_add(s[0], s[1]), a, b);
  r.s = a + b;
  f2_split(f2_add(u[0], u[1]), a, b);
  r.u = a + b;
  if (isnan(r.u)) {  // (a masked logit: -inf times 0)
    float v = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
      const float y = max_nan((x[i] - m) * c2, kLowest);
      v = fmaf(y, exp2_fast(y), v);
    }
    r.u = v;
  }
  return r;
}
__device__ __forceinline__ void join(Stat &a, Stat b, float c2) {
  if (b.m == -INFINITY) return;
  if (a.m == -INFINITY) {
    a = b;
    return;
  }
  const float m = max_nan(a.m, b.m);
  const float da = max_nan((a.m - m) * c2, kLowest), db = max_nan((b.m - m) * c2, kLowest);
  const float fa = exp2_fast(da), fb = exp2_fast(db);
  a.u = fmaf(da, a.s, a.u) * fa + fmaf(db, b.s, b.u) * fb;
  a.s = a.s * fa + b.s * fb;
  a.m = m;
}

// 32 values of a thread with one rounding each, to a 32-byte boundary.
template <class T>
__device__ __forceinline__ void store_row_of(uint16_t *to, const float (&x)[32]) {
  uint32_t r[16];
#pragma unroll
  for (int i = 0; i < 16; ++i) r[i] = pack2(T{}, x[2 * i], x[2 * i + 1]);
  store32(to, r);
  store32(to + 16, r + 8);
}

// The same to a half (0 or 1) of a row of a box, the lane's.
template <class T>
__device__ __forceinline__ void box_row(uint8_t *box, int half, const float (&x)[32]) {
  const int lane = threadIdx.x & 31;
#pragma unroll
  for (int q = 0; q < 4; ++q)
    *(uint4 *)(box + lane * 128 + (((half * 4 + q) ^ (lane & 7)) << 4)) = {
        pack2(T{}, x[8 * q], x[8 * q + 1]), pack2(T{}, x[8 * q + 2], x[8 * q + 3]),
        pack2(T{}, x[8 * q + 4], x[8 * q + 5]), pack2(T{}, x[8 * q + 6], x[8 * q + 7])};
}

// ---- the kernel --------------------------------------------------------------------------
// MINE > 0: reductions in several parts, whose tiles both groups of warps take together, up to MINE
// chunks of 32 columns each.
template <Kind KIND, class T, int MINE>
__global__ void __launch_bounds__(kThreads, 1) hidden_kernel(const __grid_constant__ Jobs J) {
  constexpr bool kStats = KIND == kStatsCols || KIND == kStatsRows;
  constexpr bool kParted = MINE > 0;
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2],
      drain;
  __shared__ uint32_t tmem_holder;
  __shared__ int abort_flag;
  volatile int *abort = &abort_flag;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31;
  const int rank = blockIdx.x & 1, pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  uint8_t *ring = (uint8_t *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  uint8_t *epi = ring + (size_t)J.stages * J.stage_bytes;

  auto begin = [&]() {  // barriers and tensor memory
    if (tid == 0) {
      for (int s = 0; s < kMaxStages; ++s) {
        mbar_init(&full[s], 1);
        mbar_init(&empty[s], 1);
      }
      for (int i = 0; i < 2; ++i) {
        mbar_init(&acc_full[i], 1);
        // (the warps of both blocks that read it)
        mbar_init(&acc_empty[i], kParted ? 2 * kEpiWarps : kEpiWarps);
      }
      mbar_init(&drain, 1);
      abort_flag = 0;
      fence_mbar_init();
    }
    if (warp == 1) pair_tmem_alloc(&tmem_holder, 512);
    tc_fence_before();
    __syncthreads();
    cluster_sync();
    tc_fence_after();
  };
  // Where few launches find any work, what they need waits until they have.
  const bool asks = kStats && J.far;
  if (!asks) begin();
  pdl_wait();
  pdl_trigger();
  if (asks) {
    const Work &W = J.job[0].w;
    const int n = KIND == kStatsRows ? W.M : W.N;
    bool far = false;  // (alike in both blocks)
    for (int i = tid; i < n; i += kThreads) far |= BOUTE_INB(i, W.Tp) && is_far(W.lse[i]);
    if (!__syncthreads_or(far)) {
      if (tid == 0) W.head->status[blockIdx.x] = 0;
      return;
    }
    begin();
  }
  const uint32_t tmem = tmem_holder;

  if (warp == 0) {
    // ------------------------------------------------------------------ operand tiles
    if (lane == 0) {
      int s = 0, used = 0;
      uint32_t phase = 0;
      for (int i = 0; !*abort; ++i) {
        const Unit t = unit_of<KIND>(J, pair, pairs, i);
        if (t.job < 0) break;
        const Job &job = J.job[KIND == kGrads ? t.job : 0];
        const Work &W = job.w;
        const int half_n = W.tile_n / 2;
        const int m0 = (t.m * 2 + rank) * W.tile_m, n0 = t.n * W.tile_n + rank * half_n;
        for (int kb = t.k0; kb < t.k1; ++kb) {
          if (!pair_wait(&empty[s], phase ^ 1u, abort)) break;
          uint8_t *a = ring + (size_t)s * J.stage_bytes, *b = a + kABytes;
          const uint32_t bar = peer(&full[s], 0);
          if (rank == 0) mbar_arrive_expect_tx(&full[s], 2u * (uint32_t)W.tx_bytes);
          const int k = kb * kBlockK;
          if (KIND == kGrads && W.a_mn) {
            load_box(a, &job.a, m0, k, bar);
            load_box(a + kABytes / 2, &job.a, m0 + 64, k, bar);
          } else {
            load_box(a, &job.a, k, m0, bar);
          }
          if (KIND == kGrads && W.b_mn) {
            for (int q = 0; q < half_n; q += 64) {
              load_box(b + q * 128, &job.b, n0 + q, k, bar);
              if (t.job == 1 && W.low > 0)  // (a box of the first half: the second is the same)
                load_box(b + q * 128 + kBlockK / 2 * 128, &job.b, n0 + q, k, bar);
            }
          } else {
            load_box(b, &job.b, k, n0, bar);
          }
          used = max(used, s + 1);
          if (++s == J.stages) s = 0, phase ^= 1u;
        }
      }
      if (*abort && rank == 0)  // let the copies land before the blocks' memory goes
        for (int i = 0; i < used; ++i) mbar_wait(&full[i], i < s ? phase : phase ^ 1u);
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------------- products
    // (The warp stays together, so that descriptors are in uniform registers: with one lane alone
    // in the loop, issuing took longer than the products, 1.6 PFLOP/s for 2.1.)
    if (rank == 0) {
      constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
      const bool issuer = elect_one();
      int s = 0;
      uint32_t phase = 0, seq = 0;  // seq: accumulators so far
      bool ok = true;
      for (int i = 0; ok; ++i) {
        const Unit t = unit_of<KIND>(J, pair, pairs, i);
        if (t.job < 0) break;
        const Work &W = J.job[KIND == kGrads ? t.job : 0].w;
        const bool a_mn = KIND == kGrads && W.a_mn, b_mn = KIND == kGrads && W.b_mn;
        const uint32_t idesc = pair_idesc(kBf16, a_mn, b_mn, W.tile_n);
        const uint64_t ad0 = operand_desc(smem_u32(ring), a_mn);
        const uint64_t bd0 = operand_desc(smem_u32(ring) + kABytes, b_mn);
        const int a_step = desc_step(a_mn), b_step = desc_step(b_mn);
        const int part = kParted ? J.part : INT_MAX;
        for (int k0 = t.k0; ok && (k0 < t.k1 || k0 == t.k0); ++seq) {
          const int k1 = part < t.k1 - k0 ? k0 + part : t.k1;
          const uint32_t acc = seq & 1u, to = tmem + acc * kMaxTileN;
          ok = __all_sync(kAll, pair_wait<true>(&acc_empty[acc], ((seq >> 1) & 1u) ^ 1u, abort));
          if (!ok) break;
          tc_fence_after();
          for (int kb = k0; kb < k1; ++kb) {
            ok = __all_sync(kAll, pair_wait(&full[s], phase, abort));
            if (!ok) break;
            tc_fence_after();
            if (issuer) {
              const uint64_t at = (uint64_t)((uint32_t)(s * J.stage_bytes) >> 4);
              const uint64_t ad = ad0 + at, bd = bd0 + at;
              const int left = W.K - kb * kBlockK;  // (of a short last block, the steps with data)
#pragma unroll
              for (int k = 0; k < kBlockK / 16; ++k)
                if (k * 16 < left)
                  pair_mma(to, ad + k * a_step, bd + k * b_step, idesc, kb > k0 || k > 0);
              pair_commit(&empty[s]);
            }
            __syncwarp();
            if (++s == J.stages) s = 0, phase ^= 1u;
          }
          if (ok && issuer) pair_commit(&acc_full[acc]);
          __syncwarp();
          if (k1 == t.k0) {  // (an empty part of dh's)
            ++seq;
            break;
          }
          k0 = k1;
        }
      }
      if (!ok && issuer) {  // no product in flight when the tensor memory goes
        pair_commit(&drain);
        mbar_wait(&drain, 0);
      }
    }
  } else {
    // ------------------------------------------------------------ accumulators' tiles
    const int group = (warp - 2) / 4, quarter = warp & 3;
    const int gtid = tid - 64 - group * kGroup;
    const uint32_t from = tmem + ((uint32_t)quarter << 21);
    auto release = [&](int acc) {  // an accumulator, to the issuing warp
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_peer(&acc_empty[acc], 0);
    };
    float mul = 1.f;
    if (!kStats) mul = coef_scale(J.job[0].w.head, J.job[0].w.bounds, KIND == kGrads);
    // (of coefficients of which a wait left out some, no number is written)
    if (KIND == kGrads && *(volatile int *)&J.job[0].w.head->late != 0) mul = NAN;
    uint32_t seq = 0;  // accumulators so far, where both groups take all
    // The groups take the tiles in turn, or, in parts, the first half of each tile's columns one
    // and the rest the other.
    for (int i = kParted ? 0 : group;; i += kParted ? 1 : 2) {
      const Unit t = unit_of<KIND>(J, pair, pairs, i);
      if (t.job < 0) break;
      const Work &W = J.job[KIND == kGrads ? t.job : 0].w;
      const int half = (W.tile_n / 32 + 1) / 2, chunk0 = kParted ? group * half : 0;
      const int chunks = !kParted ? W.tile_n / 32 : group == 0 ? half : W.tile_n / 32 - half;
      const int row = (t.m * 2 + rank) * W.tile_m + quarter * 32;
      const int col = t.n * W.tile_n + chunk0 * 32;
      // what does not wait for the products
      Position *pos = (Position *)epi + group * kMaxTileN;
      Target *tgt = (Target *)(epi + 2 * kMaxTileN * sizeof(Position)) + group * kMaxTileN;
      Position own = {1e30f, 0.f, 0.f, 0.f};
      int target = -1;
      float own_m = 0.f;
      if constexpr (KIND == kCoefCols) {
        named_barrier_sync(1 + group, kGroup);  // (the last tile's are read)
        for (int c = gtid; c < chunks * 32; c += kGroup) {
          Position p = {1e30f, 0.f, 0.f, 0.f};
          Target to = {-1, 0.f};
          if (col + c < W.N && BOUTE_INB(col + c, W.N)) {
            p = W.pos[col + c];
            p.a *= mul, p.b *= mul, p.g *= mul;
            to = W.tgt[col + c];
            to.j -= W.row0;
          }
          pos[c] = p;
          tgt[c] = to;
        }
      } else if constexpr (KIND == kCoefRows) {
        if (row + lane < W.M && BOUTE_INB(row + lane, W.M)) {
          own = W.pos[row + lane];
          own.a *= mul, own.b *= mul, own.g *= mul;
          target = W.tgt[row + lane].j - W.row0;
          own_m = W.tgt[row + lane].m;
        }
      } else if constexpr (KIND == kStatsRows) {
        if (row + lane < W.M && BOUTE_INB(row + lane, W.M)) {
          const long long j = W.targets[row + lane];
          target = j >= 0 && j < W.N ? (int)j : -1;
        }
      }
      Stat run = {-INFINITY, 0.f, 0.f};
      const int red0 = kParted ? chunk0 * 32 : group * 4 * kMaxTileN;
      // 64 columns of 32 rows go out as a box (a row's bytes at once: 268 MB of dW took 77 us by
      // each thread's 32 bytes of its row), a last half by the threads
      uint8_t *box = epi + kBoxes<KIND> + (warp - 2) * kBoxBytes;
      auto send = [&](int c, const float (&x)[32]) {
        const CUtensorMap *out = &J.job[KIND == kGrads ? t.job : 0].out;
        if (c % 2 == 0) {
          if (lane == 0) bulk_wait_read();
          __syncwarp();
        }
        box_row<T>(box, c & 1, x);
        if (c % 2 == 0) return;
        fence_proxy_async_smem();
        __syncwarp();
        if (lane == 0) {
          store_box(out, box, col + (c - 1) * 32, row);
          bulk_commit();
        }
      };
      bool ok = true;
      float sum[kParted ? MINE : 1][32];
      if constexpr (kParted) {
        for (int k0 = t.k0; k0 < t.k1 || k0 == t.k0; k0 += J.part, ++seq) {
          const int acc = seq & 1u;
          ok = __all_sync(kAll, pair_wait(&acc_full[acc], (seq >> 1) & 1u, abort));
          if (!ok) break;
          tc_fence_after();
#pragma unroll
          for (int c = 0; c < MINE; ++c) {
            if (c >= chunks) continue;
#pragma unroll
            for (int h = 0; h < 32; h += 16) {
              float v[16];
              tmem_ld16(from + acc * kMaxTileN + (chunk0 + c) * 32 + h, v);
              if (k0 == t.k0)
#pragma unroll
                for (int q = 0; q < 16; ++q) sum[c][h + q] = 0.f;
#pragma unroll
              for (int q = 0; q < 16; ++q) sum[c][h + q] += v[q];
            }
          }
          release(acc);
        }
      } else {
        ok = __all_sync(kAll, pair_wait(&acc_full[group], (i >> 1) & 1u, abort));
      }
      // (where the group meets at a barrier, it goes on or gives up as one)
      if (KIND == kStatsCols || KIND == kCoefCols) ok = group_all(1 + group, kGroup, ok);
      if (!ok) break;
      if (!kParted) tc_fence_after();
#pragma unroll(kParted ? MINE : 1)
      for (int c = 0; c < (kParted ? MINE : chunks); ++c) {
        if (kParted && c >= chunks) continue;
        float(&x)[32] = sum[kParted ? c : 0];
        if (!kParted) {
          tmem_ld32(from + group * kMaxTileN + c * 32, x);
          if (c == chunks - 1) release(group);
        }
        const int d0 = col + c * 32;
        const bool boxed = c < (chunks & ~1);
        if constexpr (KIND == kStatsCols) {
          float *buf = (float *)epi + (warp - 2) * 32 * kPitch;
          Stat *red = (Stat *)(epi + kEpiWarps * 32 * kPitch * 4) + red0;
          const int at = d0 + lane;
          long long wanted = -1;
          if (at < W.N && BOUTE_INB(at, W.N)) wanted = W.targets[at];
          // (rows of the accumulator beyond the block's hold what was in its shared memory)
          const int rows = min(W.tile_m - quarter * 32, W.M - row);
          if (lane >= rows || W.k != 1.f)
#pragma unroll
            for (int q = 0; q < 32; ++q) x[q] = lane >= rows ? -INFINITY : x[q] * W.k;
#pragma unroll
          for (int q = 0; q < 32; q += 4)
            *(float4 *)(buf + lane * kPitch + q) = {x[q], x[q + 1], x[q + 2], x[q + 3]};
          __syncwarp();
#pragma unroll
          for (int q = 0; q < 32; ++q) x[q] = buf[q * kPitch + lane];
          if (wanted >= row && wanted < row + min(rows, 32))
            W.picked[at] = buf[(int)(wanted - row) * kPitch + lane];
          red[quarter * kMaxTileN + c * 32 + lane] = stat_of(x, W.c2);
          __syncwarp();
        } else if constexpr (KIND == kStatsRows) {
          if (d0 + 32 > W.N || W.k != 1.f)
#pragma unroll
            for (int q = 0; q < 32; ++q) x[q] = d0 + q >= W.N ? -INFINITY : x[q] * W.k;
          if (__any_sync(kAll, target >= d0 && target < d0 + 32))
#pragma unroll
            for (int q = 0; q < 32; ++q)
              if (target == d0 + q) W.picked[row + lane] = x[q];
          join(run, stat_of(x, W.c2), W.c2);
        } else if constexpr (KIND == kCoefCols) {
          const Target aim = tgt[c * 32 + lane];
          const unsigned here = __ballot_sync(kAll, aim.j >= row && aim.j < row + 32);
          if (__any_sync(kAll, aim.m != 0.f))
#pragma unroll
            for (int q = 0; q < 32; ++q) x[q] -= tgt[c * 32 + q].m;
#pragma unroll
          for (int q = 0; q < 32; ++q) {
            const Position p = pos[c * 32 + q];
            const float lp = max_nan(fmaf(x[q], W.scale, -p.ls), -1e4f);
            x[q] = exp2_fast(lp * kLog2e) * fmaf(p.b, lp, p.a);
          }
          if (here)
#pragma unroll
            for (int q = 0; q < 32; ++q)
              if ((here >> q & 1u) && tgt[c * 32 + q].j == row + lane) x[q] += pos[c * 32 + q].g;
          if (d0 + 32 > W.N)  // (columns of no position, which a token of infinities makes NaN)
#pragma unroll
            for (int q = 0; q < 32; ++q)
              if (d0 + q >= W.N) x[q] = 0.f;
          uint16_t *to = W.coef + (row + lane) * W.Tp + d0;
          const bool mine = row + lane < W.M && BOUTE_INB(d0 + 31, W.Tp);
          if (boxed) send(c, x);
          else if (mine) store_row_of<T>(to, x);
          if (W.low > 0 && mine && BOUTE_INB(d0 + W.low + 31, W.Tp)) {
#pragma unroll
            for (int q = 0; q < 32; ++q) x[q] -= to_float(from_float<T>(x[q]));
            store_row_of<T>(to + W.low, x);
          }
        } else if constexpr (KIND == kCoefRows) {
          const unsigned long long by = f2_dup(W.scale), less = f2_dup(-own.ls);
          if (__any_sync(kAll, own_m != 0.f))
#pragma unroll
            for (int q = 0; q < 32; ++q) x[q] -= own_m;
          const unsigned long long a2 = f2_dup(own.a), b2 = f2_dup(own.b), l2e = f2_dup(kLog2e);
#pragma unroll
          for (int q = 0; q < 32; q += 2) {
            float l0, l1, y0, y1;
            f2_split(f2_fma(f2_pack(x[q], x[q + 1]), by, less), l0, l1);
            const unsigned long long lp = f2_pack(max_nan(l0, -1e4f), max_nan(l1, -1e4f));
            f2_split(f2_mul(lp, l2e), y0, y1);
            f2_split(f2_mul(f2_pack(exp2_fast(y0), exp2_fast(y1)), f2_fma(b2, lp, a2)), x[q],
                     x[q + 1]);
          }
          if (__any_sync(kAll, target >= d0 && target < d0 + 32))
#pragma unroll
            for (int q = 0; q < 32; ++q)
              if (target == d0 + q) x[q] += own.g;
          send(c, x);
        } else if (t.job == 0) {  // dh: rows of its elements, columns of the positions
          if (row + lane < W.M && BOUTE_INB(row + lane, W.M)) {
            const int n = min(32, W.N - d0);
            float *to = W.sums + ((long long)t.split * W.N + d0) * W.M + row + lane;
            if (t.k0 == t.k1)  // (a short piece's empty part)
#pragma unroll
              for (int q = 0; q < 32; ++q) x[q] = 0.f;
            if (W.add) {
              float was[32];  // (all on their way at once)
#pragma unroll
              for (int q = 0; q < 32; ++q)
                if (q < n) was[q] = to[(long long)q * W.M];
#pragma unroll
              for (int q = 0; q < 32; ++q)
                if (q < n) x[q] += was[q];
            }
#pragma unroll
            for (int q = 0; q < 32; ++q)
              if (q < n) to[(long long)q * W.M] = x[q];
          }
        } else {  // dW
#pragma unroll
          for (int q = 0; q < 32; ++q) x[q] *= mul;
          T *to = (T *)W.out + (row + lane) * W.ldo + d0;
          if (boxed && W.boxes) {
            send(c, x);
          } else if (boxed) {  // rows at any address: by way of the box, a row by its lanes
            if (c % 2 == 0) __syncwarp();
            box_row<T>(box, c & 1, x);
            if (c % 2 == 1) {
              __syncwarp();
              const int rows = min(32, W.M - row);
              for (int r = 0; r < rows; ++r) {
                T *line = (T *)W.out + (row + r) * W.ldo + d0 - 32;
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                  const int e = h * 32 + lane;
                  const int at = r * 128 + (((e / 8) ^ (r & 7)) << 4) + e % 8 * 2;
                  const T v = *(const T *)(box + at);
                  if (d0 - 32 + e < W.N && BOUTE_INB(row + r, W.M)) line[e] = v;
                }
              }
            }
          } else if (row + lane < W.M && d0 < W.N && BOUTE_INB(row + lane, W.M)) {
            if (d0 + 32 <= W.N && W.width >= 32) {
              store_row_of<T>((uint16_t *)to, x);
            } else if (d0 + 32 <= W.N && W.width >= 16) {
#pragma unroll
              for (int q = 0; q < 32; q += 8)
                *(uint4 *)(to + q) = {
                    pack2(T{}, x[q], x[q + 1]), pack2(T{}, x[q + 2], x[q + 3]),
                    pack2(T{}, x[q + 4], x[q + 5]), pack2(T{}, x[q + 6], x[q + 7])};
            } else {
#pragma unroll
              for (int q = 0; q < 32; ++q)
                if (d0 + q < W.N) to[q] = from_float<T>(x[q]);
            }
          }
        }
        __syncwarp();
      }
      if constexpr (kStats) {
        constexpr int kOf = KIND == kStatsCols || kParted ? 2 : 1;  // (blocks', groups')
        const long long parts = (long long)kOf * (KIND == kStatsCols ? W.nM : W.nN);
        const long long all = parts * W.Tp;
        auto write = [&](Stat a, long long at) {
          if (!BOUTE_INB(at, all)) return;
          W.part[at] = a.m;
          W.part[all + at] = a.s;
          W.part[2 * all + at] = a.u;
        };
        if constexpr (KIND == kStatsCols) {
          named_barrier_sync(1 + group, kGroup);
          const Stat *red = (const Stat *)(epi + kEpiWarps * 32 * kPitch * 4) + red0;
          for (int c = gtid; c < chunks * 32; c += kGroup) {
            Stat a = red[c];
            for (int q = 1; q < 4; ++q) join(a, red[q * kMaxTileN + c], W.c2);
            if (col + c < W.N) write(a, (2ll * t.m + rank) * W.Tp + col + c);
          }
        } else if (row + lane < W.M) {
          write(run, (kParted ? 2ll * t.n + group : t.n) * W.Tp + row + lane);
        }
      }
    }
  }
  if (warp >= 2 && lane == 0) bulk_wait();
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  Header *head = J.job[0].w.head;
  if (tid == 0 && kStats) head->status[blockIdx.x] = *abort ? BOUTE_ERR_TIMEOUT : 0;
  if (tid == 0 && !kStats && *abort) set_status(&head->late, BOUTE_ERR_TIMEOUT);
  cluster_sync();
  if (warp == 1) pair_tmem_dealloc(tmem, 512);
}

// The pieces' sums of kJoinAt positions a block (a sector of each piece's): a warp's lanes are four
// pieces of each, and its warps 32 times those.
constexpr int kJoinWarps = 32, kJoinAt = 8;
__device__ __forceinline__ Stat join_lanes(Stat a, int from, float c2) {
#pragma unroll
  for (int o = 16; o > 0; o >>= 1)
    if (o >= from)
      join(a, {__shfl_xor_sync(kAll, a.m, o), __shfl_xor_sync(kAll, a.s, o),
               __shfl_xor_sync(kAll, a.u, o)}, c2);
  return a;
}
__global__ void __launch_bounds__(32 * kJoinWarps)
    hidden_join_kernel(const Header *head, int blocks, const float *part, const float *picked,
                       const long long *targets, long long T, long long Tp, int parts, int V,
                       float scale, float k, float c2, float *logprob, float *entropy, float *lse) {
  __shared__ Stat red[kJoinAt][kJoinWarps + 1];
  pdl_wait();
  pdl_trigger();
  constexpr int kPieces = 32 / kJoinAt, kAtOnce = 4;  // of a warp; on their way to a thread
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const long long t0 = (long long)blockIdx.x * kJoinAt, all = parts * Tp;
  long long t = t0 + lane % kJoinAt;
  Stat a = {-INFINITY, 0.f, 0.f};
  for (int p0 = warp * kPieces + lane / kJoinAt; p0 < parts;
       p0 += kAtOnce * kJoinWarps * kPieces) {
    Stat b[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int p = p0 + i * kJoinWarps * kPieces;
      const long long at = p * Tp + t;
      b[i] = {-INFINITY, 0.f, 0.f};
      if (p < parts && t < T && BOUTE_INB(at, all))
        b[i] = {part[at], part[all + at], part[2 * all + at]};
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) join(a, b[i], c2);
  }
  a = join_lanes(a, kJoinAt, c2);
  if (lane < kJoinAt) red[lane][warp] = a;
  const bool late = __syncthreads_or(threadIdx.x < blocks && head->status[threadIdx.x] != 0);
  if (warp >= kJoinAt) return;
  a = join_lanes(red[warp][lane], 1, c2);  // a warp's position
  t = t0 + warp;
  if (lane != 0 || t >= T || !BOUTE_INB(t, T)) return;
  const long long target = targets[t];
  const float ls = logf(a.s);
  const float back = k == 1.f ? 1.f : 0.5f;
  const float top = scale * (a.m * back);  // (a scale may take it to an infinity)
  float l = top + ls, H = ls - kLn2 * (a.u / a.s), lp;
  lp = target >= V ? NAN : target < 0 ? 0.f : scale * ((picked[t] - a.m) * back) - ls;
  if (top == -INFINITY) {
    l = -INFINITY;
    H = 0.f;
    lp = target >= V ? NAN : target < 0 ? 0.f : -INFINITY;
  } else if (isnan(a.s) || top == INFINITY) {
    l = H = NAN;
    if (target >= 0) lp = NAN;
  }
  if (late) l = H = lp = NAN;
  logprob[t] = lp;
  entropy[t] = H;
  lse[t] = l;
}

// What each position's coefficients need, of 256 positions a block, and the largest bound of one:
// |p (ln p + H)| < 4 for every distribution over BOUTE_MAX_VOCAB tokens. Positions that have no
// coefficients, or none that are numbers, set no bound: the scale is the others'. Far positions
// take their largest logit and ln s from the statistics' parts.
__global__ void __launch_bounds__(256)
    hidden_positions_kernel(Header *head, int blocks, const long long *targets, long long t0,
                            long long T, int V, float scale, const float *lse,
                            const float *entropy, const float *g_logprob, const float *g_entropy,
                            const float *part, int parts, long long Tp, float k, float c2,
                            Position *pos, Target *tgt) {
  __shared__ unsigned red[8];
  pdl_wait();
  pdl_trigger();
  const long long i = blockIdx.x * 256ll + threadIdx.x, t = t0 + i, all = parts * Tp;
  float bound = 0.f;
  if (t < T && BOUTE_INB(t, T)) {
    const long long target = targets[t];
    const float g = target < 0 ? 0.f : g_logprob[t], gh = g_entropy ? g_entropy[t] : 0.f;
    Position p = {lse[t], -scale * g, -scale * gh, scale * g};
    Target to = {target >= 0 && target < V ? (int)target : -1, 0.f};
    if (g_entropy) p.a -= scale * gh * entropy[t];
    if (is_far(p.ls)) {
      Stat a = {-INFINITY, 0.f, 0.f};
      constexpr int kAtOnce = 8;  // on their way to a thread (one by one 392 took 260 us)
      for (int q0 = 0; q0 < parts; q0 += kAtOnce) {
        Stat b[kAtOnce];
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) {
          const long long at = (q0 + q) * Tp + i;
          b[q] = {-INFINITY, 0.f, 0.f};
          if (q0 + q < parts && BOUTE_INB(at, all)) b[q] = {part[at], part[all + at], 0.f};
        }
#pragma unroll
        for (int q = 0; q < kAtOnce; ++q) join(a, b[q], c2);
      }
      to.m = k == 1.f ? a.m : 0.5f * a.m;
      p.ls = logf(a.s);
    }
    const float most = scale * (fabsf(g) + 4.f * fabsf(gh));
    if (isfinite(most) && p.ls > -INFINITY && target < V) bound = most;
    if (p.ls == -INFINITY) p = {1e30f, 0.f, 0.f, 0.f};  // a row without a token left
    if (target >= V) p.a = NAN;
    pos[t] = p;
    tgt[t] = to;
  }
  const unsigned most = __reduce_max_sync(kAll, __float_as_uint(bound));
  if ((threadIdx.x & 31) == 0) red[threadIdx.x / 32] = most;
  const bool late = __syncthreads_or(threadIdx.x < blocks && head->status[threadIdx.x] != 0);
  if (threadIdx.x == 0) {
    unsigned all = 0;
    for (int w = 0; w < 8; ++w) all = max(all, red[w]);
    head->largest[t0 / 256 + blockIdx.x] = all;
    if (blockIdx.x == 0 && (t0 == 0 || late)) head->late = late ? BOUTE_ERR_TIMEOUT : 0;
  }
}

// dh from the sums of its splits, `each` elements apart, and with low > 0 of their coefficients'
// low parts, low elements on: E neighbouring elements a thread.
template <class T, int E>
__global__ void __launch_bounds__(256)
    hidden_dh_kernel(const Header *head, int bounds, const float *sums, int splits, long long each,
                     long long low, long long rows, int D, T *dh, long long ldd) {
  pdl_wait();
  pdl_trigger();
  const float mul = coef_scale(head, bounds, true);
  const long long i = (blockIdx.x * 256ll + threadIdx.x) * E, n = rows * D;
  if (i >= n) return;
  const long long t = i / D;
  const int d = (int)(i - t * D);
  float v[E];
#pragma unroll
  for (int e = 0; e < E; ++e) v[e] = 0.f;
  constexpr int kAtOnce = E == 1 ? 16 : 4;  // sums on their way to a thread
  const int all = low > 0 ? 2 * splits : splits;
  for (int s0 = 0; s0 < all; s0 += kAtOnce) {
    float x[kAtOnce][E];
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j) {
      const int s = s0 + j;
      const long long at = (s < splits ? s * each : (s - splits) * each + low) + i;
#pragma unroll
      for (int e = 0; e < E; ++e) x[j][e] = 0.f;
      if (s >= all || !BOUTE_INB(at, splits * each)) continue;
      if constexpr (E == 4) {
        const float4 q = *(const float4 *)(sums + at);
        x[j][0] = q.x, x[j][1] = q.y, x[j][2] = q.z, x[j][3] = q.w;
      } else {
        x[j][0] = sums[at];
      }
    }
#pragma unroll
    for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
      for (int e = 0; e < E; ++e) v[e] += x[j][e];
  }
  const bool late = head->late != 0;
#pragma unroll
  for (int e = 0; e < E; ++e) dh[t * ldd + d + e] = from_float<T>(late ? NAN : mul * v[e]);
}

// Rows of D 16-bit elements to a pitch of whole vectors, with zeros behind them.
__global__ void __launch_bounds__(256)
    hidden_align_kernel(const uint16_t *x, long long rows, int D, long long ld, uint16_t *out,
                        int ldo) {
  pdl_wait();
  pdl_trigger();
  const long long i = blockIdx.x * 256ll + threadIdx.x;
  const int per = ldo / 8;
  if (i >= rows * per) return;
  const long long r = i / per;
  const int d0 = (int)(i % per) * 8;
  const char *from = (const char *)(x + r * ld + d0);
  const int sh = (int)((uintptr_t)from & 15), left = 2 * (D - d0);  // bytes of the row from here on
  uint4 a = {0u, 0u, 0u, 0u}, b = a;
  // (words that hold a byte of the row)
  if (left > 0 && BOUTE_INB(d0, ld)) a = *(const uint4 *)(from - sh);
  if (sh != 0 && 16 - sh < left) b = *(const uint4 *)(from - sh + 16);
  a = shifted(a, b, sh);
  uint32_t w[4] = {a.x, a.y, a.z, a.w};
#pragma unroll
  for (int e = 0; e < 4; ++e)
    w[e] = left >= 4 * e + 4 ? w[e] : left >= 4 * e + 2 ? w[e] & 0xffffu : 0u;
  *(uint4 *)(out + r * ldo + d0) = {w[0], w[1], w[2], w[3]};
}

// ---- plans -------------------------------------------------------------------------------
constexpr size_t kCoefBytes = 256u << 20;  // a piece's coefficients at most, in several pieces
constexpr size_t kSumBytes = 128u << 20;   // dh's split sums at most, when split
constexpr long long kAtOnce = 8192;        // positions of one pass of the statistics

long long up(long long x, long long to) { return (x + to - 1) / to * to; }
size_t span(size_t bytes) { return (bytes + 255) / 256 * 256; }

// Columns in tiles of a multiple of 32 up to 256, as even as they come.
void tile_columns(int n, int &tiles, int &width) {
  tiles = (n + kMaxTileN - 1) / kMaxTileN;
  width = (int)up((n + tiles - 1) / tiles, 32);
}

// Whether the positions are the tiles' rows, of which 256 are a tile's whatever there are. The
// statistics gain most where the reduction is short (32768 tokens, in us, rows and columns: 300
// positions of 256 elements 17.3 and 18.5, 515 x 50021 x 1024 48.7 and 49.9, 4096 x 1024 147 and
// 155), the coefficients pass through shared memory either way (gradients: 384 x 256 46 and 49,
// x 1024 92 and 89, 700 x 1024 127 and 130).
bool in_rows(long long T, int D, bool grad) {
  const long long t = up(T, kPairM);
  if (grad) return D < 512 ? 2 * t <= 3 * T : 10 * t <= 11 * T;
  return D < 512 ? 5 * t <= 9 * T : 2 * t <= 3 * T;
}

// A block's rows of a tile, a multiple of 8 up to 128, so that the pairs' rounds over V rows are
// full: where one tile holds the positions, reading the weight bounds the call.
int even_rows(int V) {
  const int pairs = num_sms() / 2;
  const int rounds = (V + kPairM * pairs - 1) / (kPairM * pairs);
  const long long blocks = 2ll * rounds * pairs;
  return (int)std::min<long long>(128, up((V + blocks - 1) / blocks, 8));
}

// A matrix as the copies can read it: in place, or aligned in the workspace. They need rows at
// multiples of 16 bytes; `lines`: where the matrix is read often, of 128, as the 128 bytes that a
// copy takes of a row are then one line.
struct Operand {
  const void *p;
  long long ld;
  bool moved;
};
Operand operand(const void *p, long long rows, int D, long long ld, bool lines) {
  const int most = lines ? 128 : 16;
  const bool ok = (uintptr_t)p % most == 0 && (rows <= 1 || ld % (most / 2) == 0);
  const long long to = up(D, ok || lines ? 64 : 8);
  return {p, !ok || rows <= 1 ? to : ld, !ok};
}

struct Plan {
  Operand h, w;
  bool rows;               // positions in the tiles' rows
  bool fine;               // the coefficients have low parts
  int tiles_t, tile_t;     // of the positions in columns
  int tile_m;              // a block's tokens of the vocabulary (statistics in columns)
  long long part_Tp;       // the pitch of the statistics' parts: positions of one pass
  long long Tp;            // the positions with what the last tile has beyond them
  int piece;               // tokens of the vocabulary at once (gradient)
  int splits;              // of dh's reduction
  size_t header, part, picked, pos, tgt, coef, sums, h_at, w_at, bytes;
  // positions that the coefficients have columns for, and that dh's sums have rows for
  long long columns() const { return fine ? 2 * Tp : Tp; }
  long long sum_rows(long long T) const { return fine ? 2 * Tp : T; }
};

int pairs_of(long long units) {
  return (int)std::min<long long>(units, std::min(num_sms(), kBlocks) / 2);
}
int blocks_of(int k) { return (k + kBlockK - 1) / kBlockK; }

// Blocks of the reduction that a logit takes on the tensor cores at once, as even as they come.
// Their sums cut off what fp32 does not hold, step by step; the parts are added up, rounded, in
// registers. (Entropies of 4096 positions, 5000 tokens: in parts of 16 blocks 3.5e-7 (bf16) and
// 4.7e-7 (fp16) off, of 8 1.5e-7 and 2.1e-7, of 64 2.5e-6. 4096 x 131072 x 4096 takes 2411 us in
// parts of 8, 2375 of 16, and the gradient with 4096 elements 2 % more; with 2048 elements it was
// 2 % more for the statistics, at 515 positions 10, up to 64, where the weight is waited for,
// nothing.)
int part_of(int D, bool few) {
  const int blocks = blocks_of(D), most = few || blocks > 32 ? 8 : 16;
  const int parts = (blocks + most - 1) / most;
  return (blocks + parts - 1) / parts;
}

// The same of dh's reduction over tokens and of dW's over positions, where one is of more than
// grad_long blocks: up to there the steps cut off a quarter of what rounding to the type does, at
// most, half of that on average. (512 tokens, dW of terms of one sign, without and with parts:
// 131072 positions 8.4e-4 and 5e-5 off, 2^20 5.7e-3 and 1.1e-4; in parts throughout, 515 x 50021 x
// 1000 took 181 us for 173.)
constexpr int kGradPart = 64;
constexpr int grad_long(int dtype) { return dtype == BOUTE_F16 ? 256 : 2048; }

// The number of parts of dh's reduction over a piece, each a unit of its own of the pairs: the
// fewest whose units are small beside a pair's share of the whole launch (other: dW's part of it),
// so that dW's units even the pairs out.
int dh_splits(long long tiles, int blocks, int width, double other, size_t each, int pairs) {
  const double share = (tiles * (double)blocks * width + other) / pairs;
  int s = 1;
  while (s < 64 && (s + 1) * 4 <= blocks && (s + 1) * each <= kSumBytes &&
         blocks * (double)width / s > 0.7 * share)
    ++s;
  return s;
}

Plan make_plan(const void *h, long long T, int D, long long ldh, const void *w, int V,
               long long ldw, bool grad) {
  Plan p{};
  const long long t = std::max(1ll, grad ? T : std::min(T, kAtOnce));
  tile_columns((int)t, p.tiles_t, p.tile_t);
  p.rows = in_rows(t, D, grad);
  p.Tp = p.rows ? up(t, kPairM) : (long long)p.tiles_t * p.tile_t;
  // The hidden states are read once for every 256 tokens of the vocabulary, by way of whole lines
  // for more than 128 positions (when it was tried, 515 positions of 1000 elements, 50021 tokens:
  // 70 us in place, 61 so; 4096: 305 and 259; gradient of 515: 223 and 202). The weight is read
  // once for every 256 positions, too seldom for a copy to pay (35 us more, also for the 16 times
  // of 4096 positions).
  p.h = operand(h, T, D, ldh, T > 128);
  // The coefficients of up to half a block's positions are two 16-bit numbers each, the second in
  // the block's other half, where the products are made all the same. (One position's gradient
  // would be its coefficients' rounding off throughout; of many the roundings are apart: 1.35 times
  // the error of the one rounding at the end.)
  p.fine = grad && T <= kBlockK / 2;
  p.w = operand(w, V, D, ldw, false);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at += span(bytes);
    return from;
  };
  p.header = take(sizeof(Header));
  p.tile_m = !grad && !p.rows && p.tiles_t == 1 ? even_rows(V) : 128;
  p.part_Tp = std::min(p.Tp, kAtOnce);
  const long long parts = p.rows ? 2ll * ((V + kMaxTileN - 1) / kMaxTileN)
                                 : 2ll * ((V + 2 * p.tile_m - 1) / (2 * p.tile_m));
  p.picked = take(p.part_Tp * sizeof(float));
  const size_t part = 3 * sizeof(float) * (size_t)(parts * p.part_Tp);
  if (!grad) {
    p.part = take(part);
  } else {
    p.piece = (int)std::min<long long>(
        up(V, kPairM),
        std::max<long long>(kPairM,
                            (long long)(kCoefBytes / (2 * p.columns())) / kPairM * kPairM));
    const size_t each = (size_t)p.sum_rows(T) * D * sizeof(float);
    int tiles_d, tile_d;
    tile_columns(D, tiles_d, tile_d);
    p.splits = dh_splits((long long)((D + kPairM - 1) / kPairM) * p.tiles_t, blocks_of(p.piece),
                         p.fine ? 2 * p.tile_t : p.tile_t,
                         (double)(p.piece / kPairM) * tiles_d * blocks_of((int)p.sum_rows(t)) *
                             tile_d,
                         each,
                         num_sms() / 2);
    p.pos = take(p.Tp * sizeof(Position));
    p.tgt = take(p.Tp * sizeof(Target));
    // (the statistics of far positions come before the coefficients)
    p.part = p.coef = take(std::max<size_t>(part, (size_t)p.piece * p.columns() * 2));
    p.sums = take(p.splits * each);
  }
  if (p.h.moved) p.h_at = take((size_t)T * p.h.ld * 2);
  if (p.w.moved) p.w_at = take((size_t)V * p.w.ld * 2);
  p.bytes = at;
  return p;
}

// A block's bytes of a stage.
int stage_of(const Work &W) {
  const int half = W.tile_n / 2;
  return kABytes + (W.b_mn ? (half + 63) / 64 * 64 : half) * 128;
}

template <Kind KIND, int MINE = 0>
int launch(int dtype, Jobs &J, cudaStream_t s) {
  static_assert(kBoxes<KIND> % 1024 == 0 && sizeof(Stat) == 12, "");
  // as many stages as fit beside the epilogue's shared memory, 1 KB of barriers, 1 KB of alignment
  constexpr size_t kSmem = 232448 - 1024;
  J.stage_bytes = 0;
  for (int i = 0; i < (KIND == kGrads ? 2 : 1); ++i) {
    Work &W = J.job[i].w;
    J.units[i] = W.nM * W.nN * W.splits;
    J.stage_bytes = std::max(J.stage_bytes, stage_of(W));
    W.tx_bytes = stage_of(W) - (128 - W.tile_m) * 128;
  }
  if (KIND != kGrads) J.units[1] = 0;
  J.stages = (int)std::min<size_t>(kMaxStages, (kSmem - 1024 - kEpi<KIND>) / J.stage_bytes);
  const int pairs = pairs_of((long long)J.units[0] + J.units[1]);
  J.light_from = J.units[0] % pairs;
  J.ahead = 0;
  if (KIND == kGrads && J.light_from > 0) {
    const Work &A = J.job[0].w, &B = J.job[1].w;
    // (a long unit of dW costs what 1.15 of dh's do: 1024 positions of 32768 tokens, 2048 elements
    // 287 us without that, 272 with, 4096 positions 943 and 919; 300 of 30000, 512 elements 53 and
    // 54)
    const double each = blocks_of(B.K) * B.tile_n * (blocks_of(B.K) >= 16 ? 1.15 : 1.0);
    J.ahead = (int)((double)blocks_of(A.K) * A.tile_n / A.splits / each);
  }
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    if constexpr (std::is_same<T, float>::value) {
      return (int)BOUTE_ERR_INVALID_ARG;
    } else {
      if (raise_smem(hidden_kernel<KIND, T, MINE>, kSmem) != cudaSuccess)
        return last_launch_status();
      const size_t smem = 1024 + (size_t)J.stages * J.stage_bytes + kEpi<KIND>;
      return launch_cluster(hidden_kernel<KIND, T, MINE>, 2 * pairs, kThreads, 2, smem, s, J);
    }
  });
}

// Copies what the tensor maps cannot read in place.
int align_operand(Operand &x, long long rows, int D, long long ld, char *to, cudaStream_t s) {
  if (!x.moved || rows == 0) return BOUTE_OK;
  const long long n = rows * (x.ld / 8);
  const int r = launch_cluster(hidden_align_kernel, (n + 255) / 256, 256, 1, 0, s,
                               (const uint16_t *)x.p, rows, D, ld, (uint16_t *)to, (int)x.ld);
  x.p = to;
  return r;
}

// A launch that takes logits, in parts; rows, columns: the positions'. The statistics and the
// coefficients take them alike: a far position's x - m is of equal sums, and where all tokens share
// a large term, what the steps beside it cut off is in lse as well. (One of 512, 4096 elements, in
// one part: p 7e-3 off. 130 positions of 32768 tokens, 4096 elements: 2 % of the gradient's time,
// 4096 1.)
template <Kind ROWS, Kind COLUMNS>
int launch_logits(const Plan &p, int dtype, int D, Jobs &J, cudaStream_t s, bool &parted) {
  const bool few = !p.rows && J.job[0].w.tile_n <= 64;
  J.part = part_of(D, few);
  parted = J.part < blocks_of(D);
  if (p.rows) return parted ? launch<ROWS, 4>(dtype, J, s) : launch<ROWS>(dtype, J, s);
  return !parted ? launch<COLUMNS>(dtype, J, s)
         : few   ? launch<COLUMNS, 1>(dtype, J, s)
                 : launch<COLUMNS, 4>(dtype, J, s);
}

// The statistics of n positions from t0 on, in W.part; if W.lse is there, where it has far ones
// alone. parts: of each position, blocks: whose status is written. h_map, w_map: the operands', of
// a caller who has them.
int launch_stats(const Plan &p, int dtype, int D, int V, long long t0, int n, const Work &with,
                 cudaStream_t s, int &parts, int &blocks, const CUtensorMap *h_map = nullptr,
                 const CUtensorMap *w_map = nullptr) {
  Jobs J{};
  Work &W = J.job[0].w;
  W = with;
  W.K = D;
  W.tile_m = p.tile_m;
  W.splits = 1;
  W.Tp = p.part_Tp;
  J.far = W.lse != nullptr;
  CUtensorMap &mh = p.rows ? J.job[0].a : J.job[0].b, &mw = p.rows ? J.job[0].b : J.job[0].a;
  if (p.rows) {
    W.M = n, W.N = V;
    W.nM = (n + kPairM - 1) / kPairM;
    W.nN = parts = (V + kMaxTileN - 1) / kMaxTileN;
    W.tile_n = kMaxTileN;
    W.rows_first = 1;
  } else {
    W.M = V, W.N = n;
    W.nM = (V + 2 * p.tile_m - 1) / (2 * p.tile_m);
    parts = 2 * W.nM;
    tile_columns(n, W.nN, W.tile_n);
  }
  if (w_map) {
    mw = *w_map;
  } else if (int r = make_map(&mw, dtype, p.w.p, D, V, p.w.ld,
                              p.rows ? kMaxTileN / 2 : p.tile_m)) {
    return r;
  }
  if (h_map) {
    mh = *h_map;
  } else if (int r = make_map(&mh, dtype, (const char *)p.h.p + t0 * p.h.ld * 2, D, n, p.h.ld,
                              p.rows ? 128 : W.tile_n / 2)) {
    return r;
  }
  bool parted;
  if (int r = launch_logits<kStatsRows, kStatsCols>(p, dtype, D, J, s, parted)) return r;
  if (parted && p.rows) parts *= 2;  // (of both groups' columns)
  blocks = 2 * pairs_of(J.units[0]);
  return BOUTE_OK;
}

int sizes_ok(const void *h, int dtype, long long T, int D, long long ldh, const void *w, int V,
             long long ldw) {
  if ((dtype != BOUTE_F16 && dtype != BOUTE_BF16) || T < 0 || D < 1 || V < 1 || ldh < D ||
      ldw < D || (T > 0 && !array_ok(h, 2)) || !array_ok(w, 2))
    return dtype == BOUTE_F32 ? BOUTE_ERR_UNSUPPORTED : BOUTE_ERR_INVALID_ARG;
  return T > BOUTE_MAX_HIDDEN || V > BOUTE_MAX_VOCAB || D > BOUTE_MAX_HIDDEN_SIZE
             ? BOUTE_ERR_UNSUPPORTED
             : BOUTE_OK;
}

}  // namespace

BOUTE_BOUNDS_READER(hidden)

int make_map(CUtensorMap *map, int dtype, const void *base, long long inner, long long rows,
             long long ld, int box_rows) {
  using Encode = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *,
                              const cuuint64_t *, const cuuint64_t *, const cuuint32_t *,
                              const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void *f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault,
                                         &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    return (Encode)f;
  }();
  if (!encode) return BOUTE_ERR_CUDA;
  const cuuint64_t dims[2] = {(cuuint64_t)inner, (cuuint64_t)rows}, pitch[1] = {(cuuint64_t)ld * 2};
  const cuuint32_t box[2] = {(cuuint32_t)kBlockK, (cuuint32_t)box_rows}, one[2] = {1, 1};
  return encode(map, dtype == BOUTE_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16
                                        : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16,
                2, const_cast<void *>(base), dims, pitch, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS
             ? BOUTE_OK
             : BOUTE_ERR_CUDA;
}

}  // namespace boute

using namespace boute;

extern "C" int boute_hidden_logprobs_workspace(const void *hidden, int dtype, long long T, int D,
                                               long long ldh, const void *weight, int V,
                                               long long ldw, int grad, long long *bytes) {
  if (!bytes) return BOUTE_ERR_INVALID_ARG;
  if (int r = sizes_ok(hidden, dtype, T, D, ldh, weight, V, ldw)) return r;
  *bytes = (long long)make_plan(hidden, T, D, ldh, weight, V, ldw, grad != 0).bytes;
  return BOUTE_OK;
}

extern "C" int boute_hidden_logprobs(const void *hidden, int dtype, long long T, int D,
                                     long long ldh, const void *weight, int V, long long ldw,
                                     const long long *targets, float scale, float *logprob,
                                     float *entropy, float *lse, void *workspace, long long bytes,
                                     void *stream) {
  BOUTE_TRACE();
  if (!(scale > 0.f) || !isfinite(scale) ||
      (T > 0 && (!array_ok(targets, 8) || !array_ok(logprob, 4) || !array_ok(entropy, 4) ||
                 !array_ok(lse, 4) || !array_ok(workspace, 256))))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = sizes_ok(hidden, dtype, T, D, ldh, weight, V, ldw)) return r;
  Plan p = make_plan(hidden, T, D, ldh, weight, V, ldw, false);
  if (T > 0 && bytes < (long long)p.bytes) return BOUTE_ERR_INVALID_ARG;
  if (T > 0 && outputs_overlap({array_of(logprob, T, 4), array_of(entropy, T, 4),
                                array_of(lse, T, 4), array_of(workspace, p.bytes, 1)},
                               {rows_of(hidden, T, D, ldh, 2), rows_of(weight, V, D, ldw, 2),
                                array_of(targets, T, 8)}))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = device_ok()) return r;
  if (T == 0) return BOUTE_OK;
  const cudaStream_t s = (cudaStream_t)stream;
  char *ws = (char *)workspace;
  if (int r = align_operand(p.h, T, D, ldh, ws + p.h_at, s)) return r;
  if (int r = align_operand(p.w, V, D, ldw, ws + p.w_at, s)) return r;
  Work W{};
  W.head = (Header *)(ws + p.header);
  W.k = logits_by(scale);
  W.c2 = exponents_of(scale);
  W.part = (float *)(ws + p.part);
  W.picked = (float *)(ws + p.picked);
  for (long long t0 = 0; t0 < T; t0 += kAtOnce) {
    const int n = (int)std::min(kAtOnce, T - t0);
    W.targets = targets + t0;
    int parts, blocks;
    if (int r = launch_stats(p, dtype, D, V, t0, n, W, s, parts, blocks)) return r;
    if (int r = launch_cluster(hidden_join_kernel, (n + kJoinAt - 1) / kJoinAt, 32 * kJoinWarps, 1,
                               0, s, W.head, blocks, W.part, W.picked, W.targets, n, p.part_Tp,
                               parts, V, scale, W.k, W.c2, logprob + t0, entropy + t0, lse + t0))
      return r;
  }
  return BOUTE_OK;
}

extern "C" int boute_hidden_logprobs_grad(const void *hidden, int dtype, long long T, int D,
                                          long long ldh, const void *weight, int V, long long ldw,
                                          const long long *targets, float scale, const float *lse,
                                          const float *entropy, const float *g_logprob,
                                          const float *g_entropy, void *dhidden, long long lddh,
                                          void *dweight, long long lddw, void *workspace,
                                          long long bytes, void *stream) {
  BOUTE_TRACE();
  if (!(scale > 0.f) || !isfinite(scale) || lddh < D || lddw < D || !array_ok(dweight, 2) ||
      !optional_ok(entropy, 4) || !optional_ok(g_entropy, 4) || (g_entropy && !entropy && T > 0) ||
      (T > 0 && (!array_ok(targets, 8) || !array_ok(lse, 4) || !array_ok(g_logprob, 4) ||
                 !array_ok(dhidden, 2) || !array_ok(workspace, 256))))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = sizes_ok(hidden, dtype, T, D, ldh, weight, V, ldw)) return r;
  Plan p = make_plan(hidden, T, D, ldh, weight, V, ldw, true);
  if (T > 0 && bytes < (long long)p.bytes) return BOUTE_ERR_INVALID_ARG;
  if (T > 0 && outputs_overlap({rows_of(dhidden, T, D, lddh, 2), rows_of(dweight, V, D, lddw, 2),
                                array_of(workspace, p.bytes, 1)},
                               {rows_of(hidden, T, D, ldh, 2), rows_of(weight, V, D, ldw, 2),
                                array_of(targets, T, 8), array_of(lse, T, 4),
                                array_of(entropy, T, 4), array_of(g_logprob, T, 4),
                                array_of(g_entropy, T, 4)}))
    return BOUTE_ERR_INVALID_ARG;
  if (int r = device_ok()) return r;
  const cudaStream_t s = (cudaStream_t)stream;
  const long long ldo = V > 1 ? lddw : up(D, 8);  // (one row has no pitch)
  if (T == 0)  // (no position: the weight's gradient is 0)
    return cudaMemset2DAsync(dweight, ldo * 2, 0, (size_t)D * 2, V, s) == cudaSuccess
               ? BOUTE_OK
               : last_launch_status();
  char *ws = (char *)workspace;
  const long long both = p.sum_rows(T);  // positions, and with low parts as many again
  if (int r = align_operand(p.h, T, D, ldh, ws + p.h_at, s)) return r;
  if (int r = align_operand(p.w, V, D, ldw, ws + p.w_at, s)) return r;
  Work W{};
  W.head = (Header *)(ws + p.header);
  CUtensorMap h_k, h_mn, w_k;
  if (int r = make_map(&h_k, dtype, p.h.p, D, T, p.h.ld, p.rows ? 128 : p.tile_t / 2)) return r;
  if (int r = make_map(&h_mn, dtype, p.h.p, D, T, p.h.ld, p.fine ? kBlockK / 2 : kBlockK))
    return r;
  if (int r = make_map(&w_k, dtype, p.w.p, D, V, p.w.ld, 128)) return r;
  Position *pos = (Position *)(ws + p.pos);
  Target *tgt = (Target *)(ws + p.tgt);
  W.k = logits_by(scale);
  W.c2 = exponents_of(scale);
  W.part = (float *)(ws + p.part);
  W.picked = (float *)(ws + p.picked);
  for (long long t0 = 0; t0 < T; t0 += kAtOnce) {
    const int n = (int)std::min(kAtOnce, T - t0);
    W.targets = targets + t0;
    W.lse = lse + t0;
    int parts, blocks;
    if (int r = launch_stats(p, dtype, D, V, t0, n, W, s, parts, blocks, n == T ? &h_k : nullptr,
                             &w_k))
      return r;
    if (int r = launch_cluster(hidden_positions_kernel, (n + 255) / 256, 256, 1, 0, s, W.head,
                               blocks, targets, t0, t0 + n, V, scale, lse, entropy, g_logprob,
                               g_entropy, W.part, parts, p.part_Tp, W.k, W.c2, pos, tgt))
      return r;
  }
  W.bounds = (int)((T + 255) / 256);
  W.tile_m = 128;
  W.splits = 1;
  W.pos = pos;
  W.tgt = tgt;
  W.scale = scale;
  W.coef = (uint16_t *)(ws + p.coef);
  W.sums = (float *)(ws + p.sums);
  // a piece's coefficients: tokens x positions, or, with the positions in the tiles' rows, the
  // other way round
  W.Tp = p.rows ? p.piece : p.columns();
  W.low = p.fine ? (int)p.Tp : 0;
  for (int v0 = 0; v0 < V; v0 += p.piece) {
    const int n = std::min(p.piece, V - v0), tiles_v = (n + kPairM - 1) / kPairM;
    const char *w = (const char *)p.w.p + (size_t)v0 * p.w.ld * 2;
    const long long inner = p.rows ? n : both, outer = p.rows ? T : n;  // of the coefficients
    Jobs J{};
    Job &c = J.job[0];
    c.w = W;
    c.w.K = D, c.w.row0 = v0;
    CUtensorMap &mw = p.rows ? c.b : c.a;
    if (n == V) mw = w_k;
    else if (int r = make_map(&mw, dtype, w, D, n, p.w.ld, 128)) return r;
    (p.rows ? c.a : c.b) = h_k;
    if (p.rows) {
      c.w.M = (int)T, c.w.N = n;
      c.w.nM = (int)((T + kPairM - 1) / kPairM), c.w.nN = tiles_v, c.w.tile_n = kMaxTileN;
      c.w.rows_first = 1;
    } else {
      c.w.M = n, c.w.N = (int)T;
      c.w.nM = tiles_v, c.w.nN = p.tiles_t, c.w.tile_n = p.tile_t;
    }
    if (int r = make_map(&c.out, dtype, W.coef, inner, outer, W.Tp, 32)) return r;
    bool parted;
    if (int r = launch_logits<kCoefRows, kCoefCols>(p, dtype, D, J, s, parted)) return r;
    Job &g = J.job[0], &o = J.job[1];
    g.w = W;  // dh: rows of its elements, columns of the positions
    g.w.M = D, g.w.N = (int)both, g.w.K = n;
    g.w.nM = (D + kPairM - 1) / kPairM, g.w.nN = p.tiles_t;
    g.w.tile_n = p.fine ? 2 * p.tile_t : p.tile_t;
    g.w.splits = p.splits;
    g.w.add = v0 > 0;
    g.w.a_mn = 1, g.w.b_mn = !p.rows;
    if (int r = make_map(&g.a, dtype, w, D, n, p.w.ld, kBlockK)) return r;
    if (int r = make_map(&g.b, dtype, W.coef, inner, outer, W.Tp, p.rows ? p.tile_t / 2 : kBlockK))
      return r;
    o.w = W;  // dW of the piece
    o.w.M = n, o.w.N = D, o.w.K = (int)both;
    o.w.nM = tiles_v;
    tile_columns(D, o.w.nN, o.w.tile_n);
    o.w.a_mn = p.rows, o.w.b_mn = 1;
    if (int r = make_map(&o.a, dtype, W.coef, inner, outer, W.Tp, p.rows ? kBlockK : 128)) return r;
    o.b = h_mn;
    o.w.out = (char *)dweight + (size_t)v0 * ldo * 2;
    o.w.ldo = ldo;
    const uint64_t bits = (uintptr_t)dweight | (uint64_t)(ldo * 2);
    o.w.width = bits % 32 == 0 ? 32 : bits % 16 == 0 ? 16 : 2;
    o.w.boxes = bits % 16 == 0;
    if (int r = o.w.boxes ? make_map(&o.out, dtype, o.w.out, D, n, ldo, 32) : 0) return r;
    J.part = kGradPart;
    const bool lengthy =
        std::max(blocks_of((int)both), (blocks_of(n) + p.splits - 1) / p.splits) >
        grad_long(dtype);
    if (int r = lengthy ? launch<kGrads, 4>(dtype, J, s) : launch<kGrads>(dtype, J, s)) return r;
  }
  return with_dtype(dtype, [&](auto t) {
    using E = decltype(t);
    if constexpr (std::is_same<E, float>::value) {
      return (int)BOUTE_ERR_INVALID_ARG;
    } else {
      const long long n = T * D, each = both * D, low = p.fine ? p.Tp * D : 0;
      if (D % 4 == 0 && n >= 1 << 18)  // (few elements take a thread each, to be read by more SMs)
        return launch_cluster(hidden_dh_kernel<E, 4>, (n / 4 + 255) / 256, 256, 1, 0, s, W.head,
                              W.bounds, W.sums, p.splits, each, low, T, D, (E *)dhidden, lddh);
      return launch_cluster(hidden_dh_kernel<E, 1>, (n + 255) / 256, 256, 1, 0, s, W.head, W.bounds,
                            W.sums, p.splits, each, low, T, D, (E *)dhidden, lddh);
    }
  });
}
