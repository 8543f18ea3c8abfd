// Log-probabilities of given tokens from a model's last hidden states and its vocabulary's
// weight, without the logits, and the gradient with respect to both.
//
// With x = h . w_j (fp32, of 16-bit products), c = scale log2 e, and per token of the vocabulary's
// pieces m = max x, s = sum 2^((x - m) c), u = sum (x - m) c 2^((x - m) c):
//   lse = scale m + ln s,  logprob = scale (x_t - m) - ln s,  entropy = ln s - ln 2 u / s.
// The gradient takes the logits again, piece by piece of the vocabulary, as coefficients
//   c_tj = scale (g ([j = t] - p_j) - g_H p_j (ln p_j + H)),
// of which dh = c W and dW = c^T h are two more products.
//
// All products run on the tensor cores: a pair of blocks takes tiles of 256 tokens of the
// vocabulary (rows) x up to 256 positions (columns), one warp bringing operand tiles, one issuing
// products, and two groups of four warps taking the accumulators' tiles in turn, so that a tile's
// sums or stores go on behind the next one's products.
#include <float.h>
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

enum Mode { kStats = 0, kCoef = 1, kDHidden = 2, kDWeight = 3 };

// At the start of a call's workspace.
constexpr int kBlocks = 256;  // of a launch at most
struct Header {
  // BOUTE_ERR_TIMEOUT where a wait ran out: of each block of the statistics' launch, which writes
  // its own; of all launches of the gradient, which clears it first
  int status[kBlocks];
  unsigned largest;  // bits of the largest bound of a coefficient (gradient)
};
// What the coefficients of a position need.
struct Position {
  float lse, a, b, g;  // p (a + b ln p), + g at its target
};

// The power of two by which the coefficients are scaled while they are 16-bit numbers: the largest
// comes to 2^14 (fp16: what is 2^-28 of that has all its bits, and 2^-39 some).
__device__ __forceinline__ float coef_scale(unsigned largest, bool inverse) {
  const int e = (int)(largest >> 23) - 127;  // (the largest is in [2^e, 2^(e + 1)))
  if (largest == 0u || largest >= 0x7f800000u) return 1.f;
  const int k = min(max(13 - e, -126), 126);
  return exp2i(inverse ? -k : k);
}

struct Work {
  int M, N, K;             // rows, columns, reduction
  int tile_m, tile_n, nM, nN, splits;  // (tile_m: rows of a block, 128 but for few positions)
  int stages, stage_bytes, tx_bytes;  // (of a block; what its copies bring)
  Header *head;
  // statistics
  float c2;
  float *part;             // 3 x parts x Tp: maxima, s, u
  float *picked;           // Tp: x of the targets
  const long long *targets;
  long long Tp;
  // coefficients
  const Position *pos;
  const int *tgt;          // targets, -1 for none
  float scale;
  uint16_t *coef;          // M x Tp
  int row0;                // of the piece in the vocabulary
  // gradients
  float *sums;             // splits x N x M
  int add;                 // to what earlier pieces left there
  char *out;               // M x N, pitch ldo
  long long ldo;
  int width;               // bytes that the rows' alignment allows in a store
};

struct Unit {
  int m, n, k0, k1;  // tiles; blocks of the reduction
};
__device__ __forceinline__ Unit unit_of(const Work &W, int u) {
  const int kb = (W.K + kBlockK - 1) / kBlockK;  // (times a split: 2^14 x 64 at most)
  int s = 0, r = u, k0 = 0, k1 = kb;
  if (W.splits > 1) {
    const int per = W.nM * W.nN;
    s = u / per;
    r = u - s * per;
    k0 = s * kb / W.splits;
    k1 = (s + 1) * kb / W.splits;
  }
  const int m = r / W.nN;
  return {m, r - m * W.nN, k0, k1};
}

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
  float s[4] = {0.f, 0.f, 0.f, 0.f}, u[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < 32; ++i) {
    const float y = (x[i] - m) * c2, e = exp2_fast(y);
    s[i & 3] += e;
    u[i & 3] = fmaf(y, e, u[i & 3]);
  }
  Stat r = {m, (s[0] + s[1]) + (s[2] + s[3]), (u[0] + u[1]) + (u[2] + u[3])};
  if (isnan(r.u)) {  // (a masked logit: -inf times 0)
    float v = 0.f;
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

// ---- the kernel --------------------------------------------------------------------------
template <Mode MODE, class T>
__global__ void __launch_bounds__(kThreads, 1)
    hidden_kernel(const __grid_constant__ CUtensorMap map_a,
                  const __grid_constant__ CUtensorMap map_b, const Work W) {
  constexpr bool kAMn = MODE == kDHidden, kBMn = MODE == kDHidden || MODE == kDWeight;
  extern __shared__ uint8_t raw[];
  __shared__ __align__(8) uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2],
      drain;
  __shared__ uint32_t tmem_holder;
  __shared__ int abort_flag;
  volatile int *abort = &abort_flag;
  const int tid = threadIdx.x, warp = tid / 32, lane = tid & 31;
  const int rank = blockIdx.x & 1, pair = blockIdx.x / 2, pairs = gridDim.x / 2;
  uint8_t *ring = (uint8_t *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
  uint8_t *epi = ring + (size_t)W.stages * W.stage_bytes;
  const int units = W.nM * W.nN * W.splits;
  const int half_n = W.tile_n / 2;

  if (tid == 0) {
    for (int s = 0; s < kMaxStages; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], 1);
    }
    for (int i = 0; i < 2; ++i) {
      mbar_init(&acc_full[i], 1);
      mbar_init(&acc_empty[i], kEpiWarps);  // a group's four warps of both blocks
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
  const uint32_t tmem = tmem_holder;
  pdl_wait();
  pdl_trigger();

  if (warp == 0) {
    // ------------------------------------------------------------------ operand tiles
    if (lane == 0) {
      int s = 0, used = 0;
      uint32_t phase = 0;
      for (int u = pair; u < units && !*abort; u += pairs) {
        const Unit t = unit_of(W, u);
        const int m0 = (t.m * 2 + rank) * W.tile_m, n0 = t.n * W.tile_n + rank * half_n;
        for (int kb = t.k0; kb < t.k1; ++kb) {
          if (!pair_wait(&empty[s], phase ^ 1u, abort)) break;
          uint8_t *a = ring + (size_t)s * W.stage_bytes, *b = a + kABytes;
          const uint32_t bar = peer(&full[s], 0);
          if (rank == 0) mbar_arrive_expect_tx(&full[s], 2u * (uint32_t)W.tx_bytes);
          const int k = kb * kBlockK;
          if constexpr (kAMn) {
            load_box(a, &map_a, m0, k, bar);
            load_box(a + kABytes / 2, &map_a, m0 + 64, k, bar);
          } else {
            load_box(a, &map_a, k, m0, bar);
          }
          if constexpr (kBMn) {
            for (int q = 0; q < half_n; q += 64) load_box(b + q * 128, &map_b, n0 + q, k, bar);
          } else {
            load_box(b, &map_b, k, n0, bar);
          }
          used = max(used, s + 1);
          if (++s == W.stages) s = 0, phase ^= 1u;
        }
      }
      if (*abort && rank == 0)  // let the copies land before the blocks' memory goes
        for (int i = 0; i < used; ++i) mbar_wait(&full[i], i < s ? phase : phase ^ 1u);
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------------- products
    // (The warp stays together, so that descriptors are in uniform registers: with one lane alone in
    // the loop, issuing took longer than the products.)
    if (rank == 0) {
      constexpr bool kBf16 = std::is_same<T, __nv_bfloat16>::value;
      const uint32_t idesc = pair_idesc(kBf16, kAMn, kBMn, W.tile_n);
      const bool issuer = elect_one();
      const uint64_t ad0 = operand_desc<kAMn>(smem_u32(ring));
      const uint64_t bd0 = operand_desc<kBMn>(smem_u32(ring) + kABytes);
      int s = 0;
      uint32_t phase = 0, seq = 0;
      bool ok = true;
      for (int u = pair; u < units && ok; u += pairs, ++seq) {
        const Unit t = unit_of(W, u);
        const uint32_t acc = seq & 1u, to = tmem + acc * kMaxTileN;
        ok = __all_sync(kAll, pair_wait<true>(&acc_empty[acc], ((seq >> 1) & 1u) ^ 1u, abort));
        if (!ok) break;
        tc_fence_after();
        for (int kb = t.k0; kb < t.k1; ++kb) {
          ok = __all_sync(kAll, pair_wait(&full[s], phase, abort));
          if (!ok) break;
          tc_fence_after();
          if (issuer) {
            const uint64_t at = (uint64_t)((uint32_t)(s * W.stage_bytes) >> 4);
            const uint64_t ad = ad0 + at, bd = bd0 + at;
            const int left = W.K - kb * kBlockK;  // (of a short last block, the steps with data)
#pragma unroll
            for (int k = 0; k < kBlockK / 16; ++k)
              if (k * 16 < left)
                pair_mma(to, ad + k * kDescStep<kAMn>, bd + k * kDescStep<kBMn>, idesc,
                         kb > t.k0 || k > 0);
            pair_commit(&empty[s]);
          }
          __syncwarp();
          if (++s == W.stages) s = 0, phase ^= 1u;
        }
        if (ok && issuer) pair_commit(&acc_full[acc]);
        __syncwarp();
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
    const uint32_t from = tmem + ((uint32_t)quarter << 21) + group * kMaxTileN;
    auto release = [&]() {  // the group's accumulator, to the issuing warp
      tc_fence_before();
      __syncwarp();
      if (lane == 0) arrive_peer(&acc_empty[group], 0);
    };
    const int chunks = W.tile_n / 32;
    float mul = 1.f;
    if (MODE != kStats) mul = coef_scale(W.head->largest, MODE != kCoef);
    uint32_t seq = 0;
    for (int u = pair; u < units; u += pairs, ++seq) {
      if ((seq & 1u) != (uint32_t)group) continue;
      const Unit t = unit_of(W, u);
      const int row = (t.m * 2 + rank) * W.tile_m + quarter * 32, col = t.n * W.tile_n;
      // what does not wait for the products
      Position *pos = (Position *)epi + group * kMaxTileN;
      int *tgt = (int *)(epi + 2 * kMaxTileN * sizeof(Position)) + group * kMaxTileN;
      if constexpr (MODE == kCoef) {
        named_barrier_sync(1 + group, kGroup);  // (the last tile's are read)
        for (int c = gtid; c < W.tile_n; c += kGroup) {
          Position p = {1e30f, 0.f, 0.f, 0.f};
          int j = -1;
          if (col + c < W.N && BOUTE_INB(col + c, W.N)) {
            p = W.pos[col + c];
            p.a *= mul, p.b *= mul, p.g *= mul;
            j = W.tgt[col + c] - W.row0;
          }
          pos[c] = p;
          tgt[c] = j;
        }
      }
      // (where the group meets at a barrier, it goes on or gives up as one)
      bool ok = __all_sync(kAll, pair_wait(&acc_full[group], (seq >> 1) & 1u, abort));
      if (MODE == kStats || MODE == kCoef) ok = group_all(1 + group, kGroup, ok);
      if (!ok) break;
      tc_fence_after();
      for (int c = 0; c < chunks; ++c) {
        float x[32];
        tmem_ld32(from + c * 32, x);
        if (c == chunks - 1) release();
        if (MODE == kDHidden && t.k0 == t.k1)  // (a short piece's empty part)
#pragma unroll
          for (int i = 0; i < 32; ++i) x[i] = 0.f;
        if constexpr (MODE == kStats) {
          float *buf = (float *)epi + (warp - 2) * 32 * kPitch;
          Stat *red = (Stat *)(epi + kEpiWarps * 32 * kPitch * 4) + group * 4 * kMaxTileN;
          const int at = col + c * 32 + lane;
          long long target = -1;
          if (at < W.N && BOUTE_INB(at, W.N)) target = W.targets[at];
          // (rows of the accumulator beyond the block's hold what was in its shared memory)
          const int rows = min(W.tile_m - quarter * 32, W.M - row);
          if (lane >= rows)
#pragma unroll
            for (int i = 0; i < 32; ++i) x[i] = -INFINITY;
#pragma unroll
          for (int i = 0; i < 32; i += 4)
            *(float4 *)(buf + lane * kPitch + i) = {x[i], x[i + 1], x[i + 2], x[i + 3]};
          __syncwarp();
#pragma unroll
          for (int i = 0; i < 32; ++i) x[i] = buf[i * kPitch + lane];
          if (target >= row && target < row + min(rows, 32))
            W.picked[at] = buf[(int)(target - row) * kPitch + lane];
          red[quarter * kMaxTileN + c * 32 + lane] = stat_of(x, W.c2);
          __syncwarp();
        } else if constexpr (MODE == kCoef) {
          const int j = tgt[c * 32 + lane];
          unsigned here = __ballot_sync(kAll, j >= row && j < row + 32);
#pragma unroll
          for (int i = 0; i < 32; ++i) {
            const Position p = pos[c * 32 + i];
            const float lp = max_nan(fmaf(x[i], W.scale, -p.lse), -1e4f);
            x[i] = exp2_fast(lp * kLog2e) * fmaf(p.b, lp, p.a);
          }
          if (here)
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if ((here >> i & 1u) && tgt[c * 32 + i] == row + lane) x[i] += pos[c * 32 + i].g;
          if (row + lane < W.M && BOUTE_INB(col + c * 32 + 31, W.Tp)) {
            uint32_t r[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] = pack2(T{}, x[2 * i], x[2 * i + 1]);
            uint16_t *to = W.coef + (row + lane) * W.Tp + col + c * 32;
            store32(to, r);
            store32(to + 16, r + 8);
          }
        } else if constexpr (MODE == kDHidden) {
          if (row + lane < W.M) {
            const int n = min(32, W.N - col - c * 32);
            float *to = W.sums + ((long long)(u / (W.nM * W.nN)) * W.N + col + c * 32) * W.M + row +
                        lane;
            if (W.add && BOUTE_INB(row + lane, W.M)) {
              float was[32];  // (all on their way at once)
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (i < n) was[i] = to[(long long)i * W.M];
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (i < n) x[i] += was[i];
            }
#pragma unroll
            for (int i = 0; i < 32; ++i)
              if (i < n && BOUTE_INB(row + lane, W.M)) to[(long long)i * W.M] = x[i];
          }
        } else {
          const int d0 = col + c * 32;
          if (row + lane < W.M && d0 < W.N && BOUTE_INB(row + lane, W.M)) {
            T *to = (T *)W.out + (row + lane) * W.ldo + d0;
            uint32_t r[16];
#pragma unroll
            for (int i = 0; i < 16; ++i) r[i] = pack2(T{}, mul * x[2 * i], mul * x[2 * i + 1]);
            if (d0 + 32 <= W.N && W.width >= 32) {
              store32(to, r);
              store32(to + 16, r + 8);
            } else if (d0 + 32 <= W.N && W.width >= 16) {
#pragma unroll
              for (int i = 0; i < 4; ++i)
                *(uint4 *)(to + 8 * i) = {r[4 * i], r[4 * i + 1], r[4 * i + 2], r[4 * i + 3]};
            } else {
#pragma unroll
              for (int i = 0; i < 32; ++i)
                if (d0 + i < W.N) to[i] = from_float<T>(mul * x[i]);
            }
          }
        }
      }
      if constexpr (MODE == kStats) {
        named_barrier_sync(1 + group, kGroup);
        const Stat *red =
            (const Stat *)(epi + kEpiWarps * 32 * kPitch * 4) + group * 4 * kMaxTileN;
        const long long parts = 2ll * W.nM, all = parts * W.Tp;
        for (int c = gtid; c < W.tile_n; c += kGroup) {
          Stat a = red[c];
          for (int q = 1; q < 4; ++q) join(a, red[q * kMaxTileN + c], W.c2);
          const long long at = (2ll * t.m + rank) * W.Tp + col + c;
          if (col + c >= W.N || !BOUTE_INB(at, all)) continue;
          W.part[at] = a.m;
          W.part[all + at] = a.s;
          W.part[2 * all + at] = a.u;
        }
      }
    }
  }
  __syncwarp();
  tc_fence_before();
  __syncthreads();
  if (tid == 0 && MODE == kStats) W.head->status[blockIdx.x] = *abort ? BOUTE_ERR_TIMEOUT : 0;
  if (tid == 0 && MODE != kStats && *abort) set_status(W.head->status, BOUTE_ERR_TIMEOUT);
  cluster_sync();
  if (warp == 1) pair_tmem_dealloc(tmem, 512);
}

// The pieces' sums of 32 positions a block: lanes over the positions, warps over the pieces.
constexpr int kJoinWarps = 32;
__global__ void __launch_bounds__(32 * kJoinWarps)
    hidden_join_kernel(const Header *head, int blocks, const float *part, const float *picked,
                       const long long *targets, long long T, long long Tp, int parts, int V,
                       float scale, float c2, float *logprob, float *entropy, float *lse) {
  __shared__ Stat red[kJoinWarps][32];
  pdl_wait();
  pdl_trigger();
  const int lane = threadIdx.x & 31, warp = threadIdx.x / 32;
  const long long t = blockIdx.x * 32ll + lane, all = parts * Tp;
  Stat a = {-INFINITY, 0.f, 0.f};
  constexpr int kAtOnce = 8;  // parts on their way to a thread
  for (int p0 = warp; p0 < parts; p0 += kAtOnce * kJoinWarps) {
    Stat b[kAtOnce];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) {
      const int p = p0 + i * kJoinWarps;
      const long long at = p * Tp + t;
      b[i] = {-INFINITY, 0.f, 0.f};
      if (p < parts && t < T && BOUTE_INB(at, all))
        b[i] = {part[at], part[all + at], part[2 * all + at]};
    }
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i) join(a, b[i], c2);
  }
  const bool late = __syncthreads_or(threadIdx.x < blocks && head->status[threadIdx.x] != 0);
  red[warp][lane] = a;
  __syncthreads();
  for (int n = kJoinWarps / 2; n > 0; n /= 2) {
    if (warp < n) {
      a = red[warp][lane];
      join(a, red[warp + n][lane], c2);
      red[warp][lane] = a;
    }
    __syncthreads();
  }
  if (warp != 0 || t >= T || !BOUTE_INB(t, T)) return;
  const long long target = targets[t];
  const float ls = logf(a.s);
  float l = scale * a.m + ls, H = ls - kLn2 * (a.u / a.s), lp;
  lp = target >= V ? NAN : target < 0 ? 0.f : scale * (picked[t] - a.m) - ls;
  if (a.m == -INFINITY) {
    l = -INFINITY;
    H = 0.f;
    lp = target >= V ? NAN : target < 0 ? 0.f : -INFINITY;
  } else if (isnan(a.s)) {
    l = H = NAN;
    if (target >= 0) lp = NAN;
  }
  if (late) l = H = lp = NAN;
  logprob[t] = lp;
  entropy[t] = H;
  lse[t] = l;
}

// What each position's coefficients need, and the largest bound of one: |p (ln p + H)| < 4 for
// every distribution over BOUTE_MAX_VOCAB tokens.
__global__ void __launch_bounds__(256)
    hidden_positions_kernel(Header *head, const long long *targets, long long T, int V,
                            float scale, const float *lse, const float *entropy,
                            const float *g_logprob, const float *g_entropy, Position *pos,
                            int *tgt) {
  pdl_wait();
  pdl_trigger();
  const long long t = blockIdx.x * 256ll + threadIdx.x;
  float bound = 0.f;
  if (t < T && BOUTE_INB(t, T)) {
    const long long target = targets[t];
    const float g = target < 0 ? 0.f : g_logprob[t], gh = g_entropy ? g_entropy[t] : 0.f;
    Position p = {lse[t], -scale * g, -scale * gh, scale * g};
    if (g_entropy) p.a -= scale * gh * entropy[t];
    bound = scale * (fabsf(g) + 4.f * fabsf(gh));
    if (p.lse == -INFINITY) p = {1e30f, 0.f, 0.f, 0.f};  // a row without a token left
    if (target >= V) p.a = NAN;
    pos[t] = p;
    tgt[t] = target >= 0 && target < V ? (int)target : -1;
  }
  const unsigned most = __reduce_max_sync(kAll, __float_as_uint(bound));
  if ((threadIdx.x & 31) == 0 && most) atomicMax(&head->largest, most);
}

// dh from the sums of its splits.
template <class T>
__global__ void __launch_bounds__(256)
    hidden_dh_kernel(const Header *head, const float *sums, int splits, long long rows, int D,
                     T *dh, long long ldd) {
  pdl_wait();
  pdl_trigger();
  const long long i = blockIdx.x * 256ll + threadIdx.x, n = rows * D;
  if (i >= n) return;
  float v = 0.f;
  for (int s = 0; s < splits; ++s)
    if (BOUTE_INB(s * n + i, splits * n)) v += sums[s * n + i];
  v *= coef_scale(head->largest, true);
  if (head->status[0] != 0) v = NAN;
  dh[i / D * ldd + i % D] = from_float<T>(v);
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
  uint32_t w[4] = {0u, 0u, 0u, 0u};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (d0 + e < D && BOUTE_INB(d0 + e, ld)) w[e / 2] |= (uint32_t)x[r * ld + d0 + e] << 16 * (e & 1);
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

// A block's rows of a tile, a multiple of 8 up to 128, so that the pairs' rounds over V rows are
// full: where one tile holds the positions, reading the weight bounds the call.
int even_rows(int V) {
  const int pairs = num_sms() / 2;
  const int rounds = (V + kPairM * pairs - 1) / (kPairM * pairs);
  return (int)std::min<long long>(128, up((V + 2ll * rounds * pairs - 1) / (2ll * rounds * pairs), 8));
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
  int tiles_t, tile_t;     // of the positions
  int tile_m;              // a block's tokens of the vocabulary (statistics)
  long long Tp;
  int piece;               // tokens of the vocabulary at once (gradient)
  int splits;              // of dh's reduction
  size_t header, part, picked, pos, tgt, coef, sums, h_at, w_at, bytes;
};

// The number of parts of dh's reduction, of which each is a product of its own: the pairs' rounds
// over them, each 1 / splits as long, and 1 % for every part's sums.
int dh_splits(long long units, int blocks, size_t each, int pairs) {
  int best = 1;
  double least = 1e30;
  for (int s = 1; s <= 64 && s * 8 <= std::max(blocks, 8); ++s) {
    if (s > 1 && s * each > kSumBytes) break;
    const double cost = (double)((units * s + pairs - 1) / pairs) / s * (1.0 + 0.01 * s);
    if (cost < least) least = cost, best = s;
  }
  return best;
}

Plan make_plan(const void *h, long long T, int D, long long ldh, const void *w, int V,
               long long ldw, bool grad) {
  Plan p{};
  const long long t = grad ? T : std::min(T, kAtOnce);
  tile_columns((int)std::max(t, 1ll), p.tiles_t, p.tile_t);
  p.Tp = (long long)p.tiles_t * p.tile_t;
  // The hidden states are read once for every 256 tokens of the vocabulary (515 positions of 1000
  // elements, 50021 tokens: 70 us in place, 61 by way of whole lines; 4096: 305 and 259; gradient of
  // 515: 223 and 202). The weight is read once for every 256 positions, too seldom for a copy to pay
  // (another 35 us, also for the 16 reads of 4096 positions).
  p.h = operand(h, T, D, ldh, T > 128);
  p.w = operand(w, V, D, ldw, false);
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t from = at;
    at += span(bytes);
    return from;
  };
  p.header = take(sizeof(Header));
  if (!grad) {
    p.tile_m = p.tiles_t == 1 ? even_rows(V) : 128;
    p.part = take(3ull * 2 * ((V + 2 * p.tile_m - 1) / (2 * p.tile_m)) * p.Tp * sizeof(float));
    p.picked = take(p.Tp * sizeof(float));
  } else {
    p.piece = (int)std::min<long long>(
        V, std::max<long long>(kPairM, (long long)(kCoefBytes / (2 * p.Tp)) / kPairM * kPairM));
    int tiles_d = (D + kPairM - 1) / kPairM;
    const size_t each = (size_t)T * D * sizeof(float);
    p.splits = dh_splits((long long)tiles_d * p.tiles_t, (p.piece + kBlockK - 1) / kBlockK, each,
                         num_sms() / 2);
    // (a last piece that is shorter than the splits leaves some of them nothing to add)
    p.pos = take(p.Tp * sizeof(Position));
    p.tgt = take(p.Tp * sizeof(int));
    p.coef = take((size_t)p.piece * p.Tp * 2);
    p.sums = take(p.splits * each);
  }
  if (p.h.moved) p.h_at = take((size_t)T * p.h.ld * 2);
  if (p.w.moved) p.w_at = take((size_t)V * p.w.ld * 2);
  p.bytes = at;
  return p;
}

// The rings of a launch: as many stages as fit beside the epilogue's shared memory.
size_t set_stages(Work &W, bool b_mn, size_t epi) {
  const int half = W.tile_n / 2;
  W.stage_bytes = kABytes + (b_mn ? (half + 63) / 64 * 64 : half) * 128;
  W.tx_bytes = W.stage_bytes - (128 - W.tile_m) * 128;
  const size_t room = 232448 - 1024 - 1024 - epi;  // (1 KB of barriers, 1 KB of alignment)
  W.stages = (int)std::min<size_t>(kMaxStages, room / W.stage_bytes);
  return 1024 + (size_t)W.stages * W.stage_bytes + epi;
}

int pairs_of(long long units) {
  return (int)std::min<long long>(units, std::min(num_sms(), kBlocks) / 2);
}

template <Mode MODE>
int launch(int dtype, const CUtensorMap &a, const CUtensorMap &b, Work W, cudaStream_t s) {
  constexpr bool kBMn = MODE == kDHidden || MODE == kDWeight;
  const size_t epi = MODE == kStats ? kEpiWarps * 32 * kPitch * 4 + 2 * 4 * kMaxTileN * sizeof(Stat)
                     : MODE == kCoef ? 2 * kMaxTileN * (sizeof(Position) + sizeof(int))
                                     : 0;
  const size_t smem = set_stages(W, kBMn, epi);
  const long long units = (long long)W.nM * W.nN * W.splits;
  const int pairs = pairs_of(units);
  return with_dtype(dtype, [&](auto t) {
    using T = decltype(t);
    if constexpr (std::is_same<T, float>::value) {
      return (int)BOUTE_ERR_INVALID_ARG;
    } else {
      if (cudaFuncSetAttribute((const void *)hidden_kernel<MODE, T>,
                               cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem) !=
          cudaSuccess)
        return last_launch_status();
      return launch_cluster(hidden_kernel<MODE, T>, 2 * pairs, kThreads, 2, smem, s, a, b, W);
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
  if (int r = device_ok()) return r;
  if (T == 0) return BOUTE_OK;
  const cudaStream_t s = (cudaStream_t)stream;
  char *ws = (char *)workspace;
  if (int r = align_operand(p.h, T, D, ldh, ws + p.h_at, s)) return r;
  if (int r = align_operand(p.w, V, D, ldw, ws + p.w_at, s)) return r;
  CUtensorMap mw, mh;
  if (int r = make_map(&mw, dtype, p.w.p, D, V, p.w.ld, p.tile_m)) return r;
  Work W{};
  W.M = V;
  W.K = D;
  W.tile_m = p.tile_m;
  W.nM = (V + 2 * p.tile_m - 1) / (2 * p.tile_m);
  W.splits = 1;
  W.head = (Header *)(ws + p.header);
  W.c2 = scale * kLog2e;
  W.part = (float *)(ws + p.part);
  W.picked = (float *)(ws + p.picked);
  W.Tp = p.Tp;
  for (long long t0 = 0; t0 < T; t0 += kAtOnce) {
    const int n = (int)std::min(kAtOnce, T - t0);
    W.N = n;
    tile_columns(n, W.nN, W.tile_n);
    W.targets = targets + t0;
    if (int r = make_map(&mh, dtype, (const char *)p.h.p + t0 * p.h.ld * 2, D, n, p.h.ld,
                         W.tile_n / 2))
      return r;
    if (int r = launch<kStats>(dtype, mw, mh, W, s)) return r;
    if (int r = launch_cluster(hidden_join_kernel, (n + 31) / 32, 32 * kJoinWarps, 1, 0, s, W.head,
                               2 * pairs_of((long long)W.nM * W.nN), W.part, W.picked, W.targets, n, W.Tp, 2 * W.nM, V, scale, W.c2,
                               logprob + t0, entropy + t0, lse + t0))
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
  if (int r = device_ok()) return r;
  const cudaStream_t s = (cudaStream_t)stream;
  if (T == 0)  // (no position: the weight's gradient is 0)
    return cudaMemset2DAsync(dweight, lddw * 2, 0, (size_t)D * 2, V, s) == cudaSuccess
               ? BOUTE_OK
               : last_launch_status();
  char *ws = (char *)workspace;
  if (cudaMemsetAsync(ws, 0, sizeof(Header), s) != cudaSuccess) return last_launch_status();
  if (int r = align_operand(p.h, T, D, ldh, ws + p.h_at, s)) return r;
  if (int r = align_operand(p.w, V, D, ldw, ws + p.w_at, s)) return r;
  Work W{};
  W.head = (Header *)(ws + p.header);
  W.tile_m = 128;
  Position *pos = (Position *)(ws + p.pos);
  int *tgt = (int *)(ws + p.tgt);
  if (int r = launch_cluster(hidden_positions_kernel, (T + 255) / 256, 256, 1, 0, s, W.head,
                             targets, T, V, scale, lse, entropy, g_logprob, g_entropy, pos, tgt))
    return r;
  W.pos = pos;
  W.tgt = tgt;
  W.scale = scale;
  W.Tp = p.Tp;
  W.coef = (uint16_t *)(ws + p.coef);
  W.sums = (float *)(ws + p.sums);
  CUtensorMap h_k, h_mn;
  if (int r = make_map(&h_k, dtype, p.h.p, D, T, p.h.ld, p.tile_t / 2)) return r;
  if (int r = make_map(&h_mn, dtype, p.h.p, D, T, p.h.ld, kBlockK)) return r;
  for (int v0 = 0; v0 < V; v0 += p.piece) {
    const int n = std::min(p.piece, V - v0);
    const char *w = (const char *)p.w.p + (size_t)v0 * p.w.ld * 2;
    CUtensorMap w_k, w_mn, c_k, c_mn;
    if (int r = make_map(&w_k, dtype, w, D, n, p.w.ld, 128)) return r;
    if (int r = make_map(&w_mn, dtype, w, D, n, p.w.ld, kBlockK)) return r;
    if (int r = make_map(&c_k, dtype, W.coef, T, n, p.Tp, 128)) return r;
    if (int r = make_map(&c_mn, dtype, W.coef, T, n, p.Tp, kBlockK)) return r;
    const int tiles_v = (n + kPairM - 1) / kPairM;
    Work C = W;  // the coefficients of the piece
    C.M = n, C.N = (int)T, C.K = D;
    C.nM = tiles_v, C.nN = p.tiles_t, C.tile_n = p.tile_t, C.splits = 1;
    C.row0 = v0;
    if (int r = launch<kCoef>(dtype, w_k, h_k, C, s)) return r;
    Work G = W;  // dh: rows of its elements, columns of the positions
    G.M = D, G.N = (int)T, G.K = n;
    G.nM = (D + kPairM - 1) / kPairM, G.nN = p.tiles_t, G.tile_n = p.tile_t;
    G.splits = p.splits;
    G.add = v0 > 0;
    if (int r = launch<kDHidden>(dtype, w_mn, c_mn, G, s)) return r;
    Work O = W;  // dW of the piece
    O.M = n, O.N = D, O.K = (int)T;
    O.nM = tiles_v;
    tile_columns(D, O.nN, O.tile_n);
    O.splits = 1;
    O.out = (char *)dweight + (size_t)v0 * lddw * 2;
    O.ldo = lddw;
    const uint64_t bits = (uintptr_t)dweight | (uint64_t)(lddw * 2);
    O.width = bits % 32 == 0 ? 32 : bits % 16 == 0 ? 16 : 2;
    if (int r = launch<kDWeight>(dtype, c_k, h_mn, O, s)) return r;
  }
  const long long n = T * D;
  return with_dtype(dtype, [&](auto t) {
    using E = decltype(t);
    if constexpr (std::is_same<E, float>::value) {
      return (int)BOUTE_ERR_INVALID_ARG;
    } else {
      return launch_cluster(hidden_dh_kernel<E>, (n + 255) / 256, 256, 1, 0, s, W.head, W.sums,
                            p.splits, T, D, (E *)dhidden, lddh);
    }
  });
}
