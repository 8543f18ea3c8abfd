// What a kernel of CTA pairs needs for matrix products on the tensor cores: pairs of blocks that
// share a 256-row accumulator (tcgen05, cta_group::2), tiles brought by tensor-map copies, and
// shared-memory operands in either order. sm_103a only.
#pragma once

#include <cuda.h>

#include "answers.cuh"

namespace boute {

constexpr int kBlockK = 64;    // reduction columns of a stage: 128 bytes of 16-bit elements
constexpr int kPairM = 256;    // rows of a pair's accumulator, 128 a block
constexpr int kMaxTileN = 256;  // its columns; two of them fill the tensor memory

// ---- host: tensor maps ---------------------------------------------------------------
// A matrix of 16-bit elements, `inner` contiguous ones a row of pitch ld, read in boxes of 64 x
// box_rows with the 128-byte swizzle. What lies outside reads as 0. The address is a multiple of 16
// bytes, the pitch of 8 elements (any, for one row).
int make_map(CUtensorMap *map, int dtype, const void *base, long long inner, long long rows,
             long long ld, int box_rows);

#ifdef __CUDACC__
// ---- barriers ------------------------------------------------------------------------
// Waits like mbar_wait, and gives up when *abort is set (which it does where the wait runs out).
// CLUSTER: for what the pair's other block released, too.
template <bool CLUSTER = false>
__device__ __forceinline__ bool pair_wait(uint64_t *bar, uint32_t parity, volatile int *abort) {
  auto done = [&]() {
    if (!CLUSTER) return mbar_try_wait_sleep(bar, parity, 2000u);
    uint32_t ok;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2, %3;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(ok)
        : "r"(smem_u32(bar)), "r"(parity), "r"(2000u)
        : "memory");
    return ok != 0;
  };
  if (done()) return true;
  const uint64_t t0 = globaltimer();
  for (uint32_t it = 1;; ++it) {
    if (done()) return true;
    if ((it & 15) == 0) {
      if (*abort) return false;
      if (globaltimer() - t0 > BOUTE_WAIT_NS) {
        *abort = 1;
        return false;
      }
    }
  }
}
// True in one lane of a whole warp.
__device__ __forceinline__ bool elect_one() {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r));
  return r != 0;
}
// Whether ok holds in all `count` threads that meet at barrier `id`, in each of them.
__device__ __forceinline__ bool group_all(int id, int count, bool ok) {
  uint32_t r;
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 q, %1, 0;\n\t"
      "barrier.cta.red.and.pred p, %2, %3, q;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t}"
      : "=r"(r)
      : "r"((uint32_t)ok), "r"(id), "r"(count)
      : "memory");
  return r != 0;
}
// One arrival at a barrier of the pair's block r, which hands over tensor memory (that its loads
// are done is for tc_fence_before): no memory of this thread's, whose stores it would wait for at
// the scope of the cluster (gradient of 64 x 32768 x 4096: 180 us, so 157).
__device__ __forceinline__ void arrive_peer(uint64_t *bar, int r) {
  asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(peer(bar, r))
               : "memory");
}

// ---- copies --------------------------------------------------------------------------
// A box from column x (a multiple of 8) and row y on, to this block's shared memory; its bytes
// count on the barrier at `bar`, an address of either block's.
__device__ __forceinline__ void load_box(void *dst, const CUtensorMap *map, int x, int y,
                                         uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes"
      ".cta_group::2 [%0], [%1, {%2, %3}], [%4];" ::"r"(smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}

// ---- tensor memory and products --------------------------------------------------------
__device__ __forceinline__ void pair_tmem_alloc(uint32_t *dst_smem, uint32_t ncols) {
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(
                   smem_u32(dst_smem)),
               "r"(ncols)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void pair_tmem_dealloc(uint32_t taddr, uint32_t ncols) {
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols)
               : "memory");
}

// Shared-memory operands are in 128-byte rows with the 128-byte swizzle, eight rows an atom of
// 1024 bytes. Where the reduction is contiguous (K-major), a row holds 64 reduction columns of an
// operand row, and 16 of them are 32 bytes on. Where the operand's rows are contiguous (MN-major),
// a row holds one reduction column of 64 operand rows, blocks of 64 operand rows follow one another
// kBlockK rows apart, and 16 reduction columns are 2048 bytes on.
__device__ __forceinline__ uint64_t operand_desc(uint32_t saddr, bool mn) {
  uint64_t d = sdesc_sw128(saddr);
  if (mn) d = (d & ~((uint64_t)0x3fff << 16)) | (uint64_t)((kBlockK * 128) >> 4) << 16;
  return d;
}
// Of 16 reduction columns.
__device__ __forceinline__ int desc_step(bool mn) { return mn ? 2048 >> 4 : 32 >> 4; }

// kind::f16, fp32 accumulators, 256 x n; A and B of one type, each MN-major or not.
__host__ __device__ constexpr uint32_t pair_idesc(bool bf16, bool a_mn, bool b_mn, int n) {
  return (1u << 4) | ((bf16 ? 1u : 0u) << 7) | ((bf16 ? 1u : 0u) << 10) |
         ((a_mn ? 1u : 0u) << 15) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) |
         ((uint32_t)(kPairM >> 4) << 24);
}
__device__ __forceinline__ void pair_mma(uint32_t tmem_d, uint64_t adesc, uint64_t bdesc,
                                         uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(tmem_d),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}
// An arrival at this barrier of both blocks once the products issued so far are done.
__device__ __forceinline__ void pair_commit(uint64_t *bar) {
  asm volatile(
      "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 "
      "[%0], %1;" ::"r"(smem_u32(bar)),
      "h"((uint16_t)3)
      : "memory");
}

// 32 consecutive columns of this warp's 32 lanes.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, float (&v)[32]) {
  uint32_t r[32];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]),
        "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]),
        "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 32; ++i) v[i] = __uint_as_float(r[i]);
}

// 16 of them.
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, float (&v)[16]) {
  uint32_t r[16];
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,"
      "%15}, [%16];\n\t"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]),
        "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]),
        "=r"(r[14]), "=r"(r[15])
      : "r"(taddr)
      : "memory");
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = __uint_as_float(r[i]);
}

// 32 rows of 64 16-bit elements from shared memory (4 KB on a 1 KB boundary, swizzled) to column x
// (a multiple of 8) and row y on; what lies outside is not written.
__device__ __forceinline__ void store_box(const CUtensorMap *map, const void *src, int x, int y) {
  asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(
                   map),
               "r"(x), "r"(y), "r"(smem_u32(src))
               : "memory");
}

// 32 bytes to a 32-byte boundary.
__device__ __forceinline__ void store32(void *p, const uint32_t *r) {
  asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};" ::"l"(p), "r"(r[0]), "r"(r[1]),
               "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
#endif

}  // namespace boute
