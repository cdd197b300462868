// Thin inline-PTX wrappers for the 5th-generation tensor cores: TMEM allocation, tcgen05.mma with operands in shared
// memory or TMEM, TMEM loads and stores, tiled TMA loads.
#pragma once
#include <cuda.h>
#include <stdint.h>

#include "amk_ptx.cuh"

namespace amk {

// ---- descriptors ------------------------------------------------------------------------------------------------
// Shared-memory operand, 128-byte swizzle (what a TMA box of 128-byte rows leaves): start address, the two strides and
// the swizzle mode, all in units of 16 bytes.  K-major: `stride` is the distance between groups of 8 rows.  MN-major:
// `lead` is the distance between blocks of 64 elements along M/N, `stride` between groups of 8 along K.
__device__ __forceinline__ uint64_t smem_desc(unsigned addr, unsigned lead, unsigned stride) {
  return (uint64_t)((addr & 0x3ffff) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(stride >> 4) << 32 |
         (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// kind::f16 with both operands bf16, or both f16, and fp32 accumulators, A K-major; B K-major or (b_mn) MN-major
__host__ __device__ constexpr unsigned mma_idesc(int m, int n, bool b_mn, bool half) {
  return 1u << 4 | (half ? 0u : 1u << 7 | 1u << 10) | (b_mn ? 1u << 16 : 0u) | (unsigned)(n >> 3) << 17 | (unsigned)(m >> 4) << 24;
}

// true in one lane of a converged warp
__device__ __forceinline__ bool elect_one() {
  unsigned r;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(r));
  return r != 0;
}

// ---- tcgen05 ----------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tmem_alloc(unsigned* smem_out, unsigned columns) {   // one whole warp
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(smem_out)), "r"(columns)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tmem_free(unsigned base, unsigned columns) {         // the same warp
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// These three are executed by the whole converged warp and issued by the lane in which `leader` holds: the predicate is
// on the instruction, so that the code around them has no single-lane region and its addresses stay uniform.
__device__ __forceinline__ void mma_ss(bool leader, unsigned d, uint64_t a, uint64_t b, unsigned idesc, bool accumulate) {
  asm volatile(
      "{ .reg .pred p, q; setp.ne.u32 p, %4, 0; setp.ne.u32 q, %5, 0;\n"
      "  @q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"((unsigned)accumulate), "r"((unsigned)leader)
      : "memory");
}
__device__ __forceinline__ void mma_ts(bool leader, unsigned d, unsigned a, uint64_t b, unsigned idesc, bool accumulate) {
  asm volatile(
      "{ .reg .pred p, q; setp.ne.u32 p, %4, 0; setp.ne.u32 q, %5, 0;\n"
      "  @q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"((unsigned)accumulate), "r"((unsigned)leader)
      : "memory");
}
// the barrier gets one arrival when every tcgen05 operation this lane has issued so far is complete
__device__ __forceinline__ void mma_commit(bool leader, uint64_t* bar) {
  asm volatile(
      "{ .reg .pred q; setp.ne.u32 q, %1, 0;\n"
      "  @q tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0]; }" ::"r"(smem_u32(bar)),
      "r"((unsigned)leader)
      : "memory");
}
// 32 columns of this warp's 32 lanes (lane of TMEM = lane of the warp within its quarter)
__device__ __forceinline__ void tmem_ld32(unsigned (&r)[32], unsigned addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
      "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_ld16(unsigned (&r)[16], unsigned addr) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_st16(unsigned addr, const unsigned (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void tmem_st32(unsigned addr, const unsigned (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,"
      "%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(addr),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]),
      "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]), "r"(r[18]),
      "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]),
      "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
// Loaded registers may be used only behind the wait; nothing but this tells the compiler so.
template <int N>
__device__ __forceinline__ void tmem_pin(unsigned (&r)[N]) {
#pragma unroll
  for (int i = 0; i < N; i++) asm volatile("" : "+r"(r[i])::"memory");
}
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- TMA --------------------------------------------------------------------------------------------------------
// One box of a four-dimensional tensor map into shared memory, issued by the leading lane of a converged warp; the byte
// offset of coordinate x is a multiple of 16.
__device__ __forceinline__ void tma_load_4d(bool leader, void* dst, const CUtensorMap* map, int x, int y, int z, int w,
                                            uint64_t* bar) {
  asm volatile(
      "{ .reg .pred q; setp.ne.u32 q, %7, 0;\n"
      "  @q cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2,%3,%4,%5}], [%6]; }" ::"r"(
          smem_u32(dst)),
      "l"(map), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(bar)), "r"((unsigned)leader)
      : "memory");
}
__device__ __forceinline__ void prefetch_map(bool leader, const CUtensorMap* map) {
  asm volatile("{ .reg .pred q; setp.ne.u32 q, %1, 0;\n  @q prefetch.tensormap [%0]; }" ::"l"(map), "r"((unsigned)leader) : "memory");
}
__device__ __forceinline__ void expect_tx(bool leader, uint64_t* bar, unsigned bytes) {
  asm volatile(
      "{ .reg .pred q; setp.ne.u32 q, %2, 0;\n"
      "  @q mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1; }" ::"r"(smem_u32(bar)),
      "r"(bytes), "r"((unsigned)leader)
      : "memory");
}
// Asks the hardware's scheduler for a block of this grid that has not been launched: 16 bytes of answer into shared memory,
// counted on the barrier.  Not to be asked again after an answer without a block.
__device__ __forceinline__ void ask_for_block(bool leader, void* answer, uint64_t* bar) {
  asm volatile(
      "{ .reg .pred q; setp.ne.u32 q, %2, 0;\n"
      "  @q clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1]; }" ::"r"(
          smem_u32(answer)),
      "r"(smem_u32(bar)), "r"((unsigned)leader)
      : "memory");
}
// the x index of the block of an answer, which will not be launched any more; -1: there was none
__device__ __forceinline__ int block_of_answer(const void* answer) {
  int block;
  asm volatile(
      "{ .reg .b128 a; .reg .pred p;\n"
      "  ld.shared.b128 a, [%1];\n"
      "  clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, a;\n"
      "  mov.s32 %0, -1;\n"
      "  @p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %0, a; }"
      : "=r"(block)
      : "r"(smem_u32(answer))
      : "memory");
  return block;
}
// shared memory written by this thread becomes visible to the asynchronous units (tensor cores, TMA)
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

}  // namespace amk
