// Wrappers around the tensor-core, tensor-memory, tensor-map copy and cluster instructions the
// 8-bit product uses (PTX ISA, sm_100a).
#pragma once

#include <cuda.h>

#include "kb_common.cuh"

namespace kb {

// ---- tensor memory ---------------------------------------------------------------------------
template <int CG>
__device__ __forceinline__ void tmem_alloc(uint32_t* dst_smem, uint32_t cols) {   // one whole warp
  if constexpr (CG == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst_smem)),
                 "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  } else {
    asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(dst_smem)),
                 "r"(cols)
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
  }
}
template <int CG>
__device__ __forceinline__ void tmem_free(uint32_t addr, uint32_t cols) {
  if constexpr (CG == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
  else
    asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(addr), "r"(cols));
}
__device__ __forceinline__ void tc_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

// 16 or 32 columns of this warp's 32 lanes; the values are there after tmem_wait_ld, which names them, so that
// the compiler moves no arithmetic on them in front of the wait
__device__ __forceinline__ void tmem_ld16(uint32_t addr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_ld32(uint32_t addr, float* v) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr));
}
__device__ __forceinline__ void tmem_wait_ld(float (&v)[16]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
}
__device__ __forceinline__ void tmem_wait_ld(float (&v)[32]) {
  uint32_t* r = reinterpret_cast<uint32_t*>(v);
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]),
                 "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15])::"memory");
  asm volatile(""
               : "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                 "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]));
}

// ---- matrix instructions ---------------------------------------------------------------------
// Descriptor of a K-major operand in shared memory, rows of 128 bytes in the 128-byte swizzle
// (what a tensor-map copy with that swizzle writes): start address and the distance of 1024
// bytes between groups of 8 rows, both in units of 16 bytes; the bit at 46 is the descriptor
// version of this architecture and 2 at bits 61..63 names the swizzle.
__device__ __forceinline__ uint64_t smem_desc_k128(uint32_t smem_addr) {
  return (uint64_t)((smem_addr & 0x3FFFFu) >> 4) | (1ull << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) |
         (2ull << 61);
}
// Instruction descriptor: binary32 accumulator, 8-bit float operands (0: e4m3, 1: e5m2), both
// K-major, tile of M rows and N columns.
__host__ __device__ constexpr uint32_t mma_idesc_f8(bool a_e5m2, bool b_e5m2, uint32_t M, uint32_t N) {
  return (1u << 4) | ((a_e5m2 ? 1u : 0u) << 7) | ((b_e5m2 ? 1u : 0u) << 10) | ((N >> 3) << 17) | ((M >> 4) << 24);
}
// D = A B^T over one K block of 128 bytes (four steps of 32).  The whole warp calls it with equal
// arguments and one thread of it issues: operands that are the same for the warp stay in uniform
// registers, where a single thread's would have to be moved there for every instruction (250 cycles
// per block instead of 60).
template <int CG>
__device__ __forceinline__ void mma_f8_block(uint32_t d_tmem, uint64_t a_desc, uint64_t b_desc, uint32_t idesc) {
  if constexpr (CG == 1)
    asm volatile(
        "{\n.reg .pred one, more;\n.reg .b64 a, b;\n"
        "elect.sync _|one, 0xFFFFFFFF;\n"
        "setp.ne.b32 more, 0, 0;\n"
        "@one tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, more;\n"
        "setp.eq.b32 more, 0, 0;\n"
        "add.s64 a, %1, 2;\nadd.s64 b, %2, 2;\n"
        "@one tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %3, more;\n"
        "setp.eq.b32 more, 0, 0;\n"
        "add.s64 a, %1, 4;\nadd.s64 b, %2, 4;\n"
        "@one tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %3, more;\n"
        "setp.eq.b32 more, 0, 0;\n"
        "add.s64 a, %1, 6;\nadd.s64 b, %2, 6;\n"
        "@one tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], a, b, %3, more;\n"
        "}" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc)
        : "memory");
  else
    asm volatile(
        "{\n.reg .pred one, more;\n.reg .b64 a, b;\n"
        "elect.sync _|one, 0xFFFFFFFF;\n"
        "setp.ne.b32 more, 0, 0;\n"
        "@one tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, more;\n"
        "setp.eq.b32 more, 0, 0;\n"
        "add.s64 a, %1, 2;\nadd.s64 b, %2, 2;\n"
        "@one tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a, b, %3, more;\n"
        "setp.eq.b32 more, 0, 0;\n"
        "add.s64 a, %1, 4;\nadd.s64 b, %2, 4;\n"
        "@one tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a, b, %3, more;\n"
        "setp.eq.b32 more, 0, 0;\n"
        "add.s64 a, %1, 6;\nadd.s64 b, %2, 6;\n"
        "@one tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], a, b, %3, more;\n"
        "}" ::"r"(d_tmem), "l"(a_desc), "l"(b_desc), "r"(idesc)
        : "memory");
}
// The barrier gets one arrival when all matrix instructions of this warp's issuing thread are done
// (whole warp; the same thread is elected every time).
__device__ __forceinline__ void mma_commit(uint64_t* bar) {
  asm volatile(
      "{\n.reg .pred one;\nelect.sync _|one, 0xFFFFFFFF;\n"
      "@one tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(smem_u32(bar))
      : "memory");
}
// The same for a pair of CTAs: one arrival on the barrier at this place in both of them.
__device__ __forceinline__ void mma_commit_pair(uint64_t* bar) {
  asm volatile(
      "{\n.reg .pred one;\nelect.sync _|one, 0xFFFFFFFF;\n"
      "@one tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;\n}" ::"r"(
          smem_u32(bar)),
      "h"((unsigned short)3)
      : "memory");
}

// ---- tensor-map copies -----------------------------------------------------------------------
// Called by a whole warp with equal arguments, like the matrix instructions above; one thread issues.
// 2-D box of a row-major matrix to this CTA's shared memory; x (bytes here) is a multiple of 16.
__device__ __forceinline__ void tma_load_2d(uint32_t dst_smem, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "{\n.reg .pred one;\nelect.sync _|one, 0xFFFFFFFF;\n"
      "@one cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3}], [%4];\n}" ::"r"(dst_smem),
      "l"(map), "r"(x), "r"(y), "r"(bar)
      : "memory");
}
// The same by a CTA of a pair; the bytes count on a barrier of either CTA (a cluster address).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst_smem, const CUtensorMap* map, int x, int y,
                                                 uint32_t cluster_bar) {
  asm volatile(
      "{\n.reg .pred one;\nelect.sync _|one, 0xFFFFFFFF;\n"
      "@one cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes "
      "[%0], [%1, {%2, %3}], [%4];\n}" ::"r"(dst_smem),
      "l"(map), "r"(x), "r"(y), "r"(cluster_bar)
      : "memory");
}
// Announces bytes on a barrier of this CTA (whole warp, one arrival)
__device__ __forceinline__ void expect_tx_elect(uint32_t bar, uint32_t bytes) {
  asm volatile(
      "{\n.reg .pred one;\nelect.sync _|one, 0xFFFFFFFF;\n"
      "@one mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n}" ::"r"(bar),
      "r"(bytes)
      : "memory");
}

// ---- registers ---------------------------------------------------------------------------------
// Executed by all warps of a warpgroup; the shares of a CTA's warpgroups must not add up to more
// than the registers it was launched with.
template <int N>
__device__ __forceinline__ void regs_shrink() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_grow() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}

// ---- clusters --------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync_all() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_arrive() {
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t map_to_rank(uint32_t smem_addr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr), "r"(rank));
  return r;
}
__device__ __forceinline__ void st_cluster_f32x4(uint32_t addr, float x, float y, float z, float w) {
  asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(x), "f"(y), "f"(z), "f"(w)
               : "memory");
}

// Arrival on a barrier of any CTA of the cluster.  No cluster-wide release (which would wait for
// every earlier memory access of the thread): it hands over tensor memory, whose accesses the
// tcgen05 fences order.
// Predicated inside the statement: no branch for the warp to come together after.
__device__ __forceinline__ void mbar_arrive_cluster_if(uint32_t cluster_bar, bool yes) {
  asm volatile(
      "{\n.reg .pred p;\nsetp.ne.u32 p, %1, 0;\n@p mbarrier.arrive.shared::cluster.b64 _, [%0];\n}" ::"r"(cluster_bar),
      "r"(yes ? 1u : 0u)
      : "memory");
}

// The same on a barrier of this CTA
__device__ __forceinline__ void mbar_arrive_if(uint64_t* bar, bool yes) {
  asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %1, 0;\n@p mbarrier.arrive.shared::cta.b64 _, [%0];\n}" ::"r"(smem_u32(bar)),
               "r"(yes ? 1u : 0u)
               : "memory");
}

// ---- small asynchronous copies -----------------------------------------------------------------
// One binary32 value global -> shared, or zero where `in` is false (the source is not read).
__device__ __forceinline__ void cp_async_f32(float* dst_smem, const float* src, bool in) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst_smem)), "l"(src), "r"(in ? 4 : 0)
               : "memory");
}
// One arrival when all earlier cp.async of this thread have landed.
__device__ __forceinline__ void cp_async_arrive(uint64_t* bar) {
  asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}

}  // namespace kb
