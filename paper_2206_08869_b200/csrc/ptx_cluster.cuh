// Instructions beside those of ptx.cuh: tile copies through a tensor map, clusters, MMAs of CTA pairs, waits in line.
#pragma once
#include "ptx.cuh"

namespace iodf {
namespace ptx {

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}

// bounded_wait for a thread that may have copies or MMAs under way. Where it gives up, the CTA gives up: each of its threads gets here, stops
// and meets the others at the end of the kernel, where tensor memory is freed and the CTA leaves. What the thread has asked for has to end
// before: it reads this GPU's memory and takes microseconds, so ten milliseconds, in at most a thousand naps.
static __device__ __noinline__ bool settled_wait(volatile uint32_t* abort_flag, uint32_t* status, uint64_t* bar, uint32_t parity,
                                                 uint32_t limit) {
  const uint32_t b = smem_u32(bar);
  for (uint32_t it = 0; it < limit && !*abort_flag; ++it)
    if (mbar_try_wait(b, parity)) return true;
  if (!*abort_flag) {
    *abort_flag = 1;
    atomicExch(status, 1u);
  }
  const long long start = clock64();
  for (int i = 0; i < 1000 && clock64() - start < 20000000; ++i) __nanosleep(100000);
  return false;
}

// The same with the first try in line: a call costs some 145 ns, as much as a stage's copies take to issue.
__device__ __forceinline__ bool quick_wait(volatile uint32_t* abort_flag, uint32_t* status, uint64_t* bar, uint32_t parity,
                                           uint32_t limit) {
  if (mbar_try_wait(smem_u32(bar), parity)) return true;
  return settled_wait(abort_flag, status, bar, parity, limit);
}

// ---- tile of a row-major matrix global -> shared through a tensor map (128-byte swizzle), completion counted on an
// mbarrier; col in elements with col * element size a multiple of 16. Beyond the matrix zeros arrive.
__device__ __forceinline__ void tile_g2s(uint32_t dst, const void* map, int32_t col, int32_t row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(col), "r"(row), "r"(bar)
      : "memory");
}

// ---- thread-block clusters ---------------------------------------------------------------------
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
// Both by all threads of all CTAs of the cluster; shared memory written before the arrival is visible to the cluster after the wait.
// `.aligned` wants the whole warp at the instruction: lanes that parted before meet here.
__device__ __forceinline__ void cluster_arrive() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void cluster_wait() {
  __syncwarp();
  asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// Address of the same shared-memory word in CTA `rank` of the cluster, and a store to it.
__device__ __forceinline__ uint32_t cluster_addr(uint32_t saddr, uint32_t rank) {
  uint32_t r;
  asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(saddr), "r"(rank));
  return r;
}
__device__ __forceinline__ void st_cluster(uint32_t addr, uint32_t v) {
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}

// ---- CTA pairs (clusters of two): one tcgen05.mma over both, M = 256 -------------------------------
// Issued by CTA 0. Each CTA holds its 128 rows of A and of D, and one half of the rows of B, at the same shared-memory
// and tensor-memory addresses.
__device__ __forceinline__ void tmem_alloc_pair(uint32_t smem_dst, uint32_t cols) {  // a warp of each CTA
  asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_dst), "r"(cols));
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::);
}
__device__ __forceinline__ void tmem_dealloc_pair(uint32_t taddr, uint32_t cols) {   // a warp of each CTA
  asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(cols));
}
__device__ __forceinline__ void umma_i8_hl_pair(uint32_t d_tmem, uint32_t a_lo, uint32_t a_hi, uint32_t b_lo, uint32_t b_hi,
                                                uint32_t idesc, uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t.reg .b64 da, db;\n\t"
      "mov.b64 da, {%1, %2};\n\t"
      "mov.b64 db, {%3, %4};\n\t"
      "setp.ne.b32 p, %6, 0;\n\t"
      "tcgen05.mma.cta_group::2.kind::i8 [%0], da, db, %5, p;\n\t}" ::"r"(d_tmem),
      "r"(a_lo), "r"(a_hi), "r"(b_lo), "r"(b_hi), "r"(idesc), "r"(accumulate)
      : "memory");
}
// The tile copy of tile_g2s whose bytes are counted on a barrier of either CTA of the pair (address from cluster_addr).
__device__ __forceinline__ void tile_g2s_pair(uint32_t dst, const void* map, int32_t col, int32_t row, uint32_t bar) {
  asm volatile(
      "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(dst),
      "l"(map), "r"(col), "r"(row), "r"(bar)
      : "memory");
}
// Arrive on the barrier at this address in both CTAs once every tcgen05.mma issued so far by this thread has completed.
__device__ __forceinline__ void umma_commit_pair(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(bar),
               "h"((uint16_t)3)
               : "memory");
}
// Arrive on a barrier of any CTA of the cluster (address from cluster_addr), releasing at cluster scope.
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t addr) {
  asm volatile("mbarrier.arrive.release.cluster.shared::cluster.b64 _, [%0];" ::"r"(addr) : "memory");
}

}  // namespace ptx
}  // namespace iodf
