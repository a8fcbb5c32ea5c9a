// Instructions and operand layouts of the attention kernels, beside those of ptx_cluster.cuh.
#pragma once
#include "ptx_cluster.cuh"

namespace iodf {
namespace ptx {

// 32 lanes x 32 bit, 32 consecutive columns: thread i of the warp reads lane (base + i). The wait is for all of the warp's loads; r, of one of
// them, is valid from there on.
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr));
}
__device__ __forceinline__ void tmem_ld_wait32(uint32_t (&r)[32]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31]) : : "memory");
}
__device__ __forceinline__ void tmem_ld4(uint32_t taddr, uint32_t (&r)[4]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(taddr));
}

// Of a word that does not change any more.
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
  uint32_t v;
  asm("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
  return v;
}
__device__ __forceinline__ void sts128(uint32_t addr, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// All `threads` threads (whole warps) wait for one another; none of them may leave its loop unless all do.
__device__ __forceinline__ void named_barrier(int id, int threads) {
  __syncwarp();
  asm volatile("bar.sync %0, %1;" ::"r"(id), "r"(threads) : "memory");
}
// The same, and whether `mine` is true of all of them.
__device__ __forceinline__ bool all_agree(int id, int threads, bool mine) {
  uint32_t all;
  __syncwarp();
  asm volatile(
      "{\n\t.reg .pred p, q;\n\t"
      "setp.ne.u32 p, %1, 0;\n\t"
      "bar.red.and.pred q, %2, %3, p;\n\t"
      "selp.u32 %0, 1, 0, q;\n\t}"
      : "=r"(all)
      : "r"((uint32_t)mine), "r"(id), "r"(threads)
      : "memory");
  return all != 0;
}

}  // namespace ptx

// Operands of rows of `width` bytes (32, 64 or 128), K-major and swizzled over the width as a TMA copy leaves them: 16-byte piece c of
// row r lies at swizzled(r, c, width). Tiles start at multiples of 1024 bytes. Descriptor words: the start address (a
// step of 32 bytes along K adds 2), and groups of eight rows 8 * width apart with the swizzle's code.
__device__ __forceinline__ uint32_t swizzled(int r, int c, int width) {
  const int turn = width == 128 ? r & 7 : width == 64 ? (r >> 1) & 3 : (r >> 2) & 1;
  return (uint32_t)(r * width + ((c ^ turn) << 4));
}
__device__ __forceinline__ uint32_t rows_lo(uint32_t saddr) { return ptx::umma_desc_lo(saddr, 16u); }
__device__ __forceinline__ constexpr uint32_t rows_hi(int width) {
  return (uint32_t)(8 * width >> 4) | (1u << 14) | ((width == 128 ? 2u : width == 64 ? 4u : 6u) << 29);
}
// D = s32, A and B 8-bit integers, both K-major, M = m, N = n
__device__ __forceinline__ constexpr uint32_t idesc_i8(int m, int n, bool a_unsigned, bool b_unsigned) {
  return (2u << 4) | ((a_unsigned ? 0u : 1u) << 7) | ((b_unsigned ? 0u : 1u) << 10) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(m >> 4) << 24);
}

}  // namespace iodf
