// Fifth-generation tensor cores: tensor memory, operand descriptors, and the instructions that
// the products with 4-bit weights use.
#pragma once

#include "sp_tma.cuh"

namespace sp {

// ---- tensor memory (512 columns of 128 lanes x 32 bits on an SM)

// One warp allocates; the base address lands in shared memory.  columns: a power of two >= 32.
// PAIR: for products of a pair of blocks; a warp of each block allocates and frees.
template <bool PAIR = false>
__device__ __forceinline__ void tmem_alloc(uint32_t *dst, uint32_t columns) {
    if constexpr (PAIR) {
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(dst)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;");
    } else {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(dst)), "r"(columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
}
template <bool PAIR = false>
__device__ __forceinline__ void tmem_free(uint32_t base, uint32_t columns) {
    if constexpr (PAIR) asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
    else asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns) : "memory");
}
__device__ __forceinline__ void tcgen05_fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tcgen05_fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
// Arrives on the barrier (PAIR: of both blocks) when all tensor-core work this thread issued before
// has completed.
template <bool PAIR = false>
__device__ __forceinline__ void tcgen05_commit(uint32_t bar) {
    if constexpr (PAIR)
        asm volatile("tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;"
                     ::"r"(bar), "h"(static_cast<uint16_t>(3)) : "memory");
    else
        asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// 32 columns of this warp's 32 lanes (lanes 32 * (warp % 4) and following).
__device__ __forceinline__ void tmem_load32(uint32_t addr, uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]),
          "=r"(v[8]), "=r"(v[9]), "=r"(v[10]), "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]),
          "=r"(v[16]), "=r"(v[17]), "=r"(v[18]), "=r"(v[19]), "=r"(v[20]), "=r"(v[21]), "=r"(v[22]), "=r"(v[23]),
          "=r"(v[24]), "=r"(v[25]), "=r"(v[26]), "=r"(v[27]), "=r"(v[28]), "=r"(v[29]), "=r"(v[30]), "=r"(v[31])
        : "r"(addr));
}
__device__ __forceinline__ void tmem_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

// The same, written; wait before the tensor cores are told of it.
__device__ __forceinline__ void tmem_store32(uint32_t addr, const uint32_t (&v)[32]) {
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,"
        "%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
        ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
          "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
          "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]), "r"(addr)
        : "memory");
}
__device__ __forceinline__ void tmem_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// ---- operands in shared memory

constexpr uint64_t kDescVersion = uint64_t(1) << 46;
// Rows of 128 bytes along the inner dimension, 128-byte swizzle: groups of 8 rows are 1024 bytes
// apart.  The inner dimension advances by adding bytes / 16 to the descriptor.
__device__ __forceinline__ uint64_t desc_rows128(uint32_t addr) {
    return ((addr & 0x3ffffu) >> 4) | (uint64_t(1) << 16) | (uint64_t(1024 >> 4) << 32) | kDescVersion | (uint64_t(2) << 61);
}
// A 512-byte tile of scales, 32 rows of 16 bytes without swizzle: groups of 8 rows are 128 bytes apart.
__device__ __forceinline__ uint64_t desc_scales(uint32_t addr) {
    return ((addr & 0x3ffffu) >> 4) | (uint64_t(128 >> 4) << 16) | (uint64_t(128 >> 4) << 32) | kDescVersion;
}

// ---- instructions

// A tile of scales (32 rows x 16 bytes) -> four columns of tensor memory, the same for each
// quarter of the lanes.  PAIR: in both blocks, each from its own shared memory.
template <bool PAIR = false>
__device__ __forceinline__ void tmem_copy_scales(uint32_t dst, uint64_t desc) {
    if constexpr (PAIR) asm volatile("tcgen05.cp.cta_group::2.32x128b.warpx4 [%0], %1;" ::"r"(dst), "l"(desc) : "memory");
    else asm volatile("tcgen05.cp.cta_group::1.32x128b.warpx4 [%0], %1;" ::"r"(dst), "l"(desc) : "memory");
}

// D [128 x n] (+)= A [128 x 16] B [n x 16]^T of 16-bit floats, binary32 sums.
__device__ __forceinline__ uint32_t f16_instruction(int n, bool bf16) {
    return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (static_cast<uint32_t>(n >> 3) << 17) | (8u << 24);
}
// A in tensor memory: a lane a row, 8 columns of two elements each.
__device__ __forceinline__ void mma_16bit(uint32_t d, uint32_t a, uint64_t b, uint32_t instruction, bool accumulate) {
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
                 "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(instruction), "r"(accumulate ? 1u : 0u) : "memory");
}

// D [128 x n] (+)= A [128 x 64] B [n x 64]^T of 4-bit floats with a scale for every 32.
// `half`: which two of a tile's four blocks the 64 columns are.  PAIR: 256 rows of A, half of them
// and half of B's rows in each block; every block has the scales of its rows of A and of all of B.
template <bool PAIR = false>
__device__ __forceinline__ uint32_t mxf4_instruction(int n, int half) {
    const uint32_t id = half ? 2u : 0u;
    return (id << 4) | (1u << 7) | (1u << 10) | (static_cast<uint32_t>(n >> 3) << 17) | (1u << 23) | ((PAIR ? 16u : 8u) << 24) | (id << 29);
}
template <bool PAIR = false>
__device__ __forceinline__ void mma_mxf4(uint32_t d, uint64_t a, uint64_t b, uint32_t instruction, uint32_t scale_a,
                                         uint32_t scale_b, bool accumulate) {
    if constexpr (PAIR)
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::2.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(instruction), "r"(scale_a), "r"(scale_b), "r"(accumulate ? 1u : 0u) : "memory");
    else
        asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %6, 0;\n\t"
                     "tcgen05.mma.cta_group::1.kind::mxf4.block_scale.scale_vec::2X [%0], %1, %2, %3, [%4], [%5], p;\n\t}"
                     ::"r"(d), "l"(a), "l"(b), "r"(instruction), "r"(scale_a), "r"(scale_b), "r"(accumulate ? 1u : 0u) : "memory");
}

}  // namespace sp
