// Asynchronous copies into shared memory (TMA) and the barriers they complete on.
//
// Every wait is bounded: a wait that runs out marks the block as failed, after which its other
// waits give up at once, the block drains the copies it has in flight and returns; the host
// reads the mark with sp_wait_status.  Nothing traps or spins for ever.
#pragma once

#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "sp_device.cuh"
#include "sp_internal.h"

namespace sp {

constexpr uint32_t kWaitLimit = 1u << 22;  // tries of one wait: seconds, against microseconds

static __device__ unsigned int g_expired_waits;

static cudaError_t read_expired_waits(unsigned int *out, bool clear) {
    cudaError_t e = cudaMemcpyFromSymbol(out, g_expired_waits, sizeof(unsigned int));
    if (e == cudaSuccess && clear) {
        const unsigned int zero = 0;
        e = cudaMemcpyToSymbol(g_expired_waits, &zero, sizeof zero);
    }
    return e;
}
namespace {
struct WaitRegistration {
    WaitRegistration() { register_wait_reader(read_expired_waits); }
};
const WaitRegistration g_wait_registration;
}  // namespace

__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar, uint32_t count) {
    asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0u;
}
// The same at once, without waiting a while.
__device__ __forceinline__ bool mbar_test(uint32_t bar, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n\t.reg .pred p;\n\t"
                 "mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
                 "selp.u32 %0, 1, 0, p;\n\t}"
                 : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
    return ok != 0u;
}
// A wait has run out: the block gives up.
__device__ __forceinline__ void mbar_give_up(volatile uint32_t *failed) {
    *failed = 1u;
    atomicAdd(&g_expired_waits, 1u);
}
// True once the phase of the given parity has completed; false if the wait ran out or another
// thread of the block has given up.
__device__ __forceinline__ bool mbar_wait_or_fail(uint32_t bar, uint32_t parity, volatile uint32_t *failed) {
    if (mbar_try(bar, parity)) return true;
    for (uint32_t i = 0; i < kWaitLimit; ++i) {
        if (mbar_try(bar, parity)) return true;
        if (*failed != 0u) return false;
    }
    mbar_give_up(failed);
    return false;
}

// Both phases: their first looks at the barriers overlap.
__device__ __forceinline__ bool mbar_wait2_or_fail(uint32_t bar, uint32_t parity, uint32_t other, uint32_t other_parity,
                                                   volatile uint32_t *failed) {
    const bool one = mbar_test(bar, parity), two = mbar_test(other, other_parity);
    return (one || mbar_wait_or_fail(bar, parity, failed)) && (two || mbar_wait_or_fail(other, other_parity, failed));
}

__device__ __forceinline__ bool mbar_wait3_or_fail(uint32_t a, uint32_t a_parity, uint32_t b, uint32_t b_parity, uint32_t c,
                                                   uint32_t c_parity, volatile uint32_t *failed) {
    const bool one = mbar_test(a, a_parity), two = mbar_test(b, b_parity), three = mbar_test(c, c_parity);
    return (one || mbar_wait_or_fail(a, a_parity, failed)) && (two || mbar_wait_or_fail(b, b_parity, failed)) &&
           (three || mbar_wait_or_fail(c, c_parity, failed));
}

// Asynchronous copies and the tensor cores are driven by one thread, but the warp walks the loop
// together and elects it only for the instructions themselves: operands then stay in uniform
// registers.  Driven from a branch on the lane index, a stage of products took 1400 cycles of one
// thread's latencies against 512 of products (128 x 256 x 256 columns in 4 bits).
__device__ __forceinline__ bool elect_one() {
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0u;
}
// The warp's index, known to the compiler to be the same in all lanes.
__device__ __forceinline__ int uniform_warp() { return __shfl_sync(kFullWarp, static_cast<int>(threadIdx.x >> 5), 0); }

// Place in a ring of stages: the slot, and the parity of the barrier phase that its current use completes.
template <int SLOTS>
struct RingPlace {
    int slot = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next() {
        if (++slot == SLOTS) {
            slot = 0;
            parity ^= 1u;
        }
    }
};

__device__ __forceinline__ void tma_prefetch_map(const CUtensorMap *map) {
    asm volatile("prefetch.tensormap [%0];" ::"l"(map) : "memory");
}
// Box of a 2-D tensor at (x, y) -> shared memory.  x * element size is a multiple of 16 bytes.
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

// The same for data that will not be read again soon: the L2 gives its lines up first.
__device__ __forceinline__ uint64_t l2_evict_first() {
    uint64_t policy;
    asm volatile("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    return policy;
}
__device__ __forceinline__ void tma_load_2d(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar, uint64_t policy) {
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes.L2::cache_hint "
                 "[%0], [%1, {%2, %3}], [%4], %5;" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "l"(policy) : "memory");
}
// Pairs of blocks: the barrier may be the other block's (its address in the cluster's window).
__device__ __forceinline__ void tma_load_2d_pair(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar) {
    asm volatile("cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes "
                 "[%0], [%1, {%2, %3}], [%4];" ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}
__device__ __forceinline__ void mbar_expect_tx_cluster(uint32_t bar, uint32_t bytes) {
    asm volatile("mbarrier.arrive.expect_tx.relaxed.cluster.shared::cluster.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive_cluster(uint32_t bar) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(bar) : "memory");
}
// Shared memory written by ordinary stores becomes visible to the asynchronous copies.
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
// Shared memory -> box of a 2-D tensor at (x, y), both inside it; what lies outside is not written.
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t src, int x, int y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.bulk_group [%0, {%1, %2}], [%3];" ::"l"(map), "r"(x), "r"(y),
                 "r"(src) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
// Until the stores this thread issued have read their shared memory / have completed.
__device__ __forceinline__ void tma_store_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void tma_store_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

// Describes a row-major matrix of `rows` rows of `row_bytes` bytes (pitch a multiple of 16) as
// boxes of 128 bytes x `box_rows`, laid into shared memory with the 128-byte swizzle (the
// 16-byte chunk c of row r lands at chunk c ^ (r & 7)); what lies outside reads as zero.
// Elements are bytes.  api_serve.cu holds the driver entry point.
cudaError_t encode_byte_tiles(CUtensorMap *map, const void *base, int64_t rows, int64_t row_bytes,
                              int64_t pitch, int box_rows);
// The same for rows of 64 or 128 bytes that follow one another, as whole rows (swizzled over 64 or
// 128 bytes: with 64, chunk c of row r lands at c ^ (r / 2 & 3)).
cudaError_t encode_byte_rows(CUtensorMap *map, const void *base, int64_t rows, int row_bytes, int box_rows);
// Rows of 512 bytes that follow one another (tiles of scale bytes), unswizzled: boxes of box_rows rows.
cudaError_t encode_scale_tiles(CUtensorMap *map, const void *base, int64_t rows, int box_rows);
// As encode_byte_tiles for 16-bit elements (an inner extent that is not a multiple of 16 bytes is clipped
// exactly): boxes of 64 elements x box_rows.
cudaError_t encode_half_tiles(CUtensorMap *map, const void *base, int64_t rows, int64_t cols, int64_t ld,
                              int box_rows);

}  // namespace sp
