// 8-bit key/value cache: what its kernels share.  A value is an e4m3 code times a power-of-two
// scale that the block_tokens x head_dim codes of a (block, head) have in common.
#pragma once

#include <cuda.h>

#include "sp_device.cuh"
#include "sp_internal.h"

namespace sp {

constexpr int kMinCacheExponent = -126;

// The least e >= -126 with amax <= 448 * 2^e = 1.75 * 2^(e + 8), from the bits of amax >= 0.
__device__ __forceinline__ int cache_exponent(uint32_t amax_bits) {
    const int e = static_cast<int>(amax_bits >> 23) - 127 - 8 + ((amax_bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return max(e, kMinCacheExponent);
}
// 2^e; 0 below binary32's normal range (codes brought down that far are 0).
__device__ __forceinline__ float pow2(int e) {
    return e < -126 ? 0.0f : __uint_as_float(static_cast<uint32_t>(e + 127) << 23);
}
__device__ __forceinline__ int exponent_of(float scale) {
    return static_cast<int>((__float_as_uint(scale) >> 23) & 0xffu) - 127;
}

// Two e4m3 codes (low half of h) -> two packed binary16 values (exact).
__device__ __forceinline__ void e4m3_to_f16(uint32_t w, uint32_t &lo, uint32_t &hi) {
    asm("{\n\t.reg .b16 a, b;\n\t"
        "mov.b32 {a, b}, %2;\n\t"
        "cvt.rn.f16x2.e4m3x2 %0, a;\n\t"
        "cvt.rn.f16x2.e4m3x2 %1, b;\n\t}"
        : "=r"(lo), "=r"(hi) : "r"(w));
}
__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
    const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
// Two packed binary16 values -> bf16 (exact for what e4m3 holds).
__device__ __forceinline__ uint32_t f16_to_bf16(uint32_t h) {
    const float2 f = unpack2<false>(h);
    return pack_bf16(f.x, f.y);
}
constexpr uint32_t kLargeQuery = 0x5f800000u;  // 2^64: larger bf16 queries are scaled down by that
__device__ __forceinline__ void e4m3_unpack8(uint2 w, float (&v)[8]) {
    uint32_t h[4];
    e4m3_to_f16(w.x, h[0], h[1]);
    e4m3_to_f16(w.y, h[2], h[3]);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const float2 f = unpack2<false>(h[i]);
        v[2 * i] = f.x;
        v[2 * i + 1] = f.y;
    }
}
// Eight binary32 values, at most 448 in magnitude -> codes; NaN stays NaN.
__device__ __forceinline__ uint2 e4m3_pack8_finite(const float (&v)[8]) {
    uint2 w;
    asm("{\n\t.reg .b16 a, b, c, d;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 a, %3, %2;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 b, %5, %4;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 c, %7, %6;\n\t"
        "cvt.rn.satfinite.e4m3x2.f32 d, %9, %8;\n\t"
        "mov.b32 %0, {a, b};\n\t"
        "mov.b32 %1, {c, d};\n\t}"
        : "=r"(w.x), "=r"(w.y)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return w;
}
// The same where infinities may occur: they are stored as NaN.
__device__ __forceinline__ uint2 e4m3_pack8(const float (&v)[8]) {
    float u[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) u[i] = isfinite(v[i]) ? v[i] : __uint_as_float(0x7fc00000u);
    return e4m3_pack8_finite(u);
}
// Largest finite magnitude, as bits.
__device__ __forceinline__ uint32_t finite_amax8(const float (&v)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const uint32_t bits = __float_as_uint(v[i]) & 0x7fffffffu;
        if (bits < 0x7f800000u) m = max(m, bits);
    }
    return m;
}

// Block that holds the tokens from place * block_tokens of a sequence; -1 if the table names none.
__device__ __forceinline__ int64_t cache_block(const sp_cache &c, int64_t seq, int64_t place) {
    if (place >= c.table_cols) return -1;
    const int64_t id = c.table[seq * c.ld_table + place];
    return id >= 0 && id < c.n_blocks ? id : -1;
}

// Groups of sequences that share the first blocks of their first row.
struct SharedGroups {
    const int32_t *start, *prefix;  // [n_groups + 1], [n_groups]
    int64_t n_groups, max_prefix, max_group;
};
// Sequences [begin, end) of a group share the first `blocks` blocks of row begin.
struct SharedGroup {
    int64_t begin, end, blocks;
};
__device__ __forceinline__ SharedGroup shared_group(const SharedGroups &g, const sp_cache &c, int64_t i) {
    SharedGroup r;
    r.begin = max(g.start[i], 0);
    r.end = min(min(int64_t(g.start[i + 1]), r.begin + g.max_group), c.n_seqs);
    r.blocks = min(max(int64_t(0), min(int64_t(g.prefix[i]), g.max_prefix)) / c.block_tokens, c.table_cols);
    return r;
}
// Blocks that a sequence shares, 0 if it is in no group; the whole warp asks.  The last group that
// does not begin behind the sequence is found 32 candidates at a time.
__device__ __forceinline__ int64_t shared_blocks(const SharedGroups &g, const sp_cache &c, int64_t seq) {
    const int lane = threadIdx.x & 31;
    int64_t at = 0, n = g.n_groups;
    while (n > 0) {
        const int64_t stride = (n + 31) / 32, i = at + lane * stride;
        const unsigned vote = __ballot_sync(kFullWarp, lane * stride < n && g.start[i] <= seq);
        if (vote == 0u) return 0;
        const int64_t skip = (31 - __clz(vote)) * stride;
        at += skip;
        if (stride == 1) break;
        n = min(stride, n - skip);
    }
    if (n == 0) return 0;
    const SharedGroup r = shared_group(g, c, at);
    return seq >= r.begin && seq < r.end ? r.blocks : 0;
}

// What the two kernels over prefix and tails leave for the one that joins them: for a sequence and kv
// head `splits` parts, those of the prefix first.
struct SharedParts {
    float *o;    // [seq, kv head, part, row, D]: of the prefix divided by its sum, of the tails not
    float2 *ml;  // [seq, kv head, part, row]: maximum (log2) and sum
    int splits, prefix_splits;
};

// cache_attention.cu: the tokens behind the prefixes, and the join.
int shared_tail_splits(const sp_cache &c, int64_t rows, int64_t tail);
sp_status launch_cache_tails(const sp_cache &c, const SharedAttention &s, const SharedParts &parts, const CUtensorMap &k_map,
                             const CUtensorMap &v_map, cudaStream_t stream);

}  // namespace sp
