// 8-bit key/value cache: what its kernels share.  A value is an e4m3 code times a power-of-two
// scale that the block_tokens x head_dim codes of a (block, head) have in common.
#pragma once

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

}  // namespace sp
