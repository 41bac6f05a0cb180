// Microscaled 4-bit weights: layout, and what the kernels that quantise and multiply them share.
//
// A value is code * 2^(byte - 127): a 4-bit float code (sign, two exponent bits, one mantissa
// bit: 0, .5, 1, 1.5, 2, 3, 4, 6) and one scale byte for 32 consecutive columns of a row (byte
// 255: every value of the block is NaN).  Codes lie row-major, the even column in the low half
// of a byte; scale bytes lie in tiles of 128 rows x 4 blocks, which is the order in which the
// tensor cores take them.
#pragma once

#include "sp_device.cuh"
#include "sp_internal.h"

namespace sp {

constexpr int kMx4Block = 32;          // columns that share a scale
constexpr int kMx4TileRows = 128;      // rows of a tile of scale bytes
constexpr int kMx4TileBytes = 512;     // 128 rows x 4 blocks

__host__ __device__ inline int64_t mx4_blocks(int64_t n_cols) { return (n_cols + 31) / 32; }
__host__ __device__ inline int64_t mx4_tile_cols(int64_t n_cols) { return (n_cols + 127) / 128; }
__host__ __device__ inline int64_t mx4_tile_rows(int64_t n_rows) { return (n_rows + 127) / 128; }

// Whether `tiles` clusters of `slices` blocks, an SM each, run in one round.  Clusters lie within a
// group of SMs (16 to 18 of them here), so that 8 blocks leave room unused: 16 clusters of 8 took
// two rounds.
inline bool cluster_slices_fit(int64_t tiles, int slices, int sms) {
    return tiles * slices <= (slices > 4 ? 64 : sms);
}

// Scale byte of a block whose largest magnitude is `amax` (the bits of a non-negative binary32
// number): the exponent of amax less 2, the exponent of the largest code, so that amax / scale
// lies in [4, 8); at least 0 (the smallest scale), 255 for a block that is not finite.
__device__ __forceinline__ uint32_t mx4_scale_byte(uint32_t amax_bits) {
    const uint32_t e = amax_bits >> 23;
    return e == 255u ? 255u : (e > 2u ? e - 2u : 0u);
}

// 2^(127 - byte), the factor that brings a block to the grid of the code; 0 for byte 255, which
// leaves zero codes (NaN * 0 and inf * 0 are caught by the caller).  Always a normal number.
__device__ __forceinline__ float mx4_inverse_scale(uint32_t byte) {
    return __uint_as_float((254u - byte) << 23);
}

// 2^(byte - 127) as binary32: the smallest is subnormal, byte 255 gives inf (0 * inf = NaN).
__device__ __forceinline__ float mx4_scale(uint32_t byte) {
    return __uint_as_float(max(byte << 23, 0x00400000u));
}

// Two 4-bit codes of a byte -> two packed binary16 values (exact).
__device__ __forceinline__ void mx4_unpack8(uint32_t w, uint32_t (&h)[4]) {
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "mov.b32 {b0, b1, b2, b3}, %4;\n\t"
        "cvt.rn.f16x2.e2m1x2 %0, b0;\n\t"
        "cvt.rn.f16x2.e2m1x2 %1, b1;\n\t"
        "cvt.rn.f16x2.e2m1x2 %2, b2;\n\t"
        "cvt.rn.f16x2.e2m1x2 %3, b3;\n\t}"
        : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3])
        : "r"(w));
}

// Eight binary32 values already divided by the scale -> eight codes: nearest, ties to the even
// code, magnitudes above 6 become 6.
__device__ __forceinline__ uint32_t mx4_pack8(const float (&v)[8]) {
    uint32_t w;
    asm("{\n\t.reg .b8 b0, b1, b2, b3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5;\n\t"
        "cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7;\n\t"
        "mov.b32 %0, {b0, b1, b2, b3};\n\t}"
        : "=r"(w)
        : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
    return w;
}

// Largest magnitude of eight packed 16-bit floats, as the bits of a binary32 number.  The bit
// patterns of magnitudes order like the magnitudes in both types, NaN above infinity.
template <bool BF16>
__device__ __forceinline__ uint32_t amax8_bits(const uint32_t (&p)[4]) {
    uint32_t m = __vmaxu2(__vmaxu2(p[0] & 0x7fff7fffu, p[1] & 0x7fff7fffu),
                          __vmaxu2(p[2] & 0x7fff7fffu, p[3] & 0x7fff7fffu));
    m = max(m & 0xffffu, m >> 16);
    const float2 f = unpack2<BF16>(m);
    return __float_as_uint(f.x) & 0x7fffffffu;
}

// Quantises the eight elements a lane holds of a block that four neighbouring lanes share;
// returns the scale byte, leaves the codes in `codes`.
template <bool BF16>
__device__ __forceinline__ uint32_t mx4_quantize_quad(const uint32_t (&p)[4], uint32_t &codes) {
    uint32_t a = amax8_bits<BF16>(p);
    a = max(a, __shfl_xor_sync(kFullWarp, a, 1));
    a = max(a, __shfl_xor_sync(kFullWarp, a, 2));
    const uint32_t byte = mx4_scale_byte(a);
    const float inv = mx4_inverse_scale(min(byte, 254u));
    float v[8];
    if constexpr (BF16) {
        // one mixed-precision multiply-add an element (the factor is a power of two that bf16 has);
        // adding -0 keeps the sign of a zero
        const unsigned short f = static_cast<unsigned short>(__float_as_uint(inv) >> 16);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unsigned short lo, hi;
            asm("mov.b32 {%0, %1}, %2;" : "=h"(lo), "=h"(hi) : "r"(p[i]));
            asm("fma.rn.f32.bf16 %0, %1, %2, %3;" : "=f"(v[2 * i]) : "h"(lo), "h"(f), "f"(-0.0f));
            asm("fma.rn.f32.bf16 %0, %1, %2, %3;" : "=f"(v[2 * i + 1]) : "h"(hi), "h"(f), "f"(-0.0f));
        }
    } else {
        unpack8<BF16>(p, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] *= inv;
    }
    codes = byte == 255u ? 0u : mx4_pack8(v);
    return byte;
}

}  // namespace sp
