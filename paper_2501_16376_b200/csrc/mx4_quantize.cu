// Microscaled 4-bit quantisation of a 16-bit matrix and the way back.
//
// Mathematics: in every block of 32 columns  e = floor(log2 max|w|) - 2,  code = nearest 4-bit
// float to w / 2^e.  One pass over the matrix; bound by memory: 2 bytes read and 17/32 written
// per weight (the reverse for the way back).  A warp takes four rows that lie 32 apart and 256
// columns of each: a quad of lanes holds a block (16 bytes a lane, four loads in flight), the
// largest magnitude costs two shuffles, and the scale bytes of the four rows are 16 consecutive
// bytes of a tile, so they leave in one store.  Measured: 14336 x 4096 in bf16 there and back 45.8 us
// (5.8 TB/s).
#include "mx4_common.cuh"

namespace sp {

template <bool BF16, bool VEC, bool MASK>
__global__ void __launch_bounds__(256)
mx4_quantize_kernel(const uint16_t *__restrict__ W, int64_t n_rows, int64_t n_cols, int64_t ldw,
                    const uint32_t *__restrict__ mask, uint8_t *__restrict__ codes, int64_t ldc,
                    uint8_t *__restrict__ scales, int row_groups) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t col = int64_t(blockIdx.x) * 256 + lane * 8;
    const int kt = static_cast<int>(mx4_tile_cols(n_cols)), at = static_cast<int>(blockIdx.x) * 2 + (lane >> 4);
    const bool has_codes = col < mx4_blocks(n_cols) * 32;
    pdl_launch_dependents();
    pdl_wait();
    for (int group = blockIdx.y; group < row_groups; group += gridDim.y) {
        // this warp's rows: row0, row0 + 32, + 64, + 96 of a tile of 128
        const int in_tile = (group & 3) * 8 + warp;
        const int64_t row0 = int64_t(group >> 2) * kMx4TileRows + in_tile;
        const int here = static_cast<int>(min(int64_t(4), (n_rows - row0 + 31) / 32));  // of its four rows
        const uint16_t *w = W + row0 * ldw;
        uint8_t *c = codes + row0 * ldc + (col >> 1);
        uint32_t p[4][4], keep[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (i < here) {
                load8<VEC, true>(w, col, n_cols, p[i]);
                w += 32 * ldw;
                if constexpr (MASK)
                    keep[i] = col < n_cols ? mask[(row0 + 32 * i) * ((n_cols + 31) / 32) + (col >> 5)] >> (col & 31) : 0u;
            } else {
                p[i][0] = p[i][1] = p[i][2] = p[i][3] = 0u;
                keep[i] = 0u;
            }
        }
        uint32_t tile[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if constexpr (MASK) zero_pruned(p[i], keep[i]);
            uint32_t word;
            const uint32_t byte = mx4_quantize_quad<BF16>(p[i], word);
            if (i < here && has_codes) *reinterpret_cast<uint32_t *>(c) = word;
            c += 32 * ldc;
            uint32_t t = byte << (8 * ((lane >> 2) & 3));
            t |= __shfl_xor_sync(kFullWarp, t, 4);
            t |= __shfl_xor_sync(kFullWarp, t, 8);
            tile[i] = t;
        }
        if ((lane & 15) == 0 && at < kt)
            *reinterpret_cast<uint4 *>(scales + (int64_t(group >> 2) * kt + at) * kMx4TileBytes + in_tile * 16) =
                make_uint4(tile[0], tile[1], tile[2], tile[3]);
    }
}

template <bool BF16, bool VEC>
__global__ void __launch_bounds__(256)
mx4_dequantize_kernel(const uint8_t *__restrict__ codes, int64_t ldc,
                      const uint8_t *__restrict__ scales, int64_t n_rows, int64_t n_cols,
                      uint16_t *__restrict__ W, int64_t ldw, int row_groups) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t col = int64_t(blockIdx.x) * 256 + lane * 8;
    const int64_t kt = mx4_tile_cols(n_cols);
    pdl_launch_dependents();
    if (col >= n_cols) return;
    pdl_wait();
    for (int group = blockIdx.y; group < row_groups; group += gridDim.y) {
        const int in_tile = (group & 3) * 8 + warp;
        const int64_t row0 = int64_t(group >> 2) * kMx4TileRows + in_tile;
        const uint4 tile = *reinterpret_cast<const uint4 *>(
            scales + (int64_t(group >> 2) * kt + blockIdx.x * 2 + (lane >> 4)) * kMx4TileBytes + in_tile * 16);
        const uint32_t words[4] = {tile.x, tile.y, tile.z, tile.w};
        const uint8_t *c = codes + row0 * ldc + (col >> 1);
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i)
            w[i] = row0 + 32 * i < n_rows ? __ldcs(reinterpret_cast<const uint32_t *>(c + 32 * i * ldc)) : 0u;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (row0 + 32 * i >= n_rows) break;
            const uint32_t byte = (words[i] >> (8 * ((lane >> 2) & 3))) & 0xffu;
            const float s = byte == 255u ? __uint_as_float(0x7fc00000u) : mx4_scale(byte);
            uint32_t h[4], out[4];
            mx4_unpack8(w[i], h);
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                const float2 f = unpack2<false>(h[k]);
                if constexpr (BF16) {
                    __nv_bfloat162 v = __floats2bfloat162_rn(f.x * s, f.y * s);
                    out[k] = *reinterpret_cast<uint32_t *>(&v);
                } else {
                    __half2 v = __floats2half2_rn(f.x * s, f.y * s);
                    out[k] = *reinterpret_cast<uint32_t *>(&v);
                }
            }
            store8<VEC>(W + (row0 + 32 * i) * ldw, col, n_cols, out);
        }
    }
}

// A block's eight warps take neighbouring rows of one 256-column chunk.
static dim3 quantize_grid(int64_t n_rows, int64_t n_cols, int &row_groups) {
    row_groups = static_cast<int>(mx4_tile_rows(n_rows) * 4);
    return dim3(static_cast<unsigned>((n_cols + 255) / 256), static_cast<unsigned>(row_groups < 65535 ? row_groups : 65535));
}

sp_status launch_mx4_quantize(const void *W, sp_dtype dtype, int64_t n_rows, int64_t n_cols,
                              int64_t ldw, const uint32_t *mask, uint8_t *codes, int64_t ldc,
                              uint8_t *scales, cudaStream_t stream) {
    const uint16_t *Wp = static_cast<const uint16_t *>(W);
    const bool vec = aligned16(W) && ldw % 8 == 0 && n_cols % 8 == 0;
    int row_groups;
    PdlConfig pdl(quantize_grid(n_rows, n_cols, row_groups), dim3(256), stream);
    cudaError_t e;
#define SP_LAUNCH(B, V)                                                                          \
    e = mask != nullptr ? cudaLaunchKernelEx(&pdl.cfg, mx4_quantize_kernel<B, V, true>, Wp,       \
                                             n_rows, n_cols, ldw, mask, codes, ldc, scales,       \
                                             row_groups)                                         \
                        : cudaLaunchKernelEx(&pdl.cfg, mx4_quantize_kernel<B, V, false>, Wp,      \
                                             n_rows, n_cols, ldw, mask, codes, ldc, scales,       \
                                             row_groups)
    if (dtype == SP_BF16) { if (vec) SP_LAUNCH(true, true); else SP_LAUNCH(true, false); }
    else { if (vec) SP_LAUNCH(false, true); else SP_LAUNCH(false, false); }
#undef SP_LAUNCH
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

sp_status launch_mx4_dequantize(const uint8_t *codes, int64_t ldc, const uint8_t *scales,
                                int64_t n_rows, int64_t n_cols, sp_dtype dtype, void *W,
                                int64_t ldw, cudaStream_t stream) {
    uint16_t *Wp = static_cast<uint16_t *>(W);
    const bool vec = aligned16(W) && ldw % 8 == 0 && n_cols % 8 == 0;
    int row_groups;
    PdlConfig pdl(quantize_grid(n_rows, n_cols, row_groups), dim3(256), stream);
    cudaError_t e;
#define SP_LAUNCH(B, V)                                                                          \
    e = cudaLaunchKernelEx(&pdl.cfg, mx4_dequantize_kernel<B, V>, codes, ldc, scales, n_rows,     \
                           n_cols, Wp, ldw, row_groups)
    if (dtype == SP_BF16) { if (vec) SP_LAUNCH(true, true); else SP_LAUNCH(true, false); }
    else { if (vec) SP_LAUNCH(false, true); else SP_LAUNCH(false, false); }
#undef SP_LAUNCH
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

}  // namespace sp
