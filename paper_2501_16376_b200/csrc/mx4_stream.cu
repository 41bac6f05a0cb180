// Product of a few tokens with a microscaled 4-bit matrix (a decoding step): the weights stream
// by once, everything else hides behind them.
//
// Mathematics: y[t, r] = sum over blocks b of  2^(byte - 127)[r, b] * sum_{k in b} code[r, k] x[t, k].
// The codes are exact in binary16, so a block's inner sum is two m16n8k16 tensor-core products on
// the bare codes, accumulated in binary32, and the scale - a power of two - is applied to that
// sum by one multiply-add per output instead of to every weight.
//
// Bound by memory: 17/32 byte per weight.  A block of threads owns 128 rows and a slice of the
// columns; a producer thread keeps kStages x (128 rows x 512 columns) in flight by TMA; 16 warps (4
// groups of 32 rows x 4 quarters of a stage's columns) convert and multiply.  (With stages of 256
// columns a warp's overhead for a stage was a third of its instructions, and issuing them is what
// the kernel waits for besides memory.)  The column order inside a 32-column block is free as long
// as weights and activations agree on it: a lane takes 8 consecutive columns, so a weight operand
// is one 4-byte word of codes (four conversions) and an activation operand is one 16-byte load.
// With few rows the columns are cut over a cluster of up to 8 blocks whose partial sums meet
// through distributed shared memory, in rank order (results do not depend on scheduling).
// Measured: 1 token x 4096 x 4096 5.6 us, x 4096 x 14336 10.4 us (3.0 TB/s: 112 blocks of one wave,
// each 8 stages and some 3 us of start and end); 8 tokens 6.9 and 14.4 us, with 4-bit activations 7.2
// and 15.5.
//
// bf16 activations become binary16 here: every (token, 256 columns) is scaled by a power of two
// so that its largest magnitude lies in [2^14, 2^15).  What binary16 cannot hold - an element
// more than 2^30 times smaller than the largest of its 256 - goes into a second pass over the
// weights, with the remainders scaled by 2^40; a block takes that pass only if it has one.
#include "mx4_common.cuh"
#include "sp_tma.cuh"

namespace sp {

namespace {

constexpr int kStages = 3;
constexpr int kStageTiles = 4;                    // scale tiles of a stage: 512 columns
constexpr int kBoxBytes = kMx4TileRows * 128;    // codes of 128 rows x 256 columns
constexpr int kCodeBytes = 2 * kBoxBytes;
constexpr int kWarps = 16;                        // 4 groups of 32 rows x 4 scale tiles of columns
constexpr int kTokens = 8;                        // columns of an mma
constexpr int kPartPitch = 132;                 // floats between columns of a block's partial sums

struct StreamArgs {
    const uint16_t *X;
    int64_t ldx, n_tokens, n_cols, n_rows;
    const uint8_t *scales;
    uint16_t *Y;
    int64_t ldy;
    int tile_cols;     // scale tiles along a row
    int stages;        // 512-column stages of a row
    int slices;        // blocks of a cluster that share the rows
    int chunk_stages;  // stages whose activations are in shared memory at a time
    int quantize_x;
    int vec_x;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t lds32(uint32_t addr) {
    uint32_t v;
    asm volatile("ld.shared.u32 %0, [%1];" : "=r"(v) : "r"(addr));
    return v;
}
__device__ __forceinline__ uint4 lds128(uint32_t addr) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr));
    return v;
}
__device__ __forceinline__ void consumer_sync() { asm volatile("bar.sync 1, %0;" ::"n"(kWarps * 32) : "memory"); }

// One (token, 256 columns) of the activations -> binary16 in shared memory and its scale;
// returns whether a remainder is left (bf16).  pass 1 stores the remainders.
template <bool BF16>
__device__ __forceinline__ bool convert_x(const StreamArgs &a, const uint32_t (&p)[4], int lane, int pass,
                                          __half *dst, float *scale_out) {
    float v[8];
    if (a.quantize_x) {
        uint32_t word, h[4];
        const uint32_t byte = mx4_quantize_quad<BF16>(p, word);
        const float s = byte == 255u ? __uint_as_float(0x7fc00000u) : mx4_scale(byte);
        mx4_unpack8(word, h);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float2 f = unpack2<false>(h[i]);
            v[2 * i] = f.x * s;
            v[2 * i + 1] = f.y * s;
        }
    } else {
        unpack8<BF16>(p, v);
    }
    float inverse = 1.0f;
    bool rest = false;
    if constexpr (BF16) {
        uint32_t m = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t bits = __float_as_uint(v[i]) & 0x7fffffffu;
            if (bits < 0x7f800000u) m = max(m, bits);
        }
        m = __reduce_max_sync(kFullWarp, m);
        const int e = static_cast<int>(m >> 23);               // exponent of the largest + 127
        const int up = min(141 - max(e, 1), 126);
        const float f = __uint_as_float(static_cast<uint32_t>(up + 127) << 23);
        inverse = __uint_as_float(static_cast<uint32_t>(127 - up) << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float x = v[i] * f;
            const float hi = __half2float(__float2half_rn(x));
            const float r = fabsf(x) <= 65504.0f ? x - hi : 0.0f;  // 0 for what is not finite
            rest |= r != 0.0f;
            v[i] = pass == 0 ? x : r * 1099511627776.0f;           // 2^40
        }
        if (pass != 0) inverse *= 9.094947017729282e-13f;          // 2^-40
    }
    uint32_t out[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __half2 h = __floats2half2_rn(v[2 * i], v[2 * i + 1]);
        out[i] = *reinterpret_cast<uint32_t *>(&h);
    }
    *reinterpret_cast<uint4 *>(dst + lane * 8) = make_uint4(out[0], out[1], out[2], out[3]);
    if (lane == 0) *scale_out = inverse;
    return rest;
}

}  // namespace

template <bool BF16>
__global__ void __launch_bounds__(kWarps * 32 + 32)
mx4_stream_kernel(const __grid_constant__ CUtensorMap codes_map, const StreamArgs a) {
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ uint64_t full[kStages], empty[kStages];
    __shared__ uint32_t failed, has_rest;
    uint8_t *const code_smem = smem;
    uint8_t *const scale_smem = smem + kStages * kCodeBytes;
    const int x_pitch = a.chunk_stages * 1024 + 64;              // bytes; 64 mod 128: no conflicts
    uint8_t *const x_smem = scale_smem + kStages * kStageTiles * kMx4TileBytes;
    float *const xs_smem = reinterpret_cast<float *>(x_smem + kTokens * x_pitch);
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const int slices = a.slices, slice = blockIdx.x % slices, row_tile = blockIdx.x / slices;
    const int64_t row0 = int64_t(row_tile) * kMx4TileRows;
    const int first = static_cast<int>(int64_t(a.stages) * slice / slices);
    const int last = static_cast<int>(int64_t(a.stages) * (slice + 1) / slices);

    if (threadIdx.x == 0) {
        tma_prefetch_map(&codes_map);
        for (int s = 0; s < kStages; ++s) {
            mbar_init(smem_addr(&full[s]), 1);
            mbar_init(smem_addr(&empty[s]), kWarps);
        }
        failed = has_rest = 0u;
        mbar_fence_init();
    }
    // tokens that do not exist: zeros
    for (int at = static_cast<int>(a.n_tokens) * x_pitch + threadIdx.x * 16; at < kTokens * x_pitch; at += (kWarps * 32 + 32) * 16)
        *reinterpret_cast<uint4 *>(x_smem + at) = make_uint4(0u, 0u, 0u, 0u);
    for (int at = threadIdx.x; at < a.chunk_stages * 2 * kTokens; at += kWarps * 32 + 32)
        if (at % kTokens >= a.n_tokens) xs_smem[at] = 0.0f;
    __syncthreads();
    pdl_launch_dependents();
    pdl_wait();

    float acc[2][4];
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[m][i] = 0.0f;

    const int g = lane >> 2, t = lane & 3;
    const int wr = warp & 3, wk = warp >> 2;
    int step = 0;  // stages issued (producer) or taken (consumers), over both passes
    for (int pass = 0; pass < 2; ++pass) {
        if (warp == kWarps) {
            for (int s = first; s < last; ++s, ++step) {
                const int slot = step % kStages;
                bool ok = true;
                if (step >= kStages) ok = mbar_wait_or_fail(smem_addr(&empty[slot]), ((step / kStages) - 1) & 1, &failed);
                if (!__all_sync(kFullWarp, ok)) break;
                if (elect_one()) {
                    const int tiles = min(kStageTiles, a.tile_cols - kStageTiles * s);
                    const uint32_t bar = smem_addr(&full[slot]), to = smem_addr(code_smem + slot * kCodeBytes);
                    mbar_expect_tx(bar, (tiles > 2 ? kCodeBytes : kBoxBytes) + tiles * kMx4TileBytes);
                    tma_load_2d(to, &codes_map, s * 256, static_cast<int>(row0), bar);
                    if (tiles > 2) tma_load_2d(to + kBoxBytes, &codes_map, s * 256 + 128, static_cast<int>(row0), bar);
                    bulk_load(smem_addr(scale_smem + slot * kStageTiles * kMx4TileBytes),
                              a.scales + (int64_t(row_tile) * a.tile_cols + kStageTiles * s) * kMx4TileBytes,
                              tiles * kMx4TileBytes, bar);
                }
                __syncwarp();
            }
        } else {
            for (int c0 = first; c0 < last; c0 += a.chunk_stages) {
                const int c1 = min(c0 + a.chunk_stages, last);
                if (c0 != first || pass != 0) consumer_sync();  // everyone is done with the last chunk
                // (token, 256 columns) pairs over the warps, four loads on their way at a time
                const int cs = 2 * (c1 - c0), pairs = cs * static_cast<int>(a.n_tokens);
                bool rest = false;
                for (int u0 = warp; u0 < pairs; u0 += 4 * kWarps) {
                    uint32_t p[4][4];
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int u = u0 + i * kWarps, token = u / cs, s = u - token * cs;
                        if (u < pairs) {
                            const uint16_t *x = a.X + token * a.ldx;
                            const int64_t col = int64_t(2 * c0 + s) * 256 + lane * 8;
                            if (a.vec_x) load8<true, false>(x, col, a.n_cols, p[i]);
                            else load8<false, false>(x, col, a.n_cols, p[i]);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int u = u0 + i * kWarps, token = u / cs, s = u - token * cs;
                        if (u < pairs)
                            rest |= convert_x<BF16>(a, p[i], lane, pass, reinterpret_cast<__half *>(x_smem + token * x_pitch + s * 512),
                                                    xs_smem + s * kTokens + token);
                    }
                }
                if (rest) has_rest = 1u;
                consumer_sync();
                for (int s = c0; s < c1; ++s, ++step) {
                    const int slot = step % kStages;
                    mbar_wait_or_fail(smem_addr(&full[slot]), (step / kStages) & 1, &failed);
                    if (kStageTiles * s + wk < a.tile_cols) {
                        const uint32_t codes = smem_addr(code_smem + slot * kCodeBytes + (wk >> 1) * kBoxBytes) + (wr * 32 + g) * 128 + t * 4;
                        const uint32_t sc = smem_addr(scale_smem + (slot * kStageTiles + wk) * kMx4TileBytes) + g * 16 + wr * 4;
                        const uint32_t xa = smem_addr(x_smem) + g * x_pitch + (s - c0) * 1024 + wk * 256 + t * 16;
                        uint32_t scale_word[4];  // rows g, g+8, g+16, g+24 of the warp's 32
#pragma unroll
                        for (int j = 0; j < 4; ++j) scale_word[j] = lds32(sc + j * 128);
                        float st[2][4];
#pragma unroll
                        for (int b = 0; b < 4; ++b) {
                            const uint4 x = lds128(xa + b * 64);
                            // chunk of row r in the swizzled box: block ^ (r & 7); all rows here have r & 7 == g
                            const uint32_t at = codes + ((((wk & 1) * 4 + b) ^ g) << 4);
#pragma unroll
                            for (int m = 0; m < 2; ++m) {
                                uint32_t lo[4], hi[4];
                                mx4_unpack8(lds32(at + m * 2048), lo);
                                mx4_unpack8(lds32(at + m * 2048 + 1024), hi);
                                const uint32_t a0[4] = {lo[0], hi[0], lo[1], hi[1]};
                                const uint32_t a1[4] = {lo[2], hi[2], lo[3], hi[3]};
                                const float s0 = mx4_scale((scale_word[2 * m] >> (8 * b)) & 0xffu);
                                const float s1 = mx4_scale((scale_word[2 * m + 1] >> (8 * b)) & 0xffu);
                                float c[4] = {0.0f, 0.0f, 0.0f, 0.0f};
                                mma_f16(c, a0, x.x, x.y);
                                mma_f16(c, a1, x.z, x.w);
#pragma unroll
                                for (int i = 0; i < 4; ++i) {
                                    const float sc_i = i < 2 ? s0 : s1;
                                    st[m][i] = b == 0 ? sc_i * c[i] : fmaf(sc_i, c[i], st[m][i]);
                                }
                            }
                        }
                        const float2 xs = *reinterpret_cast<const float2 *>(xs_smem + (2 * (s - c0) + (wk >> 1)) * kTokens + 2 * t);
#pragma unroll
                        for (int m = 0; m < 2; ++m)
#pragma unroll
                            for (int i = 0; i < 4; ++i) acc[m][i] = fmaf(i & 1 ? xs.y : xs.x, st[m][i], acc[m][i]);
                    }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(smem_addr(&empty[slot]));
                }
            }
        }
        __syncthreads();
        if (!BF16 || has_rest == 0u || failed != 0u) break;
    }
    if (failed != 0u) {
        if (warp == kWarps && lane == 0)
            for (int s = max(0, step - kStages); s < step; ++s) mbar_wait(smem_addr(&full[s % kStages]), (s / kStages) & 1);
    }

    // the column parts meet in shared memory (the stages are free: all copies have arrived)
    float *const part = reinterpret_cast<float *>(smem);
    constexpr int kPartFloats = kTokens * kPartPitch;
    if (failed != 0u) __syncthreads();
    if (warp < kWarps) {
        float *const mine = part + wk * kPartFloats + (2 * t) * kPartPitch + wr * 32 + g;
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int i = 0; i < 4; ++i) mine[(i & 1) * kPartPitch + m * 16 + (i >> 1) * 8] = acc[m][i];
    }
    __syncthreads();
    for (int at = threadIdx.x; at < static_cast<int>(a.n_tokens) * 128; at += kWarps * 32 + 32) {
        float *p = part + (at >> 7) * kPartPitch + (at & 127);
        float sum = p[0];
#pragma unroll
        for (int k = 1; k < kStageTiles; ++k) sum += p[k * kPartFloats];
        p[0] = sum;
    }
    if (slices > 1) {
        cluster_sync();
    } else {
        __syncthreads();
    }
    // (token, row) pairs over the threads of the cluster's blocks; ranks are summed in order
    const int row = threadIdx.x & 127;
    if (warp < kWarps && row0 + row < a.n_rows) {
        for (int token = slice * (kWarps / 4) + (threadIdx.x >> 7); token < a.n_tokens; token += kWarps / 4 * slices) {
            float sum = 0.0f;
            if (slices > 1) {
                float v[8];
#pragma unroll
                for (int r = 0; r < 8; ++r)  // all on their way before the first is used
                    if (r < slices)
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[r]) : "r"(remote_address(part + token * kPartPitch + row, r)));
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r < slices) sum += v[r];
            } else {
                sum = part[token * kPartPitch + row];
            }
            uint16_t bits;
            if constexpr (BF16) bits = __bfloat16_as_ushort(__float2bfloat16_rn(sum));
            else bits = __half_as_ushort(__float2half_rn(sum));
            a.Y[token * a.ldy + row0 + row] = bits;
        }
    }
    if (slices > 1) cluster_sync();  // no block leaves while its sums are read
}

sp_status launch_mx4_stream(const Mx4Product &p, cudaStream_t stream) {
    static_assert(kMx4StreamTokens == kTokens, "the entry point sends up to a product's columns here");
    CUtensorMap map;
    cudaError_t e = encode_byte_tiles(&map, p.codes, p.n_rows, mx4_blocks(p.n_cols) * 16, p.ldc, kMx4TileRows);
    if (e != cudaSuccess) return cuda_fail(e);
    int device = 0, sms = 0;
    e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return cuda_fail(e);
    StreamArgs a = {};
    a.X = static_cast<const uint16_t *>(p.X);
    a.Y = static_cast<uint16_t *>(p.Y);
    a.n_tokens = p.n_tokens;
    a.ldx = p.ldx;
    a.n_cols = p.n_cols;
    a.n_rows = p.n_rows;
    a.scales = p.scales;
    a.ldy = p.ldy;
    a.tile_cols = static_cast<int>(mx4_tile_cols(p.n_cols));
    a.stages = (a.tile_cols + kStageTiles - 1) / kStageTiles;
    a.quantize_x = p.quantize_x;
    a.vec_x = aligned16(p.X) && p.ldx % 8 == 0 && p.n_cols % 8 == 0;
    // blocks for the SMs in one round
    const int row_tiles = static_cast<int>(mx4_tile_rows(p.n_rows));
    a.slices = 1;
    while (a.slices < 8 && cluster_slices_fit(row_tiles, a.slices * 2, sms) && a.stages >= 2 * a.slices) a.slices *= 2;
    a.chunk_stages = min((a.stages + a.slices - 1) / a.slices, 8);
    auto *kernel = p.dtype == SP_BF16 ? mx4_stream_kernel<true> : mx4_stream_kernel<false>;
    static DynamicSmem limit[2];
    e = limit[p.dtype == SP_BF16].allow(reinterpret_cast<const void *>(kernel));
    if (e != cudaSuccess) return cuda_fail(e);
    ClusterPdlConfig pdl(a.slices, dim3(static_cast<unsigned>(row_tiles * a.slices)), dim3(kWarps * 32 + 32), stream);
    pdl.cfg.dynamicSmemBytes = kStages * (kCodeBytes + kStageTiles * kMx4TileBytes) +
                               kTokens * (a.chunk_stages * 1024 + 64 + a.chunk_stages * 8);
    e = cudaLaunchKernelEx(&pdl.cfg, kernel, map, a);
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

}  // namespace sp
