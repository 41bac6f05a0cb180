// Product of two microscaled 4-bit matrices on the 4-bit tensor cores (long prompts): the
// activations are quantised first (mx4_quantize.cu, into the workspace), then
//     Y [tokens, rows] = Xq Wq^T,   both operands as they are stored, scales included.
//
// Bound by the weights' bytes at few tokens; at many, by what flows into an SM (64 bytes a cycle: a
// stage of 128 x 256 rows of 128 bytes takes 800 cycles, its products 512) unless two blocks share a
// tile.  A tile is 128 tokens x N rows of the weights (N = 64 .. 256, see choose_tile), or, for a
// pair of blocks, 256 tokens, each block with 128 of them and half of the weights' rows, of which
// the tensor cores of both read.  It is summed over the columns 256 at a time:
// one thread keeps kStages of both operands and their scale tiles in flight by TMA, one issues
// the products (64 columns each; scale tiles go to tensor memory by a copy just before), four
// warps empty the accumulators.  Two accumulators alternate so that emptying one overlaps
// filling the other; 2 x 256 columns and the scales do not fit 512, so the two share 64 columns,
// which are emptied first.  Measured, quantisation of bf16 activations included, calls replayed from a
// graph: 8191 tokens x 4096 x 14336 179 us (5.4 PFLOP/s; 55 bytes a cycle into an SM, the tensor pipe
// active 74 % of the time), 512 x 13824 x 5120 24.4 us.
#include <algorithm>

#include "mx4_common.cuh"
#include "sp_tcgen05.cuh"

namespace sp {

namespace {

constexpr int kTileTokens = 128;
constexpr int kStageBytesA = kTileTokens * 128;
constexpr int kOutBytes = 32 * 128;   // a warp's piece of the output, 32 tokens x 64 rows, on its way out
constexpr int kTmemColumns = 512;
constexpr int kScaleBuffer = 24;      // columns of a stage's scales: A 2 tiles x 4, B 2 x 8

struct GemmArgs {
    const uint8_t *scale_x, *scale_w;
    uint16_t *Y;
    int64_t n_tokens, n_rows, ldy;
    int tile_cols;  // scale tiles along the columns
    int steps;      // 256-column stages
    int token_tiles, tiles;
    int slices;     // blocks of a cluster that share a tile, each with a part of the columns (not pairs)
    int tma_y;
};

}  // namespace

template <bool BF16, int N, int STAGES, bool PAIR>
__global__ void __launch_bounds__(256, 1)
mx4_gemm_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map,
                const __grid_constant__ CUtensorMap y_map, const __grid_constant__ CUtensorMap x_scale_map,
                const __grid_constant__ CUtensorMap w_scale_map, const GemmArgs a) {
    constexpr int kBlocks = PAIR ? 2 : 1, kRowsB = N / kBlocks;  // rows of the weights that a block holds
    constexpr int kStageBytesB = kRowsB * 128;
    constexpr int kOperandBytes = kStageBytesA + kStageBytesB;
    constexpr int kScaleTilesB = N > 128 ? 2 : 1;           // row tiles of scales under a tile of N rows
    constexpr int kScaleBytes = 2 * kMx4TileBytes * (1 + kScaleTilesB);
    constexpr int kSecond = N == 256 ? 192 : N;             // column of the second accumulator
    constexpr int kShared = N == 256 ? 64 : 0;              // its first columns that the first one shares
    constexpr int kScaleColumns = N == 256 ? 448 : 2 * N;   // scales follow
    // scale columns for every stage, where there is room; else two sets in turn
    constexpr bool kScalesPerStage = kScaleColumns + STAGES * kScaleBuffer <= kTmemColumns;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ uint64_t full[STAGES], empty[STAGES], acc_full[2], acc_free, drained;
    __shared__ uint32_t tmem_base, failed;
    constexpr int kPartPitch = N + 4;  // floats; rows 16 bytes apart in the banks
    float *const part = reinterpret_cast<float *>(smem);  // of a shared tile, [token][row], when the operands are done with
    uint8_t *const operands = smem, *const out_stage = smem + STAGES * kOperandBytes, *const scales = out_stage + 4 * kOutBytes;
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const int slices = PAIR ? 1 : a.slices, slice = blockIdx.x % slices;
    const int rank = PAIR ? blockIdx.x & 1 : 0, unit = blockIdx.x / (kBlocks * slices), units = gridDim.x / (kBlocks * slices);
    const int first_step = static_cast<int>(int64_t(a.steps) * slice / slices);
    const int steps = static_cast<int>(int64_t(a.steps) * (slice + 1) / slices) - first_step;
    if (threadIdx.x == 0) {
        tma_prefetch_map(&x_map);
        tma_prefetch_map(&w_map);
        for (int s = 0; s < STAGES; ++s) {
            mbar_init(smem_addr(&full[s]), kBlocks);  // of a pair: the first block's counts, for both
            mbar_init(smem_addr(&empty[s]), 1);
        }
        mbar_init(smem_addr(&acc_full[0]), 1);
        mbar_init(smem_addr(&acc_full[1]), 1);
        mbar_init(smem_addr(&acc_free), 128 * kBlocks);
        mbar_init(smem_addr(&drained), 1);
        failed = 0u;
        mbar_fence_init();
    }
    if (warp == 2) tmem_alloc<PAIR>(&tmem_base, kTmemColumns);
    tcgen05_fence_before();
    __syncthreads();
    if constexpr (PAIR) cluster_sync();  // the peer's barriers are ready
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base;
    pdl_launch_dependents();
    pdl_wait();

    if (warp == 0) {
        RingPlace<STAGES> at;
        int step = 0;
        bool ok = true;
        for (int tile = unit; ok && tile < a.tiles; tile += units) {
            const int m = tile % a.token_tiles * kBlocks + rank, n = tile / a.token_tiles;
            const int64_t wt = int64_t(n) * N / kMx4TileRows;
            const int w_tiles = static_cast<int>(min(int64_t(kScaleTilesB), mx4_tile_rows(a.n_rows) - wt));
            const uint8_t *sx = a.scale_x + int64_t(m) * a.tile_cols * kMx4TileBytes;
            const uint8_t *sw = a.scale_w + wt * a.tile_cols * kMx4TileBytes;
            for (int k = first_step; k < first_step + steps; ++k, ++step, at.next()) {
                if (step >= STAGES) ok = mbar_wait_or_fail(smem_addr(&empty[at.slot]), at.parity ^ 1u, &failed);
                if (!__all_sync(kFullWarp, ok)) { ok = false; break; }
                if (elect_one()) {
                    const uint32_t to = smem_addr(operands + at.slot * kOperandBytes), sc = smem_addr(scales + at.slot * kScaleBytes);
                    if constexpr (PAIR) {
                        const uint32_t bar = remote_address(&full[at.slot], 0);
                        mbar_expect_tx_cluster(bar, kOperandBytes + kScaleBytes);
                        tma_load_2d_pair(to, &x_map, k * 128, m * kTileTokens, bar);
                        tma_load_2d_pair(to + kStageBytesA, &w_map, k * 128, n * N + rank * kRowsB, bar);
                        // two tiles each; of an odd last one the second is not used
                        tma_load_2d_pair(sc, &x_scale_map, 0, m * a.tile_cols + 2 * k, bar);
#pragma unroll
                        for (int i = 0; i < kScaleTilesB; ++i)
                            tma_load_2d_pair(sc + (1 + i) * 2 * kMx4TileBytes, &w_scale_map, 0, static_cast<int>(wt + i) * a.tile_cols + 2 * k, bar);
                    } else {
                        const uint32_t bar = smem_addr(&full[at.slot]);
                        const int bytes = min(2, a.tile_cols - 2 * k) * kMx4TileBytes;
                        mbar_expect_tx(bar, kOperandBytes + bytes * (1 + w_tiles));
                        tma_load_2d(to, &x_map, k * 128, m * kTileTokens, bar);
                        tma_load_2d(to + kStageBytesA, &w_map, k * 128, n * N, bar);
                        bulk_load(sc, sx + k * (2 * kMx4TileBytes), bytes, bar);
                        for (int i = 0; i < w_tiles; ++i)
                            bulk_load(sc + (1 + i) * 2 * kMx4TileBytes, sw + (int64_t(i) * a.tile_cols + 2 * k) * kMx4TileBytes, bytes, bar);
                    }
                }
                __syncwarp();
            }
        }
        if (failed != 0u && lane == 0)
            for (int s = max(0, step - STAGES); s < step; ++s) mbar_wait(smem_addr(&full[s % STAGES]), (s / STAGES) & 1);
    } else if (warp == 1 && rank == 0) {
        RingPlace<STAGES> at, before;  // `before` follows two stages behind
        int step = 0, count = 0;
        bool ok = true;
        const uint64_t desc0 = desc_rows128(smem_addr(operands)), scale0 = desc_scales(smem_addr(scales));
        for (int tile = unit; ok && tile < a.tiles; tile += units, ++count) {
            const int n = tile / a.token_tiles;
            if (count > 0) ok = mbar_wait_or_fail(smem_addr(&acc_free), (count - 1) & 1, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            const uint32_t acc = tmem + (count & 1) * kSecond;
            // a tile of 64 or 192 rows may begin in the middle of a tile of scales
            const uint32_t skip = (n * N % kMx4TileRows) / 32;
            for (int k = first_step; k < first_step + steps; ++k, ++step, at.next()) {
                ok = mbar_wait_or_fail(smem_addr(&full[at.slot]), at.parity, &failed);
                // the scale columns written now were last read two stages ago (or, a set a stage, by
                // the products whose end let this stage be filled again)
                if (!kScalesPerStage && step >= 2) {
                    ok = ok && mbar_wait_or_fail(smem_addr(&empty[before.slot]), before.parity, &failed);
                    before.next();
                }
                if (!__all_sync(kFullWarp, ok)) { ok = false; break; }
                tcgen05_fence_after();
                if (elect_one()) {
                    const uint32_t sfa = tmem + kScaleColumns + (kScalesPerStage ? at.slot : step & 1) * kScaleBuffer, sfb = sfa + 8;
                    const uint64_t da = desc0 + static_cast<uint32_t>(at.slot * (kOperandBytes / 16)), db = da + kStageBytesA / 16;
                    const uint64_t sc = scale0 + static_cast<uint32_t>(at.slot * (kScaleBytes / 16));
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if (2 * k + c >= a.tile_cols) break;
                        tmem_copy_scales<PAIR>(sfa + c * 4, sc + c * (kMx4TileBytes / 16));
#pragma unroll
                        for (int i = 0; i < kScaleTilesB; ++i)
                            tmem_copy_scales<PAIR>(sfb + c * 8 + i * 4, sc + ((1 + i) * 2 + c) * (kMx4TileBytes / 16));
                    }
#pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        if (2 * k + (p >> 1) >= a.tile_cols) break;
                        mma_mxf4<PAIR>(acc, da + p * 2, db + p * 2, mxf4_instruction<PAIR>(N, p & 1), sfa + (p >> 1) * 4,
                                 sfb + (p >> 1) * 8 + skip, k > first_step || p > 0);
                    }
                    tcgen05_commit<PAIR>(smem_addr(&empty[at.slot]));
                    if (k == first_step + steps - 1) tcgen05_commit<PAIR>(smem_addr(&acc_full[count & 1]));
                }
                __syncwarp();
            }
        }
        if (failed != 0u) {
            if (elect_one()) tcgen05_commit<PAIR>(smem_addr(&drained));
            __syncwarp();
            if (lane == 0) mbar_wait(smem_addr(&drained), 0);
        }
    } else if (warp >= 4) {
        const int quarter = warp & 3;
        int count = 0;
        auto free_accumulator = [&] {
            if constexpr (PAIR) mbar_arrive_cluster(remote_address(&acc_free, 0));
            else mbar_arrive(smem_addr(&acc_free));
        };
        for (int tile = unit; tile < a.tiles; tile += units, ++count) {
            const int m = tile % a.token_tiles * kBlocks + rank, n = tile / a.token_tiles;
            const bool ok = mbar_wait_or_fail(smem_addr(&acc_full[count & 1]), (count >> 1) & 1, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            tcgen05_fence_after();
            const uint32_t acc = tmem + (count & 1) * kSecond + (static_cast<uint32_t>(quarter * 32) << 16);
            const int64_t token0 = int64_t(m) * kTileTokens + quarter * 32, token = token0 + lane;
            if (kShared == 0) {
                tcgen05_fence_before();
                free_accumulator();
            }
#pragma unroll 1
            for (int i = 0; i < N / 64; ++i) {
                // the shared columns first: the last piece of the first accumulator, the first of the second
                const int piece = kShared != 0 && (count & 1) == 0 ? (i + N / 64 - 1) % (N / 64) : i;
                uint32_t v[64];
                tmem_load32(acc + piece * 64, *reinterpret_cast<uint32_t(*)[32]>(&v[0]));
                tmem_load32(acc + piece * 64 + 32, *reinterpret_cast<uint32_t(*)[32]>(&v[32]));
                tmem_load_wait();
                if (kShared != 0 && i == 0) {
                    tcgen05_fence_before();
                    free_accumulator();
                }
                const int64_t row = int64_t(n) * N + piece * 64;
                if (slices > 1) {
                    float *const mine = part + (quarter * 32 + lane) * kPartPitch + piece * 64;
#pragma unroll
                    for (int j = 0; j < 64; j += 4)
                        *reinterpret_cast<uint4 *>(mine + j) = make_uint4(v[j], v[j + 1], v[j + 2], v[j + 3]);
                    continue;
                }
                uint32_t h[32];
#pragma unroll
                for (int j = 0; j < 32; ++j) {
                    const float lo = __uint_as_float(v[2 * j]), hi = __uint_as_float(v[2 * j + 1]);
                    if constexpr (BF16) {
                        const __nv_bfloat162 b = __floats2bfloat162_rn(lo, hi);
                        h[j] = *reinterpret_cast<const uint32_t *>(&b);
                    } else {
                        const __half2 b = __floats2half2_rn(lo, hi);
                        h[j] = *reinterpret_cast<const uint32_t *>(&b);
                    }
                }
                if (a.tma_y) {
                    uint8_t *const stage = out_stage + quarter * kOutBytes;
                    if (lane == 0) tma_store_wait_read();
                    __syncwarp();
#pragma unroll
                    for (int j = 0; j < 8; ++j)
                        *reinterpret_cast<uint4 *>(stage + lane * 128 + ((j ^ (lane & 7)) << 4)) =
                            make_uint4(h[4 * j], h[4 * j + 1], h[4 * j + 2], h[4 * j + 3]);
                    fence_async_smem();
                    __syncwarp();
                    if (lane == 0 && token0 < a.n_tokens && row < a.n_rows)
                        tma_store_2d(&y_map, smem_addr(stage), static_cast<int>(row), static_cast<int>(token0));
                } else if (token < a.n_tokens) {
                    uint16_t *y = a.Y + token * a.ldy + row;
#pragma unroll
                    for (int j = 0; j < 64; ++j)
                        if (row + j < a.n_rows) y[j] = static_cast<uint16_t>(j & 1 ? h[j >> 1] >> 16 : h[j >> 1]);
                }
            }
        }
        if (lane == 0) tma_store_wait();
        tcgen05_fence_before();
    }
    __syncthreads();
    if constexpr (PAIR) cluster_sync();
    if (warp == 2) {
        tcgen05_fence_after();
        tmem_free<PAIR>(tmem, kTmemColumns);
    }
    if (slices > 1) {
        cluster_sync();
        const int64_t token0 = int64_t(unit % a.token_tiles) * kTileTokens, row0 = int64_t(unit / a.token_tiles) * N;
        const int tokens = static_cast<int>(min(int64_t(kTileTokens), a.n_tokens - token0));
        constexpr int kQuads = N / 4;
        for (int at = slice * 256 + threadIdx.x; at < tokens * kQuads; at += slices * 256) {
            const int token = at / kQuads, r = at % kQuads * 4;
            if (row0 + r >= a.n_rows) continue;
            float4 v[8], sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int k = 0; k < 8; ++k)  // all on their way before the first is used; added in rank order
                if (k < slices)
                    asm volatile("ld.shared::cluster.v4.f32 {%0, %1, %2, %3}, [%4];"
                                 : "=f"(v[k].x), "=f"(v[k].y), "=f"(v[k].z), "=f"(v[k].w)
                                 : "r"(remote_address(part + token * kPartPitch + r, k)));
#pragma unroll
            for (int k = 0; k < 8; ++k)
                if (k < slices) {
                    sum.x += v[k].x;
                    sum.y += v[k].y;
                    sum.z += v[k].z;
                    sum.w += v[k].w;
                }
            uint32_t h[2];
            if constexpr (BF16) {
                const __nv_bfloat162 lo = __floats2bfloat162_rn(sum.x, sum.y), hi = __floats2bfloat162_rn(sum.z, sum.w);
                h[0] = *reinterpret_cast<const uint32_t *>(&lo);
                h[1] = *reinterpret_cast<const uint32_t *>(&hi);
            } else {
                const __half2 lo = __floats2half2_rn(sum.x, sum.y), hi = __floats2half2_rn(sum.z, sum.w);
                h[0] = *reinterpret_cast<const uint32_t *>(&lo);
                h[1] = *reinterpret_cast<const uint32_t *>(&hi);
            }
            uint16_t *y = a.Y + (token0 + token) * a.ldy + row0 + r;
            if (a.tma_y && row0 + r + 4 <= a.n_rows) {
                *reinterpret_cast<uint2 *>(y) = make_uint2(h[0], h[1]);
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (row0 + r + j < a.n_rows) y[j] = static_cast<uint16_t>(j & 1 ? h[j >> 1] >> 16 : h[j >> 1]);
            }
        }
        cluster_sync();  // no block leaves while its sums are read
    }
}

// Tile of a launch: the one that needs the least time in whole rounds over the SMs.  A stage's time
// is that of its bytes, 64 a cycle into an SM: 128 tokens and the block's rows of 128 bytes, and
// the scales.  Where the tiles are few, several blocks share one along the columns, at some 4500
// cycles for adding up (64 tokens x 14336 x 4096: 20 us without, 13.2 us with 4 blocks for each of
// 32 tiles).
struct GemmTile {
    int rows;
    bool pair;
    int slices;
};
static GemmTile choose_tile(int64_t token_tiles, int64_t n_rows, int steps, int sms) {
    GemmTile best = {256, false, 1};
    int64_t least = INT64_MAX;
    for (int pair = 1; pair >= 0; --pair) {
        if (pair && token_tiles < 2) continue;
        for (int n = 256; n >= (pair ? 128 : 64); n -= 64) {
            const int64_t tiles = (token_tiles + pair) / (1 + pair) * ((n_rows + n - 1) / n);
            const int64_t units = sms / (1 + pair);
            const int64_t stage = (128 + n / (1 + pair)) * 2 + 16 * (n > 128 ? 3 : 2);
            for (int slices = 1; slices <= (!pair && n <= 128 ? 8 : 1); slices *= 2) {
                if (slices > 1 && (!cluster_slices_fit(tiles, slices, sms) || steps < 2 * slices)) break;
                const int64_t cost = (tiles * slices + units - 1) / units * ((steps + slices - 1) / slices) * stage + (slices > 1 ? 4500 : 0);
                if (cost < least) {
                    least = cost;
                    best = {n, pair != 0, slices};
                }
            }
        }
    }
    return best;
}

struct GemmMaps {
    CUtensorMap x, w, y, x_scale, w_scale;
};

template <bool BF16, int N, int STAGES, bool PAIR>
static sp_status launch_gemm(const GemmMaps &maps, GemmArgs a, int sms, cudaStream_t stream) {
    auto *kernel = mx4_gemm_kernel<BF16, N, STAGES, PAIR>;
    static DynamicSmem limit;
    cudaError_t e = limit.allow(reinterpret_cast<const void *>(kernel));
    if (e != cudaSuccess) return cuda_fail(e);
    constexpr int kBlocks = PAIR ? 2 : 1;
    const int cluster = kBlocks * a.slices;
    ClusterPdlConfig pdl(cluster, dim3(static_cast<unsigned>((a.slices > 1 ? a.tiles : std::min(a.tiles, sms / kBlocks)) * cluster)),
                         dim3(256), stream);
    pdl.cfg.dynamicSmemBytes = STAGES * (kStageBytesA + N / kBlocks * 128 + 2 * kMx4TileBytes * (N > 128 ? 3 : 2)) + 4 * kOutBytes;
    e = cudaLaunchKernelEx(&pdl.cfg, kernel, maps.x, maps.w, maps.y, maps.x_scale, maps.w_scale, a);
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

int64_t mx4_gemm_workspace(int64_t n_tokens, int64_t n_cols) {
    return (n_tokens * mx4_blocks(n_cols) * 16 + 127) / 128 * 128 + mx4_tile_rows(n_tokens) * mx4_tile_cols(n_cols) * kMx4TileBytes;
}

sp_status launch_mx4_gemm(const Mx4Product &p, void *workspace, cudaStream_t stream) {
    const int64_t pitch = mx4_blocks(p.n_cols) * 16;
    uint8_t *codes = static_cast<uint8_t *>(workspace);
    uint8_t *scales = codes + (p.n_tokens * pitch + 127) / 128 * 128;
    sp_status st = launch_mx4_quantize(p.X, p.dtype, p.n_tokens, p.n_cols, p.ldx, nullptr, codes, pitch, scales, stream);
    if (st != SP_OK) return st;
    int device = 0, sms = 0;
    cudaError_t e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return cuda_fail(e);
    GemmArgs a = {};
    a.scale_x = scales;
    a.scale_w = p.scales;
    a.Y = static_cast<uint16_t *>(p.Y);
    a.n_tokens = p.n_tokens;
    a.n_rows = p.n_rows;
    a.ldy = p.ldy;
    a.tile_cols = static_cast<int>(mx4_tile_cols(p.n_cols));
    a.steps = (a.tile_cols + 1) / 2;
    a.tma_y = aligned16(p.Y) && p.ldy % 8 == 0;
    const int64_t token_tiles = (p.n_tokens + kTileTokens - 1) / kTileTokens;
    const GemmTile tile = choose_tile(token_tiles, p.n_rows, a.steps, sms);
    const int blocks = tile.pair ? 2 : 1;
    const int64_t tiles = (token_tiles + blocks - 1) / blocks * ((p.n_rows + tile.rows - 1) / tile.rows);
    if (tiles > 0x7fffffff) return SP_ERR_SHAPE;
    a.token_tiles = static_cast<int>((token_tiles + blocks - 1) / blocks);
    a.tiles = static_cast<int>(tiles);
    a.slices = tile.slices;
    GemmMaps maps = {};
    e = encode_byte_tiles(&maps.x, codes, p.n_tokens, pitch, pitch, kTileTokens);
    if (e == cudaSuccess) e = encode_byte_tiles(&maps.w, p.codes, p.n_rows, pitch, p.ldc, tile.rows / blocks);
    if (e == cudaSuccess && a.tma_y) e = encode_half_tiles(&maps.y, p.Y, p.n_tokens, p.n_rows, p.ldy, 32);
    if (tile.pair) {
        const int64_t w_tiles = mx4_tile_rows(p.n_rows) * a.tile_cols, x_tiles = token_tiles * a.tile_cols;
        if (w_tiles > 0x7fffffff || x_tiles > 0x7fffffff) return SP_ERR_SHAPE;
        if (e == cudaSuccess) e = encode_scale_tiles(&maps.x_scale, scales, x_tiles, 2);
        if (e == cudaSuccess) e = encode_scale_tiles(&maps.w_scale, p.scales, w_tiles, 2);
    }
    if (e != cudaSuccess) return cuda_fail(e);
#define SP_LAUNCH(N, S, P)                                                             \
    return p.dtype == SP_BF16 ? launch_gemm<true, N, S, P>(maps, a, sms, stream)       \
                              : launch_gemm<false, N, S, P>(maps, a, sms, stream)
    if (tile.pair) {
        switch (tile.rows) {
            case 128: SP_LAUNCH(128, 7, true);
            case 192: SP_LAUNCH(192, 5, true);
            default: SP_LAUNCH(256, 5, true);
        }
    }
    switch (tile.rows) {
        case 64: SP_LAUNCH(64, 8, false);
        case 128: SP_LAUNCH(128, 6, false);
        case 192: SP_LAUNCH(192, 4, false);
        default: SP_LAUNCH(256, 4, false);
    }
#undef SP_LAUNCH
}

}  // namespace sp
