// Product of 16-bit activations with a microscaled 4-bit matrix on the 16-bit tensor cores (more
// tokens than the streaming kernel takes in a pass).
//
// Mathematics: Y^T [rows, tokens] = V X^T, V = code * 2^(byte - 127) brought to the activations'
// type on the way to the tensor cores.  In bf16 that is exact (4-bit codes and powers of two fit at
// every scale).  binary16 has not the range, so a row of V is kept relative to its largest scale R:
// V = code * 2^(byte - R + 13), 49152 at most, and the sums are multiplied by 2^(R - 140) when they
// leave.  That is exact for scales down to 2^36 below the largest.  Rows whose scales lie further
// apart (their small weights count where the activations of the large ones are 0) are summed again
// at the end of the block, in binary32 from the codes; a block without such a row only looks at a flag.
//
// The weights are the 128 rows of a tile because that side has to be converted, every weight once for
// up to 160 tokens, and because that operand may lie in tensor memory: a thread converts 128 columns
// of its row in registers and stores them there.  (Through shared memory the converted weights were
// written once and read once at 16 KB for 64 columns, and with the activations that kept shared
// memory busy: 333 tokens x 4096 x 11008 took 50.8 us against 41.1.)  Converting a stage of 128
// columns is a long chain, so four (three) groups of four warps do every fourth stage each, a thread
// a row.  One thread streams the activations by TMA, one the codes, one issues the products, four
// warps empty the accumulators (two, alternating) and find the next tile's R; the last tile of a
// block is emptied by the converting warps too.
//
// Bound by the tensor core and the thread that feeds it: 128 tokens take 520 cycles of products a stage,
// and its wait, even for what is there already, 140 more.  Measured (f16): 333 x 4096 x 11008
// 28.8 us (1040 TFLOP/s; two rounds of tiles, the second three quarters full; 28.4 without the span of
// the scales); 73 us with one row that is summed again, 4.5 ms with all.
#include <algorithm>

#include "mx4_common.cuh"
#include "sp_tcgen05.cuh"

namespace sp {

namespace {

constexpr int kCodeSlots = 4;                    // stages of 256 columns: codes and scales as stored
constexpr int kCodeSlotBytes = kMx4TileRows * 128 + 2 * kMx4TileBytes;
constexpr int kTmemColumns = 512;

// Tiles of up to 128 tokens leave tensor memory for four stages of converted weights (of 64 columns
// of it), up to 160 for three.
template <bool WIDE>
struct Gemm16Tile {
    static constexpr int kMostTokens = WIDE ? 160 : 128;
    static constexpr int kSlots = WIDE ? 3 : 4;             // stages of 128 columns
    static constexpr int kHalfBytes = kMostTokens * 128;    // 64 columns of activations
    static constexpr int kSlotBytes = 2 * kHalfBytes;
    static constexpr int kWeightColumns = 2 * kMostTokens;  // behind two accumulators
    static constexpr int kThreads = 256 + kSlots * 128;     // 4 warps of single roles, 4 that empty, a group of 4 for every slot
    static constexpr int kSmemBytes = kSlots * kSlotBytes + kCodeSlots * kCodeSlotBytes;
};

struct Gemm16Args {
    const uint16_t *X;
    int64_t ldx, n_cols;
    const uint8_t *codes, *scales;
    int64_t ldc;
    uint16_t *Y;
    int64_t n_tokens, n_rows, ldy;
    int tile_cols;    // scale tiles along the columns
    int steps;        // 128-column stages
    int tile_tokens;  // tokens of a tile, a multiple of 16
    int row_tiles, tiles;
    int slices;       // blocks of a cluster that share a tile, each with a part of the columns
};

constexpr int kMostSpan = 36;  // binary orders between a row's scales that binary16 holds exactly

// Largest and least scale byte of a row, from words of four blocks.  A block of NaN (byte 255) has no
// say in the largest: one more, modulo 256, makes it 0; a byte 0, the scale of a block of zeros (and
// of values too small for binary16 products), has none in the least: one less makes it 255.
struct ScaleSpan {
    uint32_t most = 0, least = 0xffffffffu;
    __device__ __forceinline__ void add(uint32_t w) {
        most = __vmaxu4(most, ((w & 0x7f7f7f7fu) + 0x01010101u) ^ (w & 0x80808080u));
        least = __vminu4(least, ((w | 0x80808080u) - 0x01010101u) ^ (~w & 0x80808080u));
    }
    static __device__ __forceinline__ int largest(uint32_t w) {
        w = __vmaxu4(w, w >> 16);
        return static_cast<int>(max(w & 0xffu, (w >> 8) & 0xffu));
    }
    __device__ __forceinline__ int top() const { return max(largest(most) - 1, 0); }
    __device__ __forceinline__ int bottom() const { return 256 - largest(~least); }
};

// 2^e as binary16 bits, 0 below its range.
__device__ __forceinline__ uint32_t half_pow2(int e) {
    return e >= -14 ? static_cast<uint32_t>(e + 15) << 10 : e >= -24 ? 1u << (e + 24) : 0u;
}

// Eight codes -> eight values in the activations' type; `factor` holds the scale in both halves.
template <bool BF16>
__device__ __forceinline__ void convert8(uint32_t w, uint32_t factor, uint32_t (&h)[4]) {
    if constexpr (BF16) {
        // bytes of the bf16 magnitudes by table, signs from bit 3 of the codes
        const uint32_t sel = w & 0x77777777u, up = w << 4;
        const uint32_t hi_a = prmt(0x3f3f3f00u, 0x40404040u, sel) | (prmt(up, w, 0x5140u) & 0x80808080u);
        const uint32_t hi_b = prmt(0x3f3f3f00u, 0x40404040u, sel >> 16) | (prmt(up, w, 0x7362u) & 0x80808080u);
        const uint32_t lo_a = prmt(0xc0800000u, 0xc0804000u, sel), lo_b = prmt(0xc0800000u, 0xc0804000u, sel >> 16);
        h[0] = prmt(lo_a, hi_a, 0x5140u);
        h[1] = prmt(lo_a, hi_a, 0x7362u);
        h[2] = prmt(lo_b, hi_b, 0x5140u);
        h[3] = prmt(lo_b, hi_b, 0x7362u);
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("mul.bf16x2 %0, %0, %1;" : "+r"(h[i]) : "r"(factor));
    } else {
        mx4_unpack8(w, h);
#pragma unroll
        for (int i = 0; i < 4; ++i) asm("mul.f16x2 %0, %0, %1;" : "+r"(h[i]) : "r"(factor));
    }
}

}  // namespace

template <bool BF16, bool WIDE>
__global__ void __launch_bounds__(Gemm16Tile<WIDE>::kThreads, 1)
mx4_gemm16_kernel(const __grid_constant__ CUtensorMap x_map, const __grid_constant__ CUtensorMap w_map, const Gemm16Args a) {
    using Tile = Gemm16Tile<WIDE>;
    constexpr int kMostTokens = Tile::kMostTokens, kSlots = Tile::kSlots, kHalfBytes = Tile::kHalfBytes;
    constexpr int kSlotBytes = Tile::kSlotBytes, kWeightColumns = Tile::kWeightColumns, kThreads = Tile::kThreads;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ uint64_t full[kSlots], empty[kSlots], code_full[kCodeSlots], code_empty[kCodeSlots];
    __shared__ uint64_t acc_full[2], acc_free, last_full, top_full[8], drained;
    __shared__ uint32_t tmem_base, failed, wide_rows, wide_mask[4];
    // Largest scale byte of a row, for eight tiles in turn.  A group may have no stage of a tile and
    // then does not look at it; it has one within four tiles, and the tile after the next is the last
    // that is published before it is converted, so no barrier is two phases ahead of a group.
    __shared__ int row_top[8][kMx4TileRows];
    uint8_t *const slots = smem, *const codes = smem + kSlots * kSlotBytes;
    float *const part = reinterpret_cast<float *>(smem);  // of a shared tile, [token][row], when the slots are done with
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    if (threadIdx.x == 0) {
        tma_prefetch_map(&x_map);
        tma_prefetch_map(&w_map);
        for (int s = 0; s < kSlots; ++s) {
            mbar_init(smem_addr(&full[s]), 5);  // the activations' copy and four converting warps
            mbar_init(smem_addr(&empty[s]), 1);
        }
        for (int s = 0; s < kCodeSlots; ++s) {
            mbar_init(smem_addr(&code_full[s]), 1);
            mbar_init(smem_addr(&code_empty[s]), 4 * kSlots);  // every converting warp
        }
        mbar_init(smem_addr(&acc_full[0]), 1);
        mbar_init(smem_addr(&acc_full[1]), 1);
        mbar_init(smem_addr(&acc_free), 128);
        mbar_init(smem_addr(&last_full), 1);
        for (int i = 0; i < 8; ++i) mbar_init(smem_addr(&top_full[i]), 128);
        mbar_init(smem_addr(&drained), 1);
        failed = wide_rows = 0u;
        mbar_fence_init();
    }
    if (warp == 2) tmem_alloc(&tmem_base, kTmemColumns);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base;
    pdl_launch_dependents();
    pdl_wait();
    // With few tiles a cluster shares each: its blocks take a part of the columns and add their sums
    // up at the end.
    const int slices = a.slices, rank = blockIdx.x % slices, unit = blockIdx.x / slices, units = gridDim.x / slices;
    const int code_begin = (a.steps + 1) / 2 * rank / slices, code_steps = (a.steps + 1) / 2 * (rank + 1) / slices - code_begin;
    const int first_step = 2 * code_begin, steps = min(2 * code_steps, a.steps - first_step);

    // Accumulator -> output (or the block's part of the sums), every step-th 32 tokens from the
    // first-th on; a warp has the rows that its quarter of tensor memory holds.
    auto empty_tile = [&](int tile, int count, int quarter, int first, int step) {
        const int m = tile % a.row_tiles, n = tile / a.row_tiles;
        const uint32_t acc = tmem + (count & 1) * kMostTokens + (static_cast<uint32_t>(quarter * 32) << 16);
        const int64_t row = int64_t(m) * kMx4TileRows + quarter * 32 + lane;
        float f0 = 1.0f, f1 = 1.0f;
        if constexpr (!BF16) {
            const int e = row_top[count & 7][quarter * 32 + lane] - 140;
            f0 = __uint_as_float(static_cast<uint32_t>(e / 2 + 127) << 23);
            f1 = __uint_as_float(static_cast<uint32_t>(e - e / 2 + 127) << 23);
        }
        const int64_t token0 = int64_t(n) * a.tile_tokens;
        const int tokens = static_cast<int>(min(int64_t(a.tile_tokens), a.n_tokens - token0));
#pragma unroll 1
        for (int c = first * 32; c < tokens; c += step * 32) {
            uint32_t v[32];
            tmem_load32(acc + c, v);
            tmem_load_wait();
            if (slices > 1) {
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (c + j < tokens) part[(c + j) * kMx4TileRows + quarter * 32 + lane] = __uint_as_float(v[j]);
            } else if (row < a.n_rows) {
                uint16_t *y = a.Y + (token0 + c) * a.ldy + row;
#pragma unroll
                for (int j = 0; j < 32; ++j)
                    if (c + j < tokens) {
                        const float x = __uint_as_float(v[j]) * f0 * f1;
                        if constexpr (BF16) y[j * a.ldy] = __bfloat16_as_ushort(__float2bfloat16_rn(x));
                        else y[j * a.ldy] = __half_as_ushort(__float2half_rn(x));
                    }
            }
            __syncwarp();
        }
    };

    if (warp == 0) {
        RingPlace<kSlots> at;
        int step = 0;
        bool ok = true;
        for (int tile = unit; ok && tile < a.tiles; tile += units) {
            const int n = tile / a.row_tiles;
            for (int k = 0; k < steps; ++k, ++step, at.next()) {
                if (step >= kSlots) ok = mbar_wait_or_fail(smem_addr(&empty[at.slot]), at.parity ^ 1u, &failed);
                if (!__all_sync(kFullWarp, ok)) { ok = false; break; }
                if (elect_one()) {
                    const uint32_t bar = smem_addr(&full[at.slot]);
                    const uint32_t to = smem_addr(slots + at.slot * kSlotBytes);
                    mbar_expect_tx(bar, a.tile_tokens * 256);
                    tma_load_2d(to, &x_map, (first_step + k) * 256, n * a.tile_tokens, bar);
                    tma_load_2d(to + kHalfBytes, &x_map, (first_step + k) * 256 + 128, n * a.tile_tokens, bar);
                }
                __syncwarp();
            }
        }
        // a barrier that the converting warps no longer complete says nothing of the copy: the
        // block ends only after its slots' copies had the time of a bounded wait
        if (failed != 0u && lane == 0)
            for (int s = max(0, step - kSlots); s < step; ++s) mbar_wait(smem_addr(&full[s % kSlots]), (s / kSlots) & 1);
    } else if (warp == 3) {
        RingPlace<kCodeSlots> at;
        int step = 0;
        bool ok = true;
        for (int tile = unit; ok && tile < a.tiles; tile += units) {
            const int m = tile % a.row_tiles;
            const uint8_t *sw = a.scales + int64_t(m) * a.tile_cols * kMx4TileBytes;
            for (int k = code_begin; k < code_begin + code_steps; ++k, ++step, at.next()) {
                if (step >= kCodeSlots) ok = mbar_wait_or_fail(smem_addr(&code_empty[at.slot]), at.parity ^ 1u, &failed);
                if (!__all_sync(kFullWarp, ok)) { ok = false; break; }
                if (elect_one()) {
                    const uint32_t bar = smem_addr(&code_full[at.slot]), to = smem_addr(codes + at.slot * kCodeSlotBytes);
                    const int bytes = min(2, a.tile_cols - 2 * k) * kMx4TileBytes;
                    mbar_expect_tx(bar, kMx4TileRows * 128 + bytes);
                    tma_load_2d(to, &w_map, k * 128, m * kMx4TileRows, bar);
                    bulk_load(to + kMx4TileRows * 128, sw + k * (2 * kMx4TileBytes), bytes, bar);
                }
                __syncwarp();
            }
        }
        if (failed != 0u && lane == 0)
            for (int s = max(0, step - kCodeSlots); s < step; ++s) mbar_wait(smem_addr(&code_full[s % kCodeSlots]), (s / kCodeSlots) & 1);
    } else if (warp == 1) {
        const uint32_t instruction = f16_instruction(a.tile_tokens, BF16);
        const uint64_t desc0 = desc_rows128(smem_addr(slots));
        if (elect_one()) {  // once: electing a thread for every stage took 85 cycles each time
            RingPlace<kSlots> at;
            int count = 0;
            bool ok = true;
            for (int tile = unit; ok && tile < a.tiles; tile += units, ++count) {
                if (count > 0 && !mbar_wait_or_fail(smem_addr(&acc_free), (count - 1) & 1, &failed)) break;
                const uint32_t acc = tmem + (count & 1) * kMostTokens;
                for (int k = 0; k < steps; ++k, at.next()) {
                    ok = mbar_wait_or_fail(smem_addr(&full[at.slot]), at.parity, &failed);
                    if (!ok) break;
                    tcgen05_fence_after();
                    const uint64_t db = desc0 + static_cast<uint32_t>(at.slot * (kSlotBytes / 16));
                    const uint32_t ta = tmem + kWeightColumns + at.slot * 64;
#pragma unroll
                    for (int p = 0; p < 8; ++p)
                        mma_16bit(acc, ta + p * 8, db + (p >> 2) * (kHalfBytes / 16) + (p & 3) * 2, instruction, k > 0 || p > 0);
                    tcgen05_commit(smem_addr(&empty[at.slot]));
                }
                if (ok) tcgen05_commit(smem_addr(&acc_full[count & 1]));
                if (ok && tile + units >= a.tiles) tcgen05_commit(smem_addr(&last_full));
            }
        }
        __syncwarp();
        if (failed != 0u) {
            if (elect_one()) tcgen05_commit(smem_addr(&drained));
            __syncwarp();
            if (lane == 0) mbar_wait(smem_addr(&drained), 0);
        }
    } else if (warp >= 8) {
        // group `slot` converts every kSlots-th stage, into its own slot; a thread has a row of it
        const int slot = (warp - 8) >> 2, row = threadIdx.x & 127, swap = row & 7;
        const uint32_t scale_at = (row & 31) * 16 + (row >> 5) * 4;
        const uint32_t to = tmem + kWeightColumns + slot * 64 + (static_cast<uint32_t>((warp & 3) * 32) << 16);
        RingPlace<kCodeSlots> code_at;
        int turn = slot, count = 0;          // stages until the group's next
        uint32_t uses = 0;                   // of the group's slot
        bool ok = true;
        for (int tile = unit; ok && tile < a.tiles; tile += units, ++count) {
            int top = 0;
            if (!BF16 && turn < steps) {
                ok = mbar_wait_or_fail(smem_addr(&top_full[count & 7]), (count >> 3) & 1, &failed);
                if (!__all_sync(kFullWarp, ok)) { ok = false; break; }
                top = row_top[count & 7][row];
            }
            // every group follows every stage of codes (a barrier that it passed over might be taken
            // for a later phase), and converts at most one half of it
            for (int c = 0; c < code_steps; ++c, code_at.next()) {
                ok = mbar_wait_or_fail(smem_addr(&code_full[code_at.slot]), code_at.parity, &failed);
                if (!__all_sync(kFullWarp, ok)) { ok = false; break; }
                const int here = min(2, steps - 2 * c), sub = turn;
                if (sub >= here) {
                    turn -= here;
                    if (lane == 0) mbar_arrive(smem_addr(&code_empty[code_at.slot]));
                    continue;
                }
                turn += kSlots - here;
                const uint8_t *in = codes + code_at.slot * kCodeSlotBytes;
                const uint32_t bytes = *reinterpret_cast<const uint32_t *>(in + kMx4TileRows * 128 + sub * kMx4TileBytes + scale_at);
                uint4 w[4];
#pragma unroll
                for (int b = 0; b < 4; ++b) w[b] = *reinterpret_cast<const uint4 *>(in + row * 128 + (((sub * 4 + b) ^ swap) << 4));
                __syncwarp();  // the codes are in registers
                if (lane == 0) mbar_arrive(smem_addr(&code_empty[code_at.slot]));
#pragma unroll
                for (int half = 0; half < 2; ++half) {
                    uint32_t v[32];
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const uint32_t byte = (bytes >> (8 * (half * 2 + b))) & 0xffu;
                        uint32_t factor;
                        if constexpr (BF16) factor = byte == 255u ? 0x7fc0u : max(byte << 7, 0x0040u);
                        else factor = byte == 255u ? 0x7e00u : half_pow2(static_cast<int>(byte) - top + 13);
                        factor |= factor << 16;
                        const uint4 c = w[half * 2 + b];
                        const uint32_t words[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
                        for (int i = 0; i < 4; ++i)
                            convert8<BF16>(words[i], factor, *reinterpret_cast<uint32_t(*)[4]>(&v[b * 16 + i * 4]));
                    }
                    if (half == 0) {
                        if (uses > 0) ok = mbar_wait_or_fail(smem_addr(&empty[slot]), (uses - 1) & 1u, &failed);
                        if (!__all_sync(kFullWarp, ok)) { ok = false; break; }
                        tcgen05_fence_after();
                    }
                    tmem_store32(to + half * 32, v);
                }
                if (!ok) break;
                tmem_store_wait();
                tcgen05_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&full[slot]));
                ++uses;
            }
        }
        ok = ok && mbar_wait_or_fail(smem_addr(&last_full), 0, &failed);
        if (__all_sync(kFullWarp, ok)) {
            tcgen05_fence_after();
            empty_tile(unit + (count - 1) * units, count - 1, warp & 3, 1 + slot, 1 + kSlots);
        }
        tcgen05_fence_before();
    } else if (warp >= 4) {
        const int quarter = warp & 3;
        int count = 0;
        // the largest scale byte of this thread's row in a tile
        auto find_top = [&](int tile, int c) {
            const uint8_t *s = a.scales + int64_t(tile % a.row_tiles) * a.tile_cols * kMx4TileBytes + lane * 16 + quarter * 4;
            ScaleSpan span;
#pragma unroll 32
            for (int i = 0; i < a.tile_cols; ++i) span.add(__ldg(reinterpret_cast<const uint32_t *>(s + int64_t(i) * kMx4TileBytes)));
            row_top[c & 7][quarter * 32 + lane] = span.top();
            if (span.top() - span.bottom() > kMostSpan) wide_rows = 1u;
            mbar_arrive(smem_addr(&top_full[c & 7]));
        };
        if (!BF16 && unit < a.tiles) find_top(unit, 0);
        for (int tile = unit; tile < a.tiles; tile += units, ++count) {
            if (!BF16 && tile + units < a.tiles) find_top(tile + units, count + 1);
            const bool ok = mbar_wait_or_fail(smem_addr(&acc_full[count & 1]), (count >> 1) & 1, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            tcgen05_fence_after();
            tcgen05_fence_before();
            mbar_arrive(smem_addr(&acc_free));  // the other accumulator was emptied before
            // the last tile is emptied by all warps but the first four
            empty_tile(tile, count, quarter, 0, tile + units < a.tiles ? 1 : 1 + kSlots);
        }
        tcgen05_fence_before();
    }
    __syncthreads();
    if (warp == 2) {
        tcgen05_fence_after();
        tmem_free(tmem, kTmemColumns);
    }
    if (slices > 1) {
        cluster_sync();
        const int r = threadIdx.x & 127;
        const int64_t row = int64_t(unit % a.row_tiles) * kMx4TileRows + r, token0 = int64_t(unit / a.row_tiles) * a.tile_tokens;
        const int tokens = static_cast<int>(min(int64_t(a.tile_tokens), a.n_tokens - token0));
        float f0 = 1.0f, f1 = 1.0f;
        if constexpr (!BF16) {
            const int e = row_top[0][r] - 140;
            f0 = __uint_as_float(static_cast<uint32_t>(e / 2 + 127) << 23);
            f1 = __uint_as_float(static_cast<uint32_t>(e - e / 2 + 127) << 23);
        }
        if (row < a.n_rows) {
            constexpr int kGroups = kThreads / 128;
            for (int c = rank * kGroups + (threadIdx.x >> 7); c < tokens; c += slices * kGroups) {
                float v[8], sum = 0.0f;
#pragma unroll
                for (int k = 0; k < 8; ++k)  // all on their way before the first is used; added in rank order
                    if (k < slices)
                        asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v[k]) : "r"(remote_address(part + c * kMx4TileRows + r, k)));
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (k < slices) sum += v[k];
                const float x = sum * f0 * f1;
                if constexpr (BF16) a.Y[(token0 + c) * a.ldy + row] = __bfloat16_as_ushort(__float2bfloat16_rn(x));
                else a.Y[(token0 + c) * a.ldy + row] = __half_as_ushort(__float2half_rn(x));
            }
        }
        cluster_sync();  // no block leaves while its sums are read
    }
    // rows whose scales lie further apart than binary16 holds: the warps of the blocks that share a tile
    // take a (row, token) each
    if constexpr (!BF16) {
        if (wide_rows == 0u) return;
        constexpr int kWarps = kThreads / 32;
        for (int tile = unit; tile < a.tiles; tile += units) {
            const int64_t m = tile % a.row_tiles, row0 = m * kMx4TileRows, token0 = int64_t(tile / a.row_tiles) * a.tile_tokens;
            const int tokens = static_cast<int>(min(int64_t(a.tile_tokens), a.n_tokens - token0));
            const uint8_t *const tile_scales = a.scales + m * a.tile_cols * kMx4TileBytes;
            auto row_scales = [&](int r) { return tile_scales + (r & 31) * 16 + (r >> 5) * 4; };
            if (threadIdx.x < 4) wide_mask[threadIdx.x] = 0u;
            __syncthreads();
            for (int r = warp; r < kMx4TileRows && row0 + r < a.n_rows; r += kWarps) {
                ScaleSpan span;
                for (int i = lane; i < a.tile_cols; i += 32)
                    span.add(*reinterpret_cast<const uint32_t *>(row_scales(r) + int64_t(i) * kMx4TileBytes));
                const int orders = __reduce_max_sync(kFullWarp, span.top()) - __reduce_min_sync(kFullWarp, span.bottom());
                if (orders > kMostSpan && lane == 0) atomicOr(&wide_mask[r >> 5], 1u << (r & 31));
            }
            __syncthreads();
            for (int r = 0; r < kMx4TileRows; ++r) {
                if (((wide_mask[r >> 5] >> (r & 31)) & 1u) == 0u) continue;
                const uint8_t *const codes_of = a.codes + (row0 + r) * a.ldc, *const scales_of = row_scales(r);
                constexpr int kEach = 4;  // tokens a warp takes together
                for (int t = (rank * kWarps + warp) * kEach; t < tokens; t += slices * kWarps * kEach) {
                    float sum[kEach] = {};
                    for (int64_t c = lane * 8; c < a.n_cols; c += 256) {
                        uint32_t h[4], p[kEach][4];
#pragma unroll
                        for (int k = 0; k < kEach; ++k) {
                            const uint16_t *const x = a.X + (token0 + min(t + k, tokens - 1)) * a.ldx;  // on 16-byte boundaries
                            if (c + 8 <= a.n_cols) load8<true, false>(x, c, a.n_cols, p[k]);
                            else load8<false, false>(x, c, a.n_cols, p[k]);
                        }
                        mx4_unpack8(*reinterpret_cast<const uint32_t *>(codes_of + (c >> 1)), h);
                        const float scale = mx4_scale(scales_of[(c >> 7) * kMx4TileBytes + ((c >> 5) & 3)]);
#pragma unroll
                        for (int k = 0; k < kEach; ++k) {
                            float part = 0.0f;
#pragma unroll
                            for (int i = 0; i < 4; ++i) {
                                const float2 v = unpack2<false>(h[i]), u = unpack2<false>(p[k][i]);
                                part = fmaf(v.y, u.y, fmaf(v.x, u.x, part));
                            }
                            sum[k] = fmaf(scale, part, sum[k]);
                        }
                    }
#pragma unroll
                    for (int k = 0; k < kEach; ++k) {
#pragma unroll
                        for (int o = 16; o > 0; o >>= 1) sum[k] += __shfl_xor_sync(kFullWarp, sum[k], o);
                        if (lane == 0 && t + k < tokens) a.Y[(token0 + t + k) * a.ldy + row0 + r] = __half_as_ushort(__float2half_rn(sum[k]));
                    }
                }
            }
            __syncthreads();
        }
    }
}

// Activations that TMA cannot read (rows not on 16-byte boundaries) are copied to rows that are.
__global__ void __launch_bounds__(256)
mx4_align_rows_kernel(const uint16_t *__restrict__ X, int64_t ldx, int64_t n_cols, uint16_t *__restrict__ out, int64_t pitch) {
    pdl_launch_dependents();
    pdl_wait();
    const int64_t row = blockIdx.x;
    for (int64_t c = threadIdx.x; c < n_cols; c += blockDim.x) out[row * pitch + c] = X[row * ldx + c];
}

// Tokens of a tile, and blocks that share it along the columns where the tiles are few: the least
// time in whole rounds over the SMs.  A stage of 128 columns takes the time of 320 tokens, for waits
// and conversion, and that of its own; with more than 128 tokens, one slot less, of 432 (8192
// columns, a tile on every SM, f16: 16 tokens 26.8 us, 128 34.0, 160 43.4; 160 as two of 80: 51.7).
// Adding up a shared tile takes about that of 3000 (64 tokens x 14336 x 4096: 19.3 us, without 49.9).
struct Gemm16Shape {
    int tokens, slices;
};
static Gemm16Shape choose_shape(int64_t n_tokens, int64_t row_tiles, int steps, int sms) {
    constexpr int kMostTokens = Gemm16Tile<true>::kMostTokens;
    Gemm16Shape best = {16, 1};
    int64_t least = INT64_MAX;
    const int64_t first = (n_tokens + kMostTokens - 1) / kMostTokens;
    for (int64_t parts = first; parts <= first + 8; ++parts) {
        const int64_t n = ((n_tokens + parts - 1) / parts + 15) / 16 * 16;
        const int64_t tiles = row_tiles * ((n_tokens + n - 1) / n);
        const int64_t stage = n + (n > Gemm16Tile<false>::kMostTokens ? 432 : 320);
        for (int slices = 1; slices <= 8; slices *= 2) {
            if (slices > 1 && (!cluster_slices_fit(tiles, slices, sms) || steps < 4 * slices)) break;
            const int64_t cost = (tiles * slices + sms - 1) / sms * ((steps + slices - 1) / slices) * stage + (slices > 1 ? 3000 : 0);
            if (cost < least) {
                least = cost;
                best = {static_cast<int>(n), slices};
            }
        }
    }
    return best;
}

template <bool BF16, bool WIDE>
static cudaError_t launch_gemm16(const CUtensorMap &x_map, const CUtensorMap &w_map, const Gemm16Args &a, int sms, cudaStream_t stream) {
    using Tile = Gemm16Tile<WIDE>;
    static DynamicSmem limit;
    cudaError_t e = limit.allow(reinterpret_cast<const void *>(mx4_gemm16_kernel<BF16, WIDE>));
    if (e != cudaSuccess) return e;
    ClusterPdlConfig pdl(a.slices, dim3(static_cast<unsigned>(a.slices > 1 ? a.tiles * a.slices : std::min(a.tiles, sms))),
                         dim3(Tile::kThreads), stream);
    pdl.cfg.dynamicSmemBytes = Tile::kSmemBytes;
    return cudaLaunchKernelEx(&pdl.cfg, mx4_gemm16_kernel<BF16, WIDE>, x_map, w_map, a);
}

int64_t mx4_gemm16_workspace(int64_t n_tokens, int64_t n_cols) { return n_tokens * ((n_cols + 7) / 8 * 8) * 2; }

bool mx4_gemm16_reads(const void *X, int64_t ldx) { return aligned16(X) && ldx % 8 == 0; }

sp_status launch_mx4_gemm16(const Mx4Product &p, void *workspace, cudaStream_t stream) {
    const void *X = p.X;
    int64_t ldx = p.ldx;
    cudaError_t e;
    if (!mx4_gemm16_reads(X, ldx)) {
        ldx = (p.n_cols + 7) / 8 * 8;
        if (p.n_tokens > 0x7fffffff) return SP_ERR_SHAPE;
        PdlConfig copy(dim3(static_cast<unsigned>(p.n_tokens)), dim3(256), stream);
        e = cudaLaunchKernelEx(&copy.cfg, mx4_align_rows_kernel, static_cast<const uint16_t *>(X), p.ldx, p.n_cols,
                               static_cast<uint16_t *>(workspace), ldx);
        if (e != cudaSuccess) return cuda_fail(e);
        sp_status st = check_launch();
        if (st != SP_OK) return st;
        X = workspace;
    }
    int device = 0, sms = 0;
    e = cudaGetDevice(&device);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, device);
    if (e != cudaSuccess) return cuda_fail(e);
    Gemm16Args a = {};
    a.X = static_cast<const uint16_t *>(X);
    a.ldx = ldx;
    a.n_cols = p.n_cols;
    a.codes = p.codes;
    a.ldc = p.ldc;
    a.scales = p.scales;
    a.Y = static_cast<uint16_t *>(p.Y);
    a.n_tokens = p.n_tokens;
    a.n_rows = p.n_rows;
    a.ldy = p.ldy;
    a.tile_cols = static_cast<int>(mx4_tile_cols(p.n_cols));
    a.steps = a.tile_cols;
    const int64_t row_tiles = mx4_tile_rows(p.n_rows);
    const Gemm16Shape shape = choose_shape(p.n_tokens, row_tiles, a.steps, sms);
    a.tile_tokens = shape.tokens;
    a.slices = shape.slices;
    const int64_t tiles = row_tiles * ((p.n_tokens + a.tile_tokens - 1) / a.tile_tokens);
    if (tiles > 0x7fffffff) return SP_ERR_SHAPE;
    a.row_tiles = static_cast<int>(row_tiles);
    a.tiles = static_cast<int>(tiles);
    CUtensorMap x_map, w_map;
    e = encode_byte_tiles(&x_map, X, p.n_tokens, p.n_cols * 2, ldx * 2, a.tile_tokens);
    if (e == cudaSuccess) e = encode_byte_tiles(&w_map, p.codes, p.n_rows, mx4_blocks(p.n_cols) * 16, p.ldc, kMx4TileRows);
    if (e != cudaSuccess) return cuda_fail(e);
    const bool wide = a.tile_tokens > Gemm16Tile<false>::kMostTokens;
    if (p.dtype == SP_BF16) e = (wide ? launch_gemm16<true, true> : launch_gemm16<true, false>)(x_map, w_map, a, sms, stream);
    else e = (wide ? launch_gemm16<false, true> : launch_gemm16<false, false>)(x_map, w_map, a, sms, stream);
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

}  // namespace sp
