// Attention of a batch whose sequences share prefixes, over the 8-bit cache.
//
// Mathematics: as in cache_attention.cu, with the tokens in two parts.  The queries of a group, its
// sequences' tokens and heads of one kv head, are the rows of one product with the prefix's keys and
// one with its values, here; each sequence's own tokens are the other kernel's; a third joins their
// sums by the rule of the online softmax.
//
// A block takes 128 (or 2 x 128) rows and a stretch of the prefix, 64 tokens a step:
//   S [128 x 64] = Q K^T     Q in tensor memory, K converted to the queries' type in shared memory
//   O [128 x D] += P V       P in tensor memory, in the place of S; V converted to bf16, read the other way
// e4m3 converts exactly to binary16 and bf16, and the queries enter as they are.  P times the value
// scale enters in two bf16 parts: 2^-18 of itself, with binary32's range, so that no scale needs a
// reference but in the last exponents.  A thread owns a row: its maximum and sum stay in registers,
// and nothing crosses lanes.  The maximum is raised only when weights exceed 2^14, which spares a pass
// over the scores.
//
// Two groups of four softmax warps, each with sums of its own, hide one another's latency: with 256
// rows each has 128 of them, with 128 they take the steps in turn and their sums are joined at the end.
// Four warps convert keys, four values, one issues products, one copies, one looks scales up.
//
// What bounds it: a step of 64 tokens and 128 rows is 16 KB of cache (0.37 us of an SM's share of the
// memory rate) and 768 cycles of products, and takes 1.0 us; the issue slots are 60 % used (a SMSP has
// some 1150 instructions a step: conversions, weights, and the waits between five kinds of warps), the
// tensor pipe 35 %.  A block starts and ends in 10 us (queries, first scores; sums written).  What did
// not pay: one group of softmax warps (2.2 us a step), conversion of keys and values by the same warps
// (a step's values wait for the product two steps before, and the next keys behind them: 2.4 us), a
// pass over the scores for their maximum (1.2 us), two warps for the two products (1.3 us), P in two binary16 parts (saves a
// sixth of the instructions, but ends at 2^-36 of the largest weight).
// Measured (replayed from a graph, tails and join included): 8 x 32 sequences of 8191 tokens, 32 heads over 8 of
// 128, 126 us (276 TFLOP/s; 15.3 ms with a warp a query); 64 sequences of 8191 tokens, 40 heads, 84 us; 16
// sequences of 4095 tokens, two queries each, 33 us; 4 sequences of 517 tokens, 16 heads of 64, 17.3 us.
#include <algorithm>

#include "cache_common.cuh"
#include "sp_tcgen05.cuh"

namespace sp {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.4028234663852886e38f;
constexpr float kRaise = 16384.0f;   // weights of 32 tokens whose sum exceeds this raise the maximum
constexpr int kScaleSlots = 8;       // steps of scales
constexpr float kFarMaximum = 16777216.0f;  // 2^24: the maximum's own rounding is off by 1 from here on
constexpr int kFarScale = -40;       // of a value scale below the reference
constexpr int kRaiseScale = 40;      // how far a value scale may exceed its reference
constexpr int kStep = 64;            // tokens
constexpr int kTmemColumns = 512;
// Of a block.  The tensor cores cut what they add to, 8 times a step, so that a sum shrinks with its length:
// by 2^-16 over 128 steps (256 rows, positive values), by 2^-12 over 1024, by 2^-8.5 over 8192.
constexpr int kMostSteps = 128;
constexpr int kConverted = 3;        // steps of converted keys, and of values; of scores too, with 128 rows

template <int D, int TILES>
struct PrefixTile {
    static constexpr int kSlots = D == 128 ? 4 : 10;           // steps of codes on their way
    static constexpr int kBuffers = TILES == 1 ? 3 : 2;        // of scores
    static constexpr int kRawBytes = 2 * kStep * D;            // keys, then values
    static constexpr int kHalfBytes = kStep * 128;             // 64 converted columns
    static constexpr int kConvBytes = D / 64 * kHalfBytes;     // keys (or values) of a step
    static constexpr int kStageBytes = 8 * 4096;               // of queries on their way: the values' place, and more
    static constexpr int kSmem = kSlots * kRawBytes + kConverted * kConvBytes + std::max(kConverted * kConvBytes, kStageBytes);
    static constexpr int kSoftmaxWarps = 8;
    static constexpr int kConvertWarps = 8;                    // half of them keys, half values
    static constexpr int kWarps = kSoftmaxWarps + kConvertWarps + 3;
    // tensor memory: queries of a tile, scores, sums of a stream
    static __device__ constexpr uint32_t q(int t) { return t * 64; }
    static __device__ constexpr uint32_t s(int b) { return TILES * 64 + b * 64; }
    static __device__ constexpr uint32_t o(int g) { return 256 + g * 128; }
};

struct PrefixArgs {
    sp_cache cache;
    SharedGroups groups;
    SharedParts parts;
    const uint16_t *Q;
    sp_strides q;
    const int32_t *lens;
    int64_t n_q, max_len;
    int group, rows;        // heads of a kv head; rows of a sequence (n_q * group)
    int row_tiles, splits;  // blocks along the rows, along the prefix
    int copies;             // of the rows in a tile, each with a share of a step's tokens
    int block_shift;
    float scale_log2;
    bool q_pieces;          // whether queries lie on 16-byte boundaries
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// a less one half of a pair of bf16 values, in one instruction.
template <int HALF>
__device__ __forceinline__ float less_bf16(float a, uint32_t pair) {
    unsigned short lo, hi;
    asm("mov.b32 {%0, %1}, %2;" : "=h"(lo), "=h"(hi) : "r"(pair));
    float d;
    asm("fma.rn.f32.bf16 %0, %1, %2, %3;" : "=f"(d) : "h"(HALF ? hi : lo), "h"(static_cast<unsigned short>(0xbf80)), "f"(a));
    return d;
}
// 32 values -> two bf16 parts of each.
__device__ __forceinline__ void split16(float2 (&p)[16], uint32_t (&part)[32]) {
#pragma unroll
    for (int j = 0; j < 16; ++j) part[j] = pack_bf16(p[j].x, p[j].y);
#pragma unroll
    for (int j = 0; j < 16; ++j) p[j] = make_float2(less_bf16<0>(p[j].x, part[j]), less_bf16<1>(p[j].y, part[j]));
#pragma unroll
    for (int j = 0; j < 16; ++j) part[16 + j] = pack_bf16(p[j].x, p[j].y);
}
__device__ __forceinline__ float max3(float a, float b, float c) {
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max16(const uint32_t *v) {
    auto f = [&](int i) { return __uint_as_float(v[i]); };
    const float a = max3(f(0), f(1), f(2)), b = max3(f(3), f(4), f(5)), c = max3(f(6), f(7), f(8));
    const float d = max3(f(9), f(10), f(11)), e = max3(f(12), f(13), f(14));
    return max3(max3(a, b, c), fmaxf(d, e), f(15));
}
__device__ __forceinline__ uint4 load_shared16(uint32_t at) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at));
    return v;
}
__device__ __forceinline__ void store_shared16(uint32_t at, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

}  // namespace

template <bool BF16, int D, int TILES>
__global__ void __launch_bounds__(PrefixTile<D, TILES>::kWarps * 32, 1)
cache_prefix_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                    const __grid_constant__ PrefixArgs a) {
    using Tile = PrefixTile<D, TILES>;
    constexpr int kSlots = Tile::kSlots, kBuffers = Tile::kBuffers, kSoftmaxWarps = Tile::kSoftmaxWarps;
    extern __shared__ __align__(1024) uint8_t smem[];
    __shared__ uint64_t raw_full[kSlots], raw_empty[kSlots], k_full[kConverted], k_empty[kConverted], v_full[kConverted], v_empty[kConverted];
    __shared__ uint64_t s_full[kBuffers], p_full[kBuffers], weighed_first, drained;
    __shared__ uint32_t tmem_base, failed, present[kSlots];
    __shared__ float4 group_sums[2][128];  // TILES == 1: maximum, sum, 2^reference of a group's rows
    __shared__ uint64_t q_full, scale_full[kScaleSlots], scale_empty[kScaleSlots];
    __shared__ float4 scale_k[kScaleSlots];  // of 16 tokens each
    __shared__ int4 scale_v[kScaleSlots];    // as exponents, less the reference
    __shared__ int2 scale_info[kScaleSlots];                       // which of the four are there; the reference
    __shared__ int all_see, any_sees, any_nan, nan_from[D];  // tokens before which all rows see, some row sees
    __shared__ uint32_t row_top[2][128];
    const sp_cache &c = a.cache;
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const int head = blockIdx.y / a.row_tiles, row0 = blockIdx.y % a.row_tiles * (128 * TILES);
    if (threadIdx.x == 0) {
        tma_prefetch_map(&k_map);
        tma_prefetch_map(&v_map);
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(smem_addr(&raw_full[i]), 1);
            mbar_init(smem_addr(&raw_empty[i]), 8);
        }
        for (int i = 0; i < kConverted; ++i) {
            mbar_init(smem_addr(&k_full[i]), 4);
            mbar_init(smem_addr(&v_full[i]), 4);
            mbar_init(smem_addr(&k_empty[i]), 1);
            mbar_init(smem_addr(&v_empty[i]), 1);
        }
        for (int b = 0; b < kBuffers; ++b) {
            mbar_init(smem_addr(&s_full[b]), 1);
            mbar_init(smem_addr(&p_full[b]), 4);
        }
        mbar_init(smem_addr(&drained), 1);
        mbar_init(smem_addr(&weighed_first), 1);
        mbar_init(smem_addr(&q_full), kSoftmaxWarps);
        for (int i = 0; i < kScaleSlots; ++i) {
            mbar_init(smem_addr(&scale_full[i]), 1);
            mbar_init(smem_addr(&scale_empty[i]), 4 * TILES);
        }
        failed = 0u;
        all_see = 0x7fffffff;
        any_sees = 0;
        any_nan = 0;
        mbar_fence_init();
    }
    for (int d = threadIdx.x; d < D; d += Tile::kWarps * 32) nan_from[d] = 0x7fffffff;
    constexpr int kProducts = kSoftmaxWarps + Tile::kConvertWarps, kCopies = kProducts + 1, kScales = kProducts + 2;
    if (warp == kProducts) tmem_alloc(&tmem_base, kTmemColumns);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base;
    pdl_launch_dependents();
    pdl_wait();

    const SharedGroup g = shared_group(a.groups, c, blockIdx.z);
    const int rows = static_cast<int>(max(int64_t(0), g.end - g.begin)) * a.rows;  // of the group
    const int shift = a.block_shift;
    const int tokens = rows > row0 ? static_cast<int>(g.blocks << shift) : 0;
    const int steps = (tokens + kStep - 1) / kStep;
    const int first = static_cast<int>(int64_t(steps) * blockIdx.x / a.splits);
    const int last = static_cast<int>(int64_t(steps) * (blockIdx.x + 1) / a.splits), count = last - first;
    const int32_t *table = c.table + g.begin * c.ld_table;
    // Block that holds the token; -1 behind the prefix and where the table names none.
    auto block_at = [&](int token) {
        const int id = token < tokens ? table[token >> shift] : -1;
        return static_cast<uint32_t>(id) < static_cast<uint32_t>(c.n_blocks) ? id : -1;
    };

    const uint32_t raw = smem_addr(smem), conv = raw + kSlots * Tile::kRawBytes;  // conv: keys, then values

    // The lanes of a warp hold the blocks of eight steps, one for every 16 tokens: a load of the table takes
    // longer than a step.
    constexpr int kHeld = 8;
    auto blocks_from = [&](int step) { return step + (lane >> 2) < count ? block_at((first + step) * kStep + lane * 16) : -1; };
    if (warp == kScales) {
        // ---- scales: the values' over a power of two that follows the largest by at most 2^40
        auto scale_of = [&](const float *scales, int id) { return id >= 0 ? scales[int64_t(id) * c.n_kv_heads + head] : 0.0f; };
        int id = blocks_from(0), next_id = blocks_from(kHeld), after_id = blocks_from(2 * kHeld), reference = -200;
        float ks = scale_of(c.k_scale, id), vs = scale_of(c.v_scale, id);
        float next_ks = scale_of(c.k_scale, next_id), next_vs = scale_of(c.v_scale, next_id);
        RingPlace<kScaleSlots> at;
        // what lies behind all that the rows see may hold any scale, and must not become the reference
        bool ok = mbar_wait_or_fail(smem_addr(&q_full), 0, &failed);
        for (int step = 0; step < count; ++step, at.next()) {
            const int turn = step % kHeld;
            if (step > 0 && turn == 0) {
                id = next_id;
                ks = next_ks;
                vs = next_vs;
                next_id = after_id;
                next_ks = scale_of(c.k_scale, next_id);
                next_vs = scale_of(c.v_scale, next_id);
                after_id = blocks_from(step + 2 * kHeld);
            }
            // lanes 0 .. 3 take a piece of 16 tokens
            const int holder = turn * 4 + (lane & 3);
            const int held_id = __shfl_sync(kFullWarp, id, holder);
            const int piece_id = (first + step) * kStep + (lane & 3) * 16 < any_sees ? held_id : -1;
            const float piece_k = __shfl_sync(kFullWarp, ks, holder), piece_v = __shfl_sync(kFullWarp, vs, holder);
            const unsigned here = __ballot_sync(kFullWarp, piece_id >= 0) & 0xfu;
            int e = piece_id >= 0 ? exponent_of(piece_v) : -200;
            e = max(e, __shfl_xor_sync(kFullWarp, e, 1));
            e = max(e, __shfl_xor_sync(kFullWarp, e, 2));
            if (e > reference + kRaiseScale) reference = e;
            if (step >= kScaleSlots) ok = ok && mbar_wait_or_fail(smem_addr(&scale_empty[at.slot]), at.parity ^ 1u, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            if (lane < 4) {
                reinterpret_cast<float *>(&scale_k[at.slot])[lane] = piece_k;
                reinterpret_cast<int *>(&scale_v[at.slot])[lane] = piece_id >= 0 ? exponent_of(piece_v) - reference : 0;
            }
            if (lane == 0) scale_info[at.slot] = make_int2(static_cast<int>(here), reference);
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&scale_full[at.slot]));
        }
    } else if (warp == kCopies) {
        // ---- copies: a lane 16 tokens
        constexpr uint32_t kPiece = 16 * D;
        RingPlace<kSlots> at;
        bool ok = true;
        int ids = blocks_from(0), next_ids = blocks_from(kHeld), issued = 0;
        for (int step = 0; step < count; ++step, at.next()) {
            const int turn = step % kHeld;
            if (step > 0 && turn == 0) {
                ids = next_ids;
                next_ids = blocks_from(step + kHeld);
            }
            const int id = __shfl_sync(kFullWarp, ids, turn * 4 + (lane & 3));
            const bool mine = lane < 4 && id >= 0;
            if (step >= kSlots) ok = mbar_wait_or_fail(smem_addr(&raw_empty[at.slot]), at.parity ^ 1u, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            const unsigned here = __ballot_sync(kFullWarp, mine);
            const uint32_t bar = smem_addr(&raw_full[at.slot]), to = raw + at.slot * Tile::kRawBytes + lane * kPiece;
            if (lane == 0) {
                present[at.slot] = here;
                mbar_expect_tx(bar, 2 * kPiece * __popc(here));
            }
            __syncwarp();
            if (mine) {
                const int y = ((id * c.n_kv_heads + head) << shift) + (((first + step) * kStep + lane * 16) & ((1 << shift) - 1));
                tma_load_2d(to, &k_map, 0, y, bar);
                tma_load_2d(to + kStep * D, &v_map, 0, y, bar);
            }
            issued = step + 1;
            __syncwarp();
        }
        if (failed != 0u && lane == 0)
            for (int s = max(0, issued - kSlots); s < issued; ++s) mbar_wait(smem_addr(&raw_full[s % kSlots]), (s / kSlots) & 1);
    } else if (warp == kProducts) {
        // ---- products.  The warp walks the loop together and elects a thread for the instructions alone:
        // operands then stay in uniform registers.  A step's scores go where the weights of three steps before
        // (with 256 rows: of the step before) were, once the product that reads those is done: products are only
        // promised to run in the order of their issue where accumulator and shape are the same (right behind
        // it: 1 to 5 % less for a call, 7 % at worst).
        const uint32_t qk = f16_instruction(kStep, BF16), pv = f16_instruction(D, true) | kColumnsB;
        const uint32_t base = __shfl_sync(kFullWarp, tmem, 0);
        const int steps_here = __shfl_sync(kFullWarp, count, 0);
        auto all = [&](bool ok) {
            ok = __all_sync(kFullWarp, ok);
            tcgen05_fence_after();
            return ok;
        };
        auto scores = [&](int t, int step) {  // of one thread
            const int s_at = TILES == 1 ? step % 3 : t;
            const uint64_t keys = desc_rows128(conv + step % kConverted * Tile::kConvBytes);
#pragma unroll
            for (int p = 0; p < D / 16; ++p)
                mma_16bit(base + Tile::s(s_at), base + Tile::q(t) + p * 8, keys + (p >> 2) * (Tile::kHalfBytes / 16) + (p & 3) * 2, qk, p > 0);
            tcgen05_commit(smem_addr(&s_full[s_at]));
            if (t == 1) tcgen05_commit(smem_addr(&k_empty[step % kConverted]));
        };
        auto values = [&](int t, int step) {
            const int p_at = TILES == 1 ? step % 3 : t, g = TILES == 1 ? step & 1 : t;
            const uint64_t v = desc_columns128(conv + (kConverted + step % kConverted) * Tile::kConvBytes, Tile::kHalfBytes);
#pragma unroll
            for (int p = 0; p < 8; ++p)  // of 32 tokens both parts, 16 tokens each
                mma_16bit(base + Tile::o(g), base + Tile::s(p_at) + p * 8, v + ((p >> 2) * 2 + (p & 1)) * (16 * 128 / 16), pv,
                          step >= (TILES == 1 ? 2 : 1) || p > 0);
            if (TILES == 1 || t == 1) tcgen05_commit(smem_addr(&v_empty[step % kConverted]));
        };
        bool ok = all(mbar_wait_or_fail(smem_addr(&q_full), 0, &failed));
        if constexpr (TILES == 1) {
            // Whichever product has its operands goes next (in a fixed order, 16 rows took 0.86 us a step
            // for 0.77).  The lanes look at the four barriers at once: weights, values, keys, the scores' place.
            int scored = 0, weighed = 0;
            const int which = lane & 3;
            const uint32_t bars = smem_addr(which == 0 ? p_full : which == 1 ? v_full : which == 2 ? k_full : v_empty);
            RingPlace<3> weigh_at, score_at;
            for (uint32_t idle = 0; ok && weighed < steps_here;) {
                // (a place that has not been used yet counts as free: its phase before)
                const bool ready = mbar_test(bars + 8 * (which < 2 ? weigh_at.slot : score_at.slot),
                                             which < 2 ? weigh_at.parity : score_at.parity ^ (which == 3 ? 1u : 0u));
                const unsigned looks = __ballot_sync(kFullWarp, ready);
                const bool weigh = (looks & 3u) == 3u && weighed < scored;
                const bool score = (looks & 12u) == 12u && scored < steps_here && scored - weighed < 3;
                if (!weigh && !score) {
                    if (++idle > kWaitLimit && lane == 0) mbar_give_up(&failed);
                    if (idle > kWaitLimit || (idle & 15u) == 0u) ok = __all_sync(kFullWarp, *static_cast<volatile uint32_t *>(&failed) == 0u);
                    continue;
                }
                idle = 0;
                __syncwarp();
                tcgen05_fence_after();
                if (elect_one()) {
                    if (weigh) values(0, weighed);
                    if (score) scores(0, scored);
                }
                __syncwarp();
                if (weigh) {
                    ++weighed;
                    weigh_at.next();
                }
                if (score) {
                    ++scored;
                    score_at.next();
                }
            }
        } else {
            // two tiles in turn (as above, 12 % more)
            if (ok && steps_here > 0 && (ok = all(mbar_wait_or_fail(smem_addr(&k_full[0]), 0, &failed)))) {
                if (elect_one()) {
                    scores(0, 0);
                    scores(1, 0);
                }
                __syncwarp();
            }
            for (int step = 0; ok && step < steps_here; ++step) {
                const int next = step + 1;
                const uint32_t v_bar = smem_addr(&v_full[step % kConverted]), v_use = step / kConverted & 1;
                const uint32_t k_bar = next < steps_here ? smem_addr(&k_full[next % kConverted]) : v_bar, k_use = next < steps_here ? next / kConverted & 1 : v_use;
#pragma unroll
                for (int t = 0; t < 2; ++t) {
                    if (t == 0) ok = all(mbar_wait3_or_fail(v_bar, v_use, k_bar, k_use, smem_addr(&p_full[0]), step & 1, &failed));
                    else ok = ok && all(mbar_wait_or_fail(smem_addr(&p_full[1]), step & 1, &failed));
                    if (!ok) break;
                    if (elect_one()) {
                        values(t, step);
                        if (t == 0) tcgen05_commit(smem_addr(&weighed_first));
                    }
                    __syncwarp();
                    if (next >= steps_here) continue;
                    ok = all(t == 0 ? mbar_wait_or_fail(smem_addr(&weighed_first), step & 1, &failed)
                                    : mbar_wait_or_fail(smem_addr(&v_empty[step % kConverted]), v_use, &failed));
                    if (!ok) break;
                    if (elect_one()) scores(t, next);
                    __syncwarp();
                }
            }
        }
        __syncwarp();
        if (failed != 0u) {
            if (elect_one()) tcgen05_commit(smem_addr(&drained));
            __syncwarp();
            if (lane == 0) mbar_wait(smem_addr(&drained), 0);
        }
    } else if (warp >= kSoftmaxWarps && warp < kProducts) {
        // ---- conversion: a thread 16 codes at a time; four warps keys, four values
        const int thread = threadIdx.x & 127;
        constexpr int kEach = kStep * D / 16 / 128;
        // Eight lanes read and write all banks: of the chunks of a row's half and those of the row whose
        // number differs in bits 0 and 2 (D = 64: of a row and the next).
        int r[kEach], ch[kEach];
        uint32_t in[kEach], out[kEach];
#pragma unroll
        for (int i = 0; i < kEach; ++i) {
            const int x = i * 128 + thread;
            r[i] = D == 128 ? (x >> 4 << 1) ^ (x & 4 ? 5 : 0) : x >> 2;
            ch[i] = D == 128 ? (x >> 1 & 4) | (x & 3) : x & 3;
            in[i] = r[i] * D + ((ch[i] ^ (D == 128 ? r[i] & 7 : (r[i] >> 1) & 3)) << 4);
            out[i] = (ch[i] >> 2) * Tile::kHalfBytes + r[i] * 128 + ((((ch[i] & 3) * 2) ^ (r[i] & 7)) << 4);
        }
        RingPlace<kSlots> at;
        auto convert_steps = [&](auto is_key) {
            constexpr bool KEY = decltype(is_key)::value;
            // (the product with the keys in a buffer fills the scores of the same number)
            uint64_t *full = KEY ? k_full : v_full, *empty = !KEY ? v_empty : TILES == 1 ? s_full : k_empty;
            // which tokens all rows see is known when the queries are there
            bool ok = KEY || mbar_wait_or_fail(smem_addr(&q_full), 0, &failed);
            int buffer = 0, uses = 0;
            for (int step = 0; step < count; ++step, at.next()) {
                if (uses > 0) ok = ok && mbar_wait2_or_fail(smem_addr(&raw_full[at.slot]), at.parity, smem_addr(&empty[buffer]), (uses - 1) & 1, &failed);
                else ok = ok && mbar_wait_or_fail(smem_addr(&raw_full[at.slot]), at.parity, &failed);
                if (!__all_sync(kFullWarp, ok)) break;
                const uint32_t from = raw + at.slot * Tile::kRawBytes + (KEY ? 0 : kStep * D), here = present[at.slot];
                const uint32_t to = conv + (KEY ? buffer : kConverted + buffer) * Tile::kConvBytes;
                uint4 w[kEach];
#pragma unroll
                for (int i = 0; i < kEach; ++i) w[i] = load_shared16(from + in[i]);
                if constexpr (!KEY) {
                    const int token0 = (first + step) * kStep;
                    if (token0 + kStep > all_see) {
                        // NaN that some rows do not see: 0 here, and noted for those who do
#pragma unroll
                        for (int i = 0; i < kEach; ++i) {
                            if (!((here >> (r[i] >> 4)) & 1u)) continue;
                            uint32_t *word = reinterpret_cast<uint32_t *>(&w[i]);
#pragma unroll
                            for (int k = 0; k < 16; ++k)
                                if (((word[k >> 2] >> (8 * (k & 3))) & 0x7fu) == 0x7fu) {
                                    atomicMin(&nan_from[ch[i] * 16 + k], token0 + r[i]);
                                    any_nan = 1;
                                    word[k >> 2] &= ~(0xffu << (8 * (k & 3)));
                                }
                        }
                    }
                    if (here != 0xfu) {
#pragma unroll
                        for (int i = 0; i < kEach; ++i)
                            if (!((here >> (r[i] >> 4)) & 1u)) w[i] = make_uint4(0u, 0u, 0u, 0u);
                    }
                }
                __syncwarp();  // the codes are in registers
                if (lane == 0) mbar_arrive(smem_addr(&raw_empty[at.slot]));
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    uint32_t h[8];
                    const uint32_t words[4] = {w[i].x, w[i].y, w[i].z, w[i].w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) e4m3_to_f16(words[k], h[2 * k], h[2 * k + 1]);
                    if constexpr (!KEY || BF16) {
                        float2 f[8];
#pragma unroll
                        for (int k = 0; k < 8; ++k) f[k] = unpack2<false>(h[k]);
#pragma unroll
                        for (int k = 0; k < 8; ++k) h[k] = pack_bf16(f[k].x, f[k].y);
                    }
                    store_shared16(to + out[i], h[0], h[1], h[2], h[3]);
                    store_shared16(to + (out[i] ^ 16u), h[4], h[5], h[6], h[7]);
                }
                fence_async_smem();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_addr(&full[buffer]));
                if (++buffer == kConverted) {
                    buffer = 0;
                    ++uses;
                }
            }
        };
        if (warp < kSoftmaxWarps + 4) convert_steps(std::true_type{});
        else convert_steps(std::false_type{});
    } else if (warp < kSoftmaxWarps) {
        // ---- softmax: a thread a row, of the steps stream, stream + kEvery, ...
        const int stream = warp >> 2, tile = TILES == 1 ? 0 : stream;
        // Up to 64 rows stand twice in their tile, and each copy takes half of a step's tokens.
        const int copy = TILES == 1 && a.copies == 2 ? (warp & 3) >> 1 : -1;
        const int row = row0 + tile * 128 + (copy >= 0 ? warp & 1 : warp & 3) * 32 + lane;
        const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
        int limit = 0x7ffffffe;            // the last token that the row sees
        float undo = fabsf(a.scale_log2);  // its sign goes to the queries: factors of scores are positive
        {
            // A warp brings 64 columns of its rows at a time (with 128 rows, the groups take one each where
            // a head has 128): read along the rows, and turned in shared memory, the values' own from here
            // on only, so that a thread gets its row's.
            constexpr int kHalves = TILES == 1 ? 1 : D / 64;
            const bool loads = TILES == 2 || stream < D / 64;
            const int half0 = TILES == 1 ? stream : 0;
            const uint32_t stage = conv + kConverted * Tile::kConvBytes + warp * 4096;
            const bool valid = row < rows;
            const int64_t seq = g.begin + row / a.rows, i = row % a.rows / a.group;
            const int64_t at = seq * a.q.seq + i * a.q.token + (head * a.group + row % a.group) * a.q.head;
            const unsigned all_valid = __ballot_sync(kFullWarp, valid);
            uint32_t q[kHalves][32];
            if (loads && a.q_pieces) {
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
                    uint4 w[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int r = k * 4 + (lane >> 3);
                        const int64_t from = __shfl_sync(kFullWarp, at, r) + (half0 + h) * 64 + (lane & 7) * 8;
                        w[k] = (all_valid >> r) & 1u ? *reinterpret_cast<const uint4 *>(a.Q + from) : make_uint4(0u, 0u, 0u, 0u);
                    }
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        const int r = k * 4 + (lane >> 3);
                        store_shared16(stage + r * 128 + (((lane & 7) ^ (r & 7)) << 4), w[k].x, w[k].y, w[k].z, w[k].w);
                    }
                    __syncwarp();
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        *reinterpret_cast<uint4 *>(&q[h][k * 4]) = load_shared16(stage + lane * 128 + ((k ^ (lane & 7)) << 4));
                    __syncwarp();
                }
            } else if (loads) {
#pragma unroll
                for (int h = 0; h < kHalves; ++h)
#pragma unroll
                    for (int k = 0; k < 32; ++k) {
                        const uint16_t *from = a.Q + at + (half0 + h) * 64 + 2 * k;
                        q[h][k] = valid ? from[0] | uint32_t(from[1]) << 16 : 0u;
                    }
            }
            if (valid) {
                const int64_t len = a.lens[seq];
                limit = static_cast<int>(max(int64_t(-1), min(min(len - a.n_q + i, min(len, a.max_len) - 1), int64_t(tokens))));
            }
            const int least = __reduce_min_sync(kFullWarp, limit), most = __reduce_max_sync(kFullWarp, valid ? limit : -1);
            if (lane == 0) {
                atomicMin(&all_see, least + 1);
                atomicMax(&any_sees, most + 1);
            }
            if constexpr (BF16) {
                // sums of products with codes up to 448 stay in binary32's range
                uint32_t top = 0;
                if (loads)
#pragma unroll
                    for (int h = 0; h < kHalves; ++h)
#pragma unroll
                        for (int k = 0; k < 32; ++k) top = __vmaxu2(top, q[h][k] & 0x7fff7fffu);
                top = max(top & 0xffffu, top >> 16);
                if constexpr (TILES == 1) {
                    row_top[stream][(warp & 3) * 32 + lane] = top;
                    asm volatile("bar.sync 1, 256;" ::: "memory");
                    top = max(top, row_top[1 - stream][(warp & 3) * 32 + lane]);
                }
                if (top > kLargeQuery >> 16) {
                    undo *= pow2(64);
#pragma unroll
                    for (int h = 0; h < kHalves; ++h)
#pragma unroll
                        for (int k = 0; k < 32; ++k) {
                            const float2 v = unpack2<true>(q[h][k]);
                            q[h][k] = pack_bf16(v.x * pow2(-64), v.y * pow2(-64));
                        }
                }
            }
            const uint32_t sign = a.scale_log2 < 0.0f ? 0x80008000u : 0u;
            __syncwarp();
            if (loads) {
#pragma unroll
                for (int h = 0; h < kHalves; ++h) {
#pragma unroll
                    for (int k = 0; k < 32; ++k) q[h][k] ^= sign;
                    tmem_store32(tmem + lanes + Tile::q(tile) + (half0 + h) * 32, q[h]);
                }
                tmem_store_wait();
                tcgen05_fence_before();
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&q_full));
        }
        constexpr int kEvery = TILES == 1 ? 2 : 1;
        const int from = TILES == 1 ? stream : 0, turns = (count - from + kEvery - 1) / kEvery;
        float m = kLowest, l = 0.0f;
        int reference = -200;  // of the value scales, as an exponent
        bool ok = mbar_wait_or_fail(smem_addr(&q_full), 0, &failed);  // all_see is final
        RingPlace<kScaleSlots> scale_at;
        if (from == 1) scale_at.next();
        bool far_maximum = false, fresh = true;  // of a row of the warp; before the first scores
        // sums of the steps before, by a row's own factor
        auto scale_sums = [&](int turn, float by) {
            if (turn == 0) return true;
            const int before = from + (turn - 1) * kEvery;  // no later product with values is issued without this step's weights
            const bool ok = mbar_wait_or_fail(smem_addr(&v_empty[before % kConverted]), (before / kConverted) & 1, &failed);
            if (!__all_sync(kFullWarp, ok)) return false;
            tcgen05_fence_after();
#pragma unroll 1
            for (int d = 0; d < D; d += 16) {
                uint32_t v[16];
                tmem_load16(tmem + lanes + Tile::o(stream) + d, v);
                tmem_load_wait(v);
#pragma unroll
                for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * by);
                tmem_store16(tmem + lanes + Tile::o(stream) + d, v);
            }
            tmem_store_wait();  // a step may come here three times: a reference and two maxima that rise
            return true;
        };
        for (int turn = 0; turn < turns; ++turn) {
            const int step = from + turn * kEvery, b = TILES == 1 ? step % 3 : stream;
            ok = ok && mbar_wait2_or_fail(smem_addr(&scale_full[scale_at.slot]), scale_at.parity, smem_addr(&s_full[b]),
                                          (TILES == 1 ? step / 3 : step) & 1, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            tcgen05_fence_after();
            const int2 info = scale_info[scale_at.slot];
            const float *ks = reinterpret_cast<const float *>(&scale_k[scale_at.slot]);
            const int *vs = reinterpret_cast<const int *>(&scale_v[scale_at.slot]);
            if (info.y != reference) {
                ok = scale_sums(turn, pow2(reference - info.y));
                if (!ok) break;
                reference = info.y;
            }
            // 32 tokens at a time; the weights lie where their scores were, first parts and second ones
            const uint32_t scores = tmem + lanes + Tile::s(b);
            const int token0 = (first + step) * kStep;
            const bool masked = info.x != 0xf || token0 + kStep > all_see;
            float step_sum = 0.0f;
#pragma unroll 1
            for (int i = 0; i < 2; ++i) {
                uint32_t part[32];
                if (copy == 1 - i) {  // the other copy's tokens
#pragma unroll
                    for (int j = 0; j < 32; ++j) part[j] = 0u;
                    tmem_store32(scores + i * 32, part);
                    continue;
                }
                const float k[2] = {fminf(fmaxf(ks[2 * i] * undo, 1.2e-38f), 3.0e38f), fminf(fmaxf(ks[2 * i + 1] * undo, 1.2e-38f), 3.0e38f)};
                const int e[2] = {vs[2 * i], vs[2 * i + 1]};
                float sum;
                auto load_scores = [&](uint32_t (&now)[32]) {
                    tmem_load32(scores + i * 32, now);
                    tmem_load_wait(now);
                    if (masked) {
#pragma unroll
                        for (int j = 0; j < 32; ++j)
                            if (token0 + i * 32 + j > limit || !((info.x >> (2 * i + (j >> 4))) & 1)) now[j] = 0xff800000u;
                    }
                };
                float2 p[16];
                for (int attempt = 0;; ++attempt) {
                    // (the first scores have no maximum to be taken from: it is found first)
                    if (attempt > 0 || !fresh) {
                        // the value scale goes into the exponent, and out of the sum again; step by step for all
                        // 32, since a warp waits for each of its instructions' operands in turn
                        const bool near = !far_maximum && min(e[0], e[1]) >= kFarScale;
                        {
                            uint32_t now[32];
                            load_scores(now);
                            if (near) {
                                const float less[2] = {static_cast<float>(e[0]) - m, static_cast<float>(e[1]) - m};
#pragma unroll
                                for (int j = 0; j < 16; ++j)
                                    p[j] = fma2(make_float2(__uint_as_float(now[2 * j]), __uint_as_float(now[2 * j + 1])),
                                                make_float2(k[j >> 3], k[j >> 3]), make_float2(less[j >> 3], less[j >> 3]));
                            } else {
                                // scores so large that a product differs from the maximum, itself rounded, by
                                // powers of two; value scales that would take the weights out of the sum
#pragma unroll
                                for (int j = 0; j < 16; ++j)  // (of pairs, a product and a sum would be made one)
                                    p[j] = make_float2(__fadd_rn(__fmul_rn(__uint_as_float(now[2 * j]), k[j >> 3]), -m),
                                                       __fadd_rn(__fmul_rn(__uint_as_float(now[2 * j + 1]), k[j >> 3]), -m));
                            }
                        }
#pragma unroll
                        for (int j = 0; j < 16; ++j) p[j] = make_float2(exp2_fast(p[j].x), exp2_fast(p[j].y));
                        float sums[2];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float2 *x = p + 8 * h;
                            const float2 t = add2(add2(add2(x[0], x[1]), add2(x[2], x[3])), add2(add2(x[4], x[5]), add2(x[6], x[7])));
                            sums[h] = t.x + t.y;
                        }
                        if (near) {
                            sum = sums[0] * pow2(-e[0]) + sums[1] * pow2(-e[1]);
                        } else {
                            sum = sums[0] + sums[1];
#pragma unroll
                            for (int j = 0; j < 16; ++j) p[j] = mul2(p[j], make_float2(pow2(e[j >> 3]), pow2(e[j >> 3])));
                        }
                        split16(p, part);
                        if (attempt == 1 || !__any_sync(kFullWarp, sum > kRaise)) break;  // once raised, a weight is at most 2
                    }
                    fresh = false;
                    // the maximum rises: the sums before, and this step's weights before, follow
                    uint32_t v[32];
                    load_scores(v);
                    const float most = fmaxf(m, fmaxf(__fmul_rn(max16(v), k[0]), __fmul_rn(max16(v + 16), k[1]))), f = exp2_fast(m - most);
                    m = most;
                    far_maximum = __any_sync(kFullWarp, fabsf(m) > kFarMaximum && m != kLowest);
                    l *= f;
                    step_sum *= f;
                    ok = scale_sums(turn, f);
                    if (!ok) break;
                    if (i > 0) {
                        tmem_store_wait();
                        tmem_load32(scores, v);
                        tmem_load_wait(v);
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            p[j] = mul2(add2(make_float2(__uint_as_float(v[j] << 16), __uint_as_float(v[j] & 0xffff0000u)),
                                             make_float2(__uint_as_float(v[16 + j] << 16), __uint_as_float(v[16 + j] & 0xffff0000u))), make_float2(f, f));
                        split16(p, v);
                        tmem_store32(scores, v);
                    }
                }
                if (!ok) break;
                step_sum += sum;
                tmem_store32(scores + i * 32, part);
            }
            if (!ok) break;
            l += step_sum;
            tmem_store_wait();
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_addr(&p_full[b]));
                mbar_arrive(smem_addr(&scale_empty[scale_at.slot]));
            }
            for (int i = 0; i < kEvery; ++i) scale_at.next();
        }
        // the sums: of both groups, each taking half of the columns, or of this one's rows
        const int lanes_row = (warp & 3) * 32 + lane;
        float4 mine = make_float4(m, l, pow2(max(reference, -126)), 0.0f), other = make_float4(kLowest, 0.0f, 0.0f, 0.0f);
        if (count > 0) ok = ok && mbar_wait_or_fail(smem_addr(&v_empty[(count - 1) % kConverted]), ((count - 1) / kConverted) & 1, &failed);
        const int other_turns = TILES == 1 ? (count - (1 - stream) + 1) / 2 : 0;
        if constexpr (TILES == 1) {
            group_sums[stream][lanes_row] = mine;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            other = group_sums[1 - stream][lanes_row];
        }
        ok = __all_sync(kFullWarp, ok);
        tcgen05_fence_after();
        const int64_t pair = (g.begin + row / a.rows) * c.n_kv_heads + head;
        const int64_t part = (pair * a.parts.splits + (copy >= 0 ? blockIdx.x * 2 + copy : blockIdx.x)) * a.rows + row % a.rows;
        const float most = fmaxf(mine.x, other.x), mine_f = exp2_fast(mine.x - most), other_f = exp2_fast(other.x - most);
        const float total = mine.y * mine_f + other.y * other_f, inverse = total == 0.0f ? 0.0f : 1.0f / total;
        if (count > 0 && ok) {
            // 32 columns at a time, turned in shared memory (the codes', which have all been converted)
            constexpr int kColumns = TILES == 1 ? D / 2 : D;
            const int d0 = TILES == 1 ? stream * kColumns : 0;
            const uint32_t stage = raw + warp * 4096;
            const unsigned all_valid = __ballot_sync(kFullWarp, row < rows);
#pragma unroll 1
            for (int d = d0; d < d0 + kColumns; d += 32) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    uint32_t v[16] = {}, w[16] = {};
                    if (turns > 0) tmem_load16(tmem + lanes + Tile::o(stream) + d + h * 16, v);
                    if (other_turns > 0) tmem_load16(tmem + lanes + Tile::o(1 - stream) + d + h * 16, w);
                    tmem_load_wait(v);
                    tmem_load_wait(w);
#pragma unroll
                    for (int j = 0; j < 16; ++j) {
                        float y = turns > 0 ? __uint_as_float(v[j]) * (mine_f * inverse) * mine.z : 0.0f;
                        if (other_turns > 0) y += __uint_as_float(w[j]) * (other_f * inverse) * other.z;
                        v[j] = __float_as_uint(y);
                    }
                    if (any_nan != 0)
#pragma unroll
                        for (int j = 0; j < 16; ++j)
                            if (nan_from[d + h * 16 + j] <= limit) v[j] = 0x7fc00000u;
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        store_shared16(stage + lane * 128 + (((h * 4 + j) ^ (lane & 7)) << 4), v[4 * j], v[4 * j + 1], v[4 * j + 2], v[4 * j + 3]);
                }
                __syncwarp();
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    const int r = k * 4 + (lane >> 3);
                    const int64_t to = __shfl_sync(kFullWarp, part, r) * D + d + (lane & 7) * 4;
                    const uint4 y = load_shared16(stage + r * 128 + (((lane & 7) ^ (r & 7)) << 4));
                    if ((all_valid >> r) & 1u) *reinterpret_cast<uint4 *>(a.parts.o + to) = y;
                }
                __syncwarp();
            }
        }
        if (row < rows && tokens > 0 && (TILES == 2 || stream == 0)) a.parts.ml[part] = make_float2(most, total);
        tcgen05_fence_before();
    }
    __syncthreads();
    if (warp == kProducts) {
        tcgen05_fence_after();
        tmem_free(tmem, kTmemColumns);
    }
}

// A block for every SM, as many stretches of a prefix as that gives, none longer than kMostSteps.  (The
// device's 148 SMs: the workspace is asked for without a device.)
struct PrefixPlan {
    int tiles, row_tiles, splits, copies, tail_splits;
};
static PrefixPlan prefix_plan(const sp_cache &c, const SharedAttention &s) {
    PrefixPlan p = {};
    const int64_t rows = s.n_q * (s.n_heads / c.n_kv_heads), all = rows * std::min(s.max_group, c.n_seqs);
    const int64_t blocks = std::min(s.max_prefix / c.block_tokens, c.table_cols), tokens = blocks * c.block_tokens;
    p.tail_splits = shared_tail_splits(c, rows, std::max(int64_t(1), s.max_len - tokens + c.block_tokens));
    if (s.n_groups == 0 || all == 0 || blocks == 0) return p;
    // A sequence alone in its group shares nothing, and its few rows leave the products' 128 idle: the
    // kernel without groups is faster with up to 8 rows (4 rows, 8000 tokens: 21 us for 28 with one (sequence,
    // kv head), 22 for 33 with 8, 30 for 86 with 64; 2 rows of 13726 tokens: 27 for 27), and with up to 16 once
    // there are enough of them (8000 tokens: 50 us for 42 with 16, 53 for 60 with 32, 100 for 149 with 128); with 32
    // rows it takes 69 for 61 with 32, 174 for 163 with 128, and twice that for 64.
    if (std::min(s.max_group, c.n_seqs) == 1 && (rows <= 8 || (rows <= 16 && c.n_seqs * c.n_kv_heads >= 32))) return p;
    p.tiles = all <= 128 ? 1 : 2;
    p.copies = all <= 64 ? 2 : 1;
    p.row_tiles = static_cast<int>((all + 128 * p.tiles - 1) / (128 * p.tiles));
    const int64_t units = s.n_groups * c.n_kv_heads * p.row_tiles, steps = (tokens + kStep - 1) / kStep;
    // Stretches that are cut for their sums' sake fill whole rounds of the device (131072 tokens, 16 units: 578 -> 520 us).
    const int64_t least = (steps + kMostSteps - 1) / kMostSteps, rounds = (units * least + 147) / 148;
    p.splits = static_cast<int>(std::max(least, std::min((steps + 1) / 2, rounds * 148 / units)));
    return p;
}

bool cache_shared_fits(const sp_cache &c, const SharedAttention &s) {
    return int64_t(prefix_plan(c, s).row_tiles) * c.n_kv_heads <= 65535;
}

int64_t cache_shared_workspace(const sp_cache &c, const SharedAttention &s) {
    const int64_t rows = s.n_q * (s.n_heads / c.n_kv_heads), pairs = c.n_seqs * c.n_kv_heads;
    if (rows == 0 || pairs == 0) return 0;
    const PrefixPlan plan = prefix_plan(c, s);
    if (plan.splits == 0 || c.n_blocks == 0) return cache_attention_workspace(c, s.n_q, s.n_heads, s.max_len, false);
    return pairs * (plan.splits * plan.copies + plan.tail_splits) * rows * (c.head_dim * 4 + 8);
}

template <bool BF16, int D, int TILES>
static cudaError_t launch_prefix(const PrefixArgs &a, const CUtensorMap &k_map, const CUtensorMap &v_map, int64_t groups,
                                 cudaStream_t stream) {
    using Tile = PrefixTile<D, TILES>;
    auto *kernel = cache_prefix_kernel<BF16, D, TILES>;
    static DynamicSmem limit;
    cudaError_t e = limit.allow(reinterpret_cast<const void *>(kernel));
    if (e != cudaSuccess) return e;
    PdlConfig pdl(dim3(a.splits, a.cache.n_kv_heads * a.row_tiles, static_cast<unsigned>(groups)), dim3(Tile::kWarps * 32), stream);
    pdl.cfg.dynamicSmemBytes = Tile::kSmem;
    return cudaLaunchKernelEx(&pdl.cfg, kernel, k_map, v_map, a);
}

sp_status launch_cache_shared(const sp_cache &c, const SharedAttention &s, void *workspace, cudaStream_t stream) {
    const PrefixPlan plan = prefix_plan(c, s);
    if (plan.splits == 0 || c.n_blocks == 0)
        return launch_cache_attention(c, s.Q, s.q, s.dtype, s.n_q, s.n_heads, s.lens, s.max_len, s.scale, s.O, s.o, s.lse, nullptr,
                                      nullptr, 0, workspace, stream);
    PrefixArgs a = {};
    a.cache = c;
    a.groups = SharedGroups{s.group_start, s.prefix, s.n_groups, s.max_prefix, s.max_group};
    a.group = s.n_heads / c.n_kv_heads;
    a.rows = static_cast<int>(s.n_q * a.group);
    a.parts.prefix_splits = plan.splits * plan.copies;
    a.parts.splits = a.parts.prefix_splits + plan.tail_splits;
    a.copies = plan.copies;
    a.parts.o = static_cast<float *>(workspace);
    a.parts.ml = reinterpret_cast<float2 *>(a.parts.o + c.n_seqs * c.n_kv_heads * a.parts.splits * a.rows * c.head_dim);
    a.Q = static_cast<const uint16_t *>(s.Q);
    a.q = s.q;
    a.lens = s.lens;
    a.n_q = s.n_q;
    a.max_len = s.max_len;
    a.row_tiles = plan.row_tiles;
    a.splits = plan.splits;
    a.block_shift = c.block_tokens == 16 ? 4 : c.block_tokens == 32 ? 5 : 6;
    a.scale_log2 = s.scale * kLog2e;
    a.q_pieces = aligned16(s.Q) && s.q.seq % 8 == 0 && s.q.token % 8 == 0 && s.q.head % 8 == 0;
    CUtensorMap k_map = {}, v_map = {};
    const int64_t pool_rows = c.n_blocks * c.n_kv_heads * c.block_tokens;
    cudaError_t e = encode_byte_rows(&k_map, c.k, pool_rows, c.head_dim, 16);
    if (e == cudaSuccess) e = encode_byte_rows(&v_map, c.v, pool_rows, c.head_dim, 16);
    if (e != cudaSuccess) return cuda_fail(e);
    const bool bf16 = s.dtype == SP_BF16, two = plan.tiles == 2;
#define SP_LAUNCH(B, DD) \
    e = two ? launch_prefix<B, DD, 2>(a, k_map, v_map, s.n_groups, stream) : launch_prefix<B, DD, 1>(a, k_map, v_map, s.n_groups, stream)
    if (bf16 && c.head_dim == 64) SP_LAUNCH(true, 64);
    else if (bf16) SP_LAUNCH(true, 128);
    else if (c.head_dim == 64) SP_LAUNCH(false, 64);
    else SP_LAUNCH(false, 128);
#undef SP_LAUNCH
    if (e != cudaSuccess) return cuda_fail(e);
    sp_status st = check_launch();
    return st == SP_OK ? launch_cache_tails(c, s, a.parts, k_map, v_map, stream) : st;
}

}  // namespace sp
