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
// and nothing crosses lanes.  The maximum is raised only when a score exceeds it by more than 2^8.
//
// Two groups of four softmax warps, each with sums of its own, hide one another's latency: with 256
// rows each has 128 of them, with 128 they take the steps in turn and their sums are joined at the end.
// Four warps convert, one issues products, one copies.
#include <algorithm>

#include "cache_common.cuh"
#include "sp_tcgen05.cuh"

namespace sp {

namespace {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.4028234663852886e38f;
constexpr float kRaise = 8.0f;       // how far (in powers of two) a score may exceed the maximum
constexpr int kRaiseScale = 40;      // how far a value scale may exceed its reference
constexpr int kStep = 64;            // tokens
constexpr int kTmemColumns = 512;
constexpr int kConverted = 3;        // steps of converted keys, and of values

template <int D, int TILES>
struct PrefixTile {
    static constexpr int kSlots = D == 128 ? 4 : 10;           // steps of codes on their way
    static constexpr int kBuffers = TILES == 1 ? 3 : 2;        // of scores
    static constexpr int kRawBytes = 2 * kStep * D;            // keys, then values
    static constexpr int kHalfBytes = kStep * 128;             // 64 converted columns
    static constexpr int kConvBytes = D / 64 * kHalfBytes;     // keys (or values) of a step
    static constexpr int kSmem = kSlots * kRawBytes + 2 * kConverted * kConvBytes;
    static constexpr int kSoftmaxWarps = 8;
    static constexpr int kWarps = kSoftmaxWarps + 4 + 2;
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
    int block_shift;
    float scale_log2;
};

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// Four e4m3 codes -> four 16-bit floats (exact).
template <bool BF16>
__device__ __forceinline__ uint2 convert4(uint32_t w) {
    uint2 h;
    e4m3_to_f16(w, h.x, h.y);
    if constexpr (BF16) {
        h.x = f16_to_bf16(h.x);
        h.y = f16_to_bf16(h.y);
    }
    return h;
}
// Pairs of binary32 values in one instruction.
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c) {
    float2 d;
    asm("{\n\t.reg .b64 a, b, c;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\tmov.b64 c, {%6, %7};\n\t"
        "fma.rn.f32x2 c, a, b, c;\n\tmov.b64 {%0, %1}, c;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "mul.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
    float2 d;
    asm("{\n\t.reg .b64 a, b;\n\tmov.b64 a, {%2, %3};\n\tmov.b64 b, {%4, %5};\n\t"
        "add.rn.f32x2 a, a, b;\n\tmov.b64 {%0, %1}, a;\n\t}"
        : "=f"(d.x), "=f"(d.y) : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y));
    return d;
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
    __shared__ uint64_t s_full[kBuffers], p_full[kBuffers], pv_done[2], drained;
    __shared__ uint32_t tmem_base, failed, present[kSlots];
    __shared__ float4 group_sums[2][128];  // TILES == 1: maximum, sum, 2^reference of a group's rows
    __shared__ int all_see, nan_from[D];
    const sp_cache &c = a.cache;
    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    const int head = blockIdx.y / a.row_tiles, row0 = blockIdx.y % a.row_tiles * (128 * TILES);
    if (threadIdx.x == 0) {
        tma_prefetch_map(&k_map);
        tma_prefetch_map(&v_map);
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(smem_addr(&raw_full[i]), 1);
            mbar_init(smem_addr(&raw_empty[i]), 4);
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
        mbar_init(smem_addr(&pv_done[0]), 1);
        mbar_init(smem_addr(&pv_done[1]), 1);
        mbar_init(smem_addr(&drained), 1);
        failed = 0u;
        all_see = 0x7fffffff;
        mbar_fence_init();
    }
    for (int d = threadIdx.x; d < D; d += Tile::kWarps * 32) nan_from[d] = 0x7fffffff;
    if (warp == kSoftmaxWarps + 4) tmem_alloc(&tmem_base, kTmemColumns);
    pdl_wait();
    pdl_launch_dependents();  // the kernel over the tails counts on what came before this one

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

    // the row of this thread: its place, and its queries
    const int stream = warp >> 2, tile = TILES == 1 ? 0 : stream, row = row0 + tile * 128 + (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    int limit = -1;        // the last token that it sees
    float undo = fabsf(a.scale_log2);  // its sign goes to the queries: factors of scores are positive
    uint4 q[D / 8];
    if (warp < kSoftmaxWarps) {
#pragma unroll
        for (int i = 0; i < D / 8; ++i) q[i] = make_uint4(0u, 0u, 0u, 0u);
        if (row < rows) {
            const int64_t seq = g.begin + row / a.rows, i = row % a.rows / a.group;
            limit = static_cast<int>(max(int64_t(-1), min(min(a.lens[seq] - a.n_q + i, min(int64_t(a.lens[seq]), a.max_len) - 1), int64_t(tokens))));
            atomicMin(&all_see, limit + 1);
            const uint16_t *from = a.Q + seq * a.q.seq + i * a.q.token + (head * a.group + row % a.group) * a.q.head;
            if ((reinterpret_cast<uintptr_t>(from) & 15u) == 0) {
#pragma unroll
                for (int i = 0; i < D / 8; ++i) q[i] = *reinterpret_cast<const uint4 *>(from + i * 8);
            } else {
#pragma unroll
                for (int i = 0; i < D / 8; ++i) {
                    uint32_t w[4];
#pragma unroll
                    for (int k = 0; k < 4; ++k) w[k] = from[i * 8 + 2 * k] | uint32_t(from[i * 8 + 2 * k + 1]) << 16;
                    q[i] = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
        }
        if constexpr (BF16) {
            // sums of products with codes up to 448 stay in binary32's range
            uint32_t top = 0;
            uint32_t *w = reinterpret_cast<uint32_t *>(q);
#pragma unroll
            for (int i = 0; i < D / 2; ++i) {
                const uint32_t lo = (w[i] << 16) & 0x7fffffffu, hi = w[i] & 0x7fff0000u;
                top = max(top, max(lo < 0x7f800000u ? lo : 0u, hi < 0x7f800000u ? hi : 0u));
            }
            if (top > kLargeQuery) {
                undo *= pow2(64);
#pragma unroll
                for (int i = 0; i < D / 2; ++i) {
                    const float2 v = unpack2<true>(w[i]);
                    w[i] = pack_bf16(v.x * pow2(-64), v.y * pow2(-64));
                }
            }
        }
    }
    if (a.scale_log2 < 0.0f)
#pragma unroll
        for (int i = 0; i < D / 8; ++i) q[i] = make_uint4(q[i].x ^ 0x80008000u, q[i].y ^ 0x80008000u, q[i].z ^ 0x80008000u, q[i].w ^ 0x80008000u);
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base;
    if (warp < 4 * TILES) {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) tmem_store32(tmem + lanes + Tile::q(tile) + i * 32, *reinterpret_cast<uint32_t(*)[32]>(&q[i * 8]));
        tmem_store_wait();
        tcgen05_fence_before();
    }
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t raw = smem_addr(smem), conv = raw + kSlots * Tile::kRawBytes;  // conv: keys, then values

    if (warp == kSoftmaxWarps + 5) {
        // ---- copies: a lane a block of the cache.  A load of the table takes longer than a step, so the
        // lanes hold the blocks of several steps, and those of the next ones are on their way
        const int blocks = kStep >> shift, held = 32 / blocks;  // of a step: 4, 2 or 1
        const uint32_t piece = static_cast<uint32_t>(D) << shift;
        RingPlace<kSlots> at;
        bool ok = true;
        auto blocks_from = [&](int step) {
            const int mine = step + lane / blocks;
            return mine < count ? block_at((first + mine) * kStep + (lane % blocks << shift)) : -1;
        };
        int ids = blocks_from(0), next_ids = blocks_from(held), issued = 0;
        for (int step = 0; step < count; ++step, at.next()) {
            const int turn = step % held;
            if (step > 0 && turn == 0) {
                ids = next_ids;
                next_ids = blocks_from(step + held);
            }
            const int id = __shfl_sync(kFullWarp, ids, turn * blocks + lane % blocks);
            const bool mine = lane < blocks && id >= 0;
            if (step >= kSlots) ok = mbar_wait_or_fail(smem_addr(&raw_empty[at.slot]), at.parity ^ 1u, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            const unsigned here = __ballot_sync(kFullWarp, mine);
            const uint32_t bar = smem_addr(&raw_full[at.slot]), to = raw + at.slot * Tile::kRawBytes + lane * piece;
            if (lane == 0) {
                present[at.slot] = here;
                mbar_expect_tx(bar, 2 * piece * __popc(here));
            }
            __syncwarp();
            if (mine) {
                const int y = (id * c.n_kv_heads + head) << shift;
                tma_load_2d(to, &k_map, 0, y, bar);
                tma_load_2d(to + kStep * D, &v_map, 0, y, bar);
            }
            issued = step + 1;
            __syncwarp();
        }
        if (failed != 0u && lane == 0)
            for (int s = max(0, issued - kSlots); s < issued; ++s) mbar_wait(smem_addr(&raw_full[s % kSlots]), (s / kSlots) & 1);
    } else if (warp == kSoftmaxWarps + 4) {
        // ---- products
        if (elect_one()) {
            const uint32_t qk = f16_instruction(kStep, BF16), pv = f16_instruction(D, true) | kColumnsB;
            // Whichever product has its operands goes next; products run in the order of their issue.  A
            // step's scores go where the weights of three steps before (of the step before) were.
            constexpr int kAhead = TILES == 1 ? 3 : 1;
            int scored[TILES] = {}, weighed[TILES] = {};
            auto ready = [&](uint64_t *bar, int use) { return mbar_test(smem_addr(bar), use & 1); };
            for (uint32_t idle = 0; weighed[0] < count || weighed[TILES - 1] < count;) {
                bool issued = false;
#pragma unroll
                for (int t = 0; t < TILES; ++t) {
                    const int v = weighed[t], v_at = v % kConverted, p_at = TILES == 1 ? v % 3 : t;
                    if (v < scored[t] && ready(&p_full[p_at], TILES == 1 ? v / 3 : v) && ready(&v_full[v_at], v / kConverted)) {
                        tcgen05_fence_after();
                        const int g = TILES == 1 ? v & 1 : t;
                        const uint64_t values = desc_columns128(conv + (kConverted + v_at) * Tile::kConvBytes, Tile::kHalfBytes);
#pragma unroll
                        for (int p = 0; p < 8; ++p)  // two parts of P, 64 tokens each
                            mma_16bit(tmem + Tile::o(g), tmem + Tile::s(p_at) + p * 8, values + (p & 3) * (16 * 128 / 16), pv,
                                      v >= (TILES == 1 ? 2 : 1) || p > 0);
                        tcgen05_commit(smem_addr(&pv_done[g]));
                        ++weighed[t];
                        if (TILES == 1 || weighed[1 - t] > v) tcgen05_commit(smem_addr(&v_empty[v_at]));
                        issued = true;
                    }
                    const int k = scored[t], k_at = k % kConverted, s_at = TILES == 1 ? k % 3 : t;
                    if (k < count && k - weighed[t] < kAhead && ready(&k_full[k_at], k / kConverted)) {
                        tcgen05_fence_after();
                        const uint64_t keys = desc_rows128(conv + k_at * Tile::kConvBytes);
#pragma unroll
                        for (int p = 0; p < D / 16; ++p)
                            mma_16bit(tmem + Tile::s(s_at), tmem + Tile::q(t) + p * 8, keys + (p >> 2) * (Tile::kHalfBytes / 16) + (p & 3) * 2, qk, p > 0);
                        tcgen05_commit(smem_addr(&s_full[s_at]));
                        ++scored[t];
                        if (TILES == 1 || scored[1 - t] > k) tcgen05_commit(smem_addr(&k_empty[k_at]));
                        issued = true;
                    }
                }
                idle = issued ? 0 : idle + 1;
                if (idle > kWaitLimit) mbar_give_up(&failed);
                if (idle != 0 && *static_cast<volatile uint32_t *>(&failed) != 0u) break;
            }
        }
        __syncwarp();
        if (failed != 0u) {
            if (elect_one()) tcgen05_commit(smem_addr(&drained));
            __syncwarp();
            if (lane == 0) mbar_wait(smem_addr(&drained), 0);
        }
    } else if (warp >= kSoftmaxWarps) {
        // ---- conversion: a thread 16 codes at a time
        const int thread = threadIdx.x - kSoftmaxWarps * 32;
        constexpr int kChunks = D / 16;
        RingPlace<kSlots> at;
        bool ok = true;
        for (int step = 0; step < count; ++step, at.next()) {
            ok = mbar_wait_or_fail(smem_addr(&raw_full[at.slot]), at.parity, &failed);
            const int buffer = step % kConverted, uses = step / kConverted;
            if (ok && uses > 0) ok = mbar_wait_or_fail(smem_addr(&k_empty[buffer]), (uses - 1) & 1, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            const uint32_t from = raw + at.slot * Tile::kRawBytes, here = present[at.slot];
            const int token0 = (first + step) * kStep;
            const bool checked = token0 + kStep > all_see;  // some rows do not see all of it
            auto convert = [&](auto is_key) {
                constexpr bool KEY = decltype(is_key)::value;
                const uint32_t src = from + (KEY ? 0 : kStep * D), dst = conv + (KEY ? buffer : kConverted + buffer) * Tile::kConvBytes;
                constexpr int kEach = kStep * kChunks / 128;
                uint4 w[kEach];
                // eight lanes: a row's chunks (D = 64: of two rows)
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const int x = i * 128 + thread, r = x / kChunks, ch = x % kChunks;
                    const int swap = D == 128 ? r & 7 : (r >> 1) & 3;
                    w[i] = load_shared16(src + r * D + ((ch ^ swap) << 4));
                }
#pragma unroll
                for (int i = 0; i < kEach; ++i) {
                    const int x = i * 128 + thread, r = x / kChunks, ch = x % kChunks;
                    if constexpr (!KEY) {
                        if (!((here >> (r >> shift)) & 1u)) {
                            w[i] = make_uint4(0u, 0u, 0u, 0u);
                        } else if (checked) {
                            uint32_t *word = reinterpret_cast<uint32_t *>(&w[i]);
#pragma unroll
                            for (int k = 0; k < 16; ++k)
                                if (((word[k >> 2] >> (8 * (k & 3))) & 0x7fu) == 0x7fu) {
                                    atomicMin(&nan_from[ch * 16 + k], token0 + r);
                                    word[k >> 2] &= ~(0xffu << (8 * (k & 3)));
                                }
                        }
                    }
                    const uint2 a0 = convert4<KEY ? BF16 : true>(w[i].x), a1 = convert4<KEY ? BF16 : true>(w[i].y);
                    const uint2 a2 = convert4<KEY ? BF16 : true>(w[i].z), a3 = convert4<KEY ? BF16 : true>(w[i].w);
                    const uint32_t to = dst + (ch >> 2) * Tile::kHalfBytes + r * 128, c0 = (ch & 3) * 2;
                    store_shared16(to + ((c0 ^ (r & 7)) << 4), a0.x, a0.y, a1.x, a1.y);
                    store_shared16(to + (((c0 + 1) ^ (r & 7)) << 4), a2.x, a2.y, a3.x, a3.y);
                }
            };
            convert(std::true_type{});
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&k_full[buffer]));
            if (uses > 0) ok = mbar_wait_or_fail(smem_addr(&v_empty[buffer]), (uses - 1) & 1, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            convert(std::false_type{});
            fence_async_smem();
            __syncwarp();
            if (lane == 0) {
                mbar_arrive(smem_addr(&v_full[buffer]));
                mbar_arrive(smem_addr(&raw_empty[at.slot]));
            }
        }
    } else {
        // ---- softmax: a thread a row, of the steps stream, stream + kEvery, ...
        constexpr int kEvery = TILES == 1 ? 2 : 1;
        const int from = TILES == 1 ? stream : 0, turns = (count - from + kEvery - 1) / kEvery;
        float m = kLowest, l = 0.0f;
        int reference = -200;  // of the value scales, as an exponent
        bool ok = true;
        // scales of a step: lanes 0 .. 3 hold those of its 16-token pieces
        auto piece_block = [&](int step) { return lane < 4 && step < count ? block_at((first + step) * kStep + lane * 16) : -1; };
        auto scale_of = [&](const float *scales, int id) { return id >= 0 ? scales[int64_t(id) * c.n_kv_heads + head] : 0.0f; };
        int id = piece_block(from), next_id = piece_block(from + kEvery);
        float ks = scale_of(c.k_scale, id), vs = scale_of(c.v_scale, id);
        for (int turn = 0; turn < turns; ++turn) {
            const int step = from + turn * kEvery, b = TILES == 1 ? step % 3 : stream;
            const unsigned here = __ballot_sync(kFullWarp, id >= 0) & 0xfu;
            const float ks_now = ks, vs_now = vs;
            id = next_id;
            ks = scale_of(c.k_scale, id);
            vs = scale_of(c.v_scale, id);
            next_id = piece_block(step + 2 * kEvery);
            // the largest value scale among the pieces that are there
            int e = lane < 4 && ((here >> lane) & 1u) ? exponent_of(vs_now) : -200;
            e = max(e, __shfl_xor_sync(kFullWarp, e, 1));
            e = max(e, __shfl_xor_sync(kFullWarp, e, 2));
            e = __shfl_sync(kFullWarp, e, 0);
            float kf[4], vf[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                kf[i] = fminf(fmaxf(__shfl_sync(kFullWarp, ks_now, i) * undo, 1.2e-38f), 3.0e38f);
                vf[i] = __shfl_sync(kFullWarp, vs_now, i);
            }
            ok = mbar_wait_or_fail(smem_addr(&s_full[b]), (TILES == 1 ? step / 3 : step) & 1, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            tcgen05_fence_after();
            uint32_t s[2][32];
            tmem_load32(tmem + lanes + Tile::s(b), s[0]);
            tmem_load32(tmem + lanes + Tile::s(b) + 32, s[1]);
            tmem_load_wait();
            const int token0 = (first + step) * kStep;
            if (here != 0xfu || token0 + kStep > all_see) {
#pragma unroll
                for (int j = 0; j < 64; ++j)
                    if (token0 + j > limit || !((here >> (j >> 4)) & 1u)) s[j >> 5][j & 31] = 0xff800000u;
            }
            const float top = fmaxf(max3(max16(s[0]) * kf[0], max16(s[0] + 16) * kf[1], max16(s[1]) * kf[2]), max16(s[1] + 16) * kf[3]);
            if (__any_sync(kFullWarp, top > m + kRaise) || e > reference + kRaiseScale) {
                const float most = fmaxf(m, top), f = exp2_fast(m - most);
                const int to = max(reference, e);
                m = most;
                l *= f;
                if (turn > 0) {
                    ok = mbar_wait_or_fail(smem_addr(&pv_done[stream]), (turn - 1) & 1, &failed);
                    if (!__all_sync(kFullWarp, ok)) break;
                    tcgen05_fence_after();
                    const float by = f * pow2(reference - to);
#pragma unroll 1
                    for (int d = 0; d < D; d += 16) {
                        uint32_t v[16];
                        tmem_load16(tmem + lanes + Tile::o(stream) + d, v);
                        tmem_load_wait();
#pragma unroll
                        for (int j = 0; j < 16; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * by);
                        tmem_store16(tmem + lanes + Tile::o(stream) + d, v);
                    }
                }
                reference = to;
            }
            // value scales relative to the reference: at most 2^40
            const float down = pow2((-reference) / 2), rest = pow2(-reference - (-reference) / 2);
            float2 sum = make_float2(0.0f, 0.0f);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float2 factor = make_float2(kf[i], kf[i]), less = make_float2(-m, -m);
                const float v = vf[i] * down * rest;
                uint32_t part[2][8];
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const uint32_t *at = &s[i >> 1][(i & 1) * 16 + 2 * j];
                    float2 p = fma2(make_float2(__uint_as_float(at[0]), __uint_as_float(at[1])), factor, less);
                    p.x = exp2_fast(p.x);
                    p.y = exp2_fast(p.y);
                    sum = add2(sum, p);
                    p = mul2(p, make_float2(v, v));
                    const uint32_t hi = pack_bf16(p.x, p.y);
                    p = fma2(make_float2(__uint_as_float(hi << 16), __uint_as_float(hi & 0xffff0000u)), make_float2(-1.0f, -1.0f), p);
                    part[0][j] = hi;
                    part[1][j] = pack_bf16(p.x, p.y);
                }
                tmem_store8(tmem + lanes + Tile::s(b) + i * 8, part[0]);
                tmem_store8(tmem + lanes + Tile::s(b) + 32 + i * 8, part[1]);
            }
            l += sum.x + sum.y;
            tmem_store_wait();
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&p_full[b]));
        }
        // the sums: of both groups, each taking half of the columns, or of this one's rows
        const int lanes_row = (warp & 3) * 32 + lane;
        float4 mine = make_float4(m, l, pow2(max(reference, -126)), 0.0f), other = make_float4(kLowest, 0.0f, 0.0f, 0.0f);
        if (turns > 0) ok = ok && mbar_wait_or_fail(smem_addr(&pv_done[stream]), (turns - 1) & 1, &failed);
        const int other_turns = TILES == 1 ? (count - (1 - stream) + 1) / 2 : 0;
        if constexpr (TILES == 1) {
            if (other_turns > 0) ok = ok && mbar_wait_or_fail(smem_addr(&pv_done[1 - stream]), (other_turns - 1) & 1, &failed);
            group_sums[stream][lanes_row] = mine;
            asm volatile("bar.sync 1, 256;" ::: "memory");
            other = group_sums[1 - stream][lanes_row];
        }
        ok = __all_sync(kFullWarp, ok);
        tcgen05_fence_after();
        const int64_t pair = (g.begin + row / a.rows) * c.n_kv_heads + head;
        const int64_t part = (pair * a.parts.splits + blockIdx.x) * a.rows + row % a.rows;
        const float most = fmaxf(mine.x, other.x), mine_f = exp2_fast(mine.x - most), other_f = exp2_fast(other.x - most);
        const float total = mine.y * mine_f + other.y * other_f, inverse = total == 0.0f ? 0.0f : 1.0f / total;
        if (count > 0 && ok) {
            constexpr int kColumns = TILES == 1 ? D / 2 : D;
            const int d0 = TILES == 1 ? stream * kColumns : 0;
#pragma unroll 1
            for (int d = d0; d < d0 + kColumns; d += 16) {
                uint32_t v[16], w[16];
                if (turns > 0) tmem_load16(tmem + lanes + Tile::o(stream) + d, v);
                if (other_turns > 0) tmem_load16(tmem + lanes + Tile::o(1 - stream) + d, w);
                tmem_load_wait();
                if (row < rows) {
                    float4 *to = reinterpret_cast<float4 *>(a.parts.o + part * D + d);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        float y[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            y[k] = turns > 0 ? __uint_as_float(v[j * 4 + k]) * (mine_f * inverse) * mine.z : 0.0f;
                            if (other_turns > 0) y[k] += __uint_as_float(w[j * 4 + k]) * (other_f * inverse) * other.z;
                            if (nan_from[d + j * 4 + k] <= limit) y[k] = __uint_as_float(0x7fc00000u);
                        }
                        to[j] = make_float4(y[0], y[1], y[2], y[3]);
                    }
                }
                __syncwarp();
            }
        }
        if (row < rows && tokens > 0 && (TILES == 2 || stream == 0)) a.parts.ml[part] = make_float2(most, total);
        tcgen05_fence_before();
    }
    __syncthreads();
    if (warp == kSoftmaxWarps + 4) {
        tcgen05_fence_after();
        tmem_free(tmem, kTmemColumns);
    }
}

// A block for every SM: as many stretches of a prefix as that gives, each of four steps at least.
// (The device's 148 SMs: the workspace is asked for without a device.)
struct PrefixPlan {
    int tiles, row_tiles, splits, tail_splits;
};
static PrefixPlan prefix_plan(const sp_cache &c, const SharedAttention &s) {
    PrefixPlan p = {};
    const int64_t rows = s.n_q * (s.n_heads / c.n_kv_heads), all = rows * std::min(s.max_group, c.n_seqs);
    const int64_t blocks = std::min(s.max_prefix / c.block_tokens, c.table_cols), tokens = blocks * c.block_tokens;
    p.tail_splits = shared_tail_splits(c, rows, std::max(int64_t(1), s.max_len - tokens + c.block_tokens));
    if (s.n_groups == 0 || all == 0 || blocks == 0) return p;
    p.tiles = all <= 128 ? 1 : 2;
    p.row_tiles = static_cast<int>((all + 128 * p.tiles - 1) / (128 * p.tiles));
    const int64_t units = s.n_groups * c.n_kv_heads * p.row_tiles, most = std::max(int64_t(1), tokens / (4 * kStep));
    p.splits = static_cast<int>(std::max(int64_t(1), std::min(most, 148 / units)));
    return p;
}

int64_t cache_shared_workspace(const sp_cache &c, const SharedAttention &s) {
    const int64_t rows = s.n_q * (s.n_heads / c.n_kv_heads), pairs = c.n_seqs * c.n_kv_heads;
    if (rows == 0 || pairs == 0) return 0;
    const PrefixPlan plan = prefix_plan(c, s);
    if (plan.splits == 0) return cache_attention_workspace(c, s.n_q, s.n_heads, s.max_len, false);
    return pairs * (plan.splits + plan.tail_splits) * rows * (c.head_dim * 4 + 8);
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
    a.parts.splits = plan.splits + plan.tail_splits;
    a.parts.prefix_splits = plan.splits;
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
    CUtensorMap k_map = {}, v_map = {};
    const int64_t pool_rows = c.n_blocks * c.n_kv_heads * c.block_tokens;
    cudaError_t e = encode_byte_rows(&k_map, c.k, pool_rows, c.head_dim, c.block_tokens);
    if (e == cudaSuccess) e = encode_byte_rows(&v_map, c.v, pool_rows, c.head_dim, c.block_tokens);
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
    return st == SP_OK ? launch_cache_tails(c, s, a.parts, stream) : st;
}

}  // namespace sp
