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
// Warps: four for each 128 rows (softmax), four convert, one issues products, one copies.
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

template <int D, int TILES>
struct PrefixTile {
    static constexpr int kSlots = D == 128 ? 6 : 12;           // steps of codes on their way
    static constexpr int kBuffers = TILES == 1 ? 2 : 1;        // of scores
    static constexpr int kRawBytes = 2 * kStep * D;            // keys, then values
    static constexpr int kHalfBytes = kStep * 128;             // 64 converted columns
    static constexpr int kConvBytes = D / 64 * kHalfBytes;     // keys (or values) of a step
    static constexpr int kSmem = kSlots * kRawBytes + 4 * kConvBytes;
    static constexpr int kSoftmaxWarps = 4 * TILES;
    static constexpr int kWarps = kSoftmaxWarps + 4 + 2;
    // tensor memory: of a tile
    static __device__ constexpr uint32_t q(int t) { return t * 256; }
    static __device__ constexpr uint32_t s(int t, int b) { return t * 256 + 64 + b * 64; }
    static __device__ constexpr uint32_t o(int t) { return TILES == 1 ? 256 : t * 256 + 128; }
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
    __shared__ uint64_t raw_full[kSlots], raw_empty[kSlots], k_full[2], k_empty[2], v_full[2], v_empty[2];
    __shared__ uint64_t s_full[TILES][kBuffers], p_full[TILES][kBuffers], pv_done[TILES], drained;
    __shared__ uint32_t tmem_base, failed, present[kSlots];
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
        for (int i = 0; i < 2; ++i) {
            mbar_init(smem_addr(&k_full[i]), 4);
            mbar_init(smem_addr(&v_full[i]), 4);
            mbar_init(smem_addr(&k_empty[i]), 1);
            mbar_init(smem_addr(&v_empty[i]), 1);
        }
        for (int t = 0; t < TILES; ++t) {
            for (int b = 0; b < kBuffers; ++b) {
                mbar_init(smem_addr(&s_full[t][b]), 1);
                mbar_init(smem_addr(&p_full[t][b]), 4);
            }
            mbar_init(smem_addr(&pv_done[t]), 1);
        }
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
    const int tile = warp >> 2, row = row0 + (warp >> 2) * 128 + (warp & 3) * 32 + lane;
    const uint32_t lanes = static_cast<uint32_t>((warp & 3) * 32) << 16;
    int limit = -1;        // the last token that it sees
    float undo = a.scale_log2;
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
    tcgen05_fence_before();
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t tmem = tmem_base;
    if (warp < kSoftmaxWarps) {
#pragma unroll
        for (int i = 0; i < D / 64; ++i) tmem_store32(tmem + lanes + Tile::q(tile) + i * 32, *reinterpret_cast<uint32_t(*)[32]>(&q[i * 8]));
        tmem_store_wait();
        tcgen05_fence_before();
    }
    __syncthreads();
    tcgen05_fence_after();
    const uint32_t raw = smem_addr(smem), conv = raw + kSlots * Tile::kRawBytes;  // conv: K, K, V, V

    if (warp == kSoftmaxWarps + 5) {
        // ---- copies: a lane a block of the cache
        const int blocks = kStep >> shift;  // of a step: 4, 2 or 1
        const uint32_t piece = static_cast<uint32_t>(D) << shift;
        RingPlace<kSlots> at;
        bool ok = true;
        int id = lane < blocks ? block_at(first * kStep + (lane << shift)) : -1, issued = 0;
        for (int step = 0; step < count; ++step, at.next()) {
            if (step >= kSlots) ok = mbar_wait_or_fail(smem_addr(&raw_empty[at.slot]), at.parity ^ 1u, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            const unsigned here = __ballot_sync(kFullWarp, id >= 0);
            const uint32_t bar = smem_addr(&raw_full[at.slot]), to = raw + at.slot * Tile::kRawBytes + lane * piece;
            if (lane == 0) {
                present[at.slot] = here;
                mbar_expect_tx(bar, 2 * piece * __popc(here));
            }
            __syncwarp();
            if (id >= 0) {
                const int y = (id * c.n_kv_heads + head) << shift;
                tma_load_2d(to, &k_map, 0, y, bar);
                tma_load_2d(to + kStep * D, &v_map, 0, y, bar);
            }
            issued = step + 1;
            id = lane < blocks && step + 1 < count ? block_at((first + step + 1) * kStep + (lane << shift)) : -1;
            __syncwarp();
        }
        if (failed != 0u && lane == 0)
            for (int s = max(0, issued - kSlots); s < issued; ++s) mbar_wait(smem_addr(&raw_full[s % kSlots]), (s / kSlots) & 1);
    } else if (warp == kSoftmaxWarps + 4) {
        // ---- products
        if (elect_one()) {
            const uint32_t qk = f16_instruction(kStep, BF16), pv = f16_instruction(D, true) | kColumnsB;
            auto scores = [&](int t, int step) {
                const int b = step % kBuffers;
                const uint64_t k = desc_rows128(conv + (step & 1) * Tile::kConvBytes);
#pragma unroll
                for (int p = 0; p < D / 16; ++p)
                    mma_16bit(tmem + Tile::s(t, b), tmem + Tile::q(t) + p * 8, k + (p >> 2) * (Tile::kHalfBytes / 16) + (p & 3) * 2, qk, p > 0);
                tcgen05_commit(smem_addr(&s_full[t][b]));
            };
            bool ok = true;
            for (int step = 0; ok && step < min(count, kBuffers); ++step) {
                ok = mbar_wait_or_fail(smem_addr(&k_full[step & 1]), 0, &failed);
                if (!ok) break;
                tcgen05_fence_after();
                for (int t = 0; t < TILES; ++t) scores(t, step);
                tcgen05_commit(smem_addr(&k_empty[step & 1]));
            }
            for (int step = 0; ok && step < count; ++step) {
                const int b = step % kBuffers, next = step + kBuffers;
                ok = mbar_wait_or_fail(smem_addr(&v_full[step & 1]), (step >> 1) & 1, &failed);
                if (ok && next < count) ok = mbar_wait_or_fail(smem_addr(&k_full[next & 1]), (next >> 1) & 1, &failed);
                if (!ok) break;
                const uint64_t v = desc_columns128(conv + (2 + (step & 1)) * Tile::kConvBytes, Tile::kHalfBytes);
                for (int t = 0; t < TILES; ++t) {
                    ok = mbar_wait_or_fail(smem_addr(&p_full[t][b]), (step / kBuffers) & 1, &failed);
                    if (!ok) break;
                    tcgen05_fence_after();
                    // two parts of P, 64 tokens each
#pragma unroll
                    for (int p = 0; p < 8; ++p)
                        mma_16bit(tmem + Tile::o(t), tmem + Tile::s(t, b) + p * 8, v + (p & 3) * (16 * 128 / 16), pv, step > 0 || p > 0);
                    tcgen05_commit(smem_addr(&pv_done[t]));
                    if (t == TILES - 1) tcgen05_commit(smem_addr(&v_empty[step & 1]));
                    if (next < count) scores(t, next);
                }
                if (ok && next < count) tcgen05_commit(smem_addr(&k_empty[next & 1]));
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
            const int buffer = step & 1;
            if (ok && step >= 2) ok = mbar_wait_or_fail(smem_addr(&k_empty[buffer]), ((step >> 1) - 1) & 1, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            const uint32_t from = raw + at.slot * Tile::kRawBytes, here = present[at.slot];
            const int token0 = (first + step) * kStep;
            const bool checked = token0 + kStep > all_see;  // some rows do not see all of it
            auto convert = [&](auto is_key) {
                constexpr bool KEY = decltype(is_key)::value;
                const uint32_t src = from + (KEY ? 0 : kStep * D), dst = conv + (KEY ? buffer : 2 + buffer) * Tile::kConvBytes;
#pragma unroll
                for (int i = 0; i < kStep * kChunks / 128; ++i) {
                    const int x = i * 128 + thread;
                    // eight lanes: a row's chunks (D = 64: of two rows)
                    const int r = x / kChunks, ch = x % kChunks;
                    const int swap = D == 128 ? r & 7 : (r >> 1) & 3;
                    uint4 w = load_shared16(src + r * D + ((ch ^ swap) << 4));
                    if constexpr (!KEY) {
                        if (!((here >> (r >> shift)) & 1u)) {
                            w = make_uint4(0u, 0u, 0u, 0u);
                        } else if (checked) {
                            uint32_t *word = reinterpret_cast<uint32_t *>(&w);
#pragma unroll
                            for (int k = 0; k < 16; ++k)
                                if (((word[k >> 2] >> (8 * (k & 3))) & 0x7fu) == 0x7fu) {
                                    atomicMin(&nan_from[ch * 16 + k], token0 + r);
                                    word[k >> 2] &= ~(0xffu << (8 * (k & 3)));
                                }
                        }
                    }
                    const uint2 a0 = convert4<KEY ? BF16 : true>(w.x), a1 = convert4<KEY ? BF16 : true>(w.y);
                    const uint2 a2 = convert4<KEY ? BF16 : true>(w.z), a3 = convert4<KEY ? BF16 : true>(w.w);
                    const uint32_t to = dst + (ch >> 2) * Tile::kHalfBytes + r * 128, c0 = (ch & 3) * 2;
                    store_shared16(to + ((c0 ^ (r & 7)) << 4), a0.x, a0.y, a1.x, a1.y);
                    store_shared16(to + (((c0 + 1) ^ (r & 7)) << 4), a2.x, a2.y, a3.x, a3.y);
                }
            };
            convert(std::true_type{});
            fence_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&k_full[buffer]));
            if (step >= 2) ok = mbar_wait_or_fail(smem_addr(&v_empty[buffer]), ((step >> 1) - 1) & 1, &failed);
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
        // ---- softmax: a thread a row
        float m = kLowest, l = 0.0f;
        int reference = -200;  // of the value scales, as an exponent
        bool ok = true;
        // scales of a step: lanes 0 .. 3 hold those of its 16-token pieces
        auto piece_block = [&](int step) { return lane < 4 && step < count ? block_at((first + step) * kStep + lane * 16) : -1; };
        auto scale_of = [&](const float *scales, int id) { return id >= 0 ? scales[int64_t(id) * c.n_kv_heads + head] : 0.0f; };
        int id = piece_block(0), next_id = piece_block(1);
        float ks = scale_of(c.k_scale, id), vs = scale_of(c.v_scale, id);
        for (int step = 0; step < count; ++step) {
            const int b = step % kBuffers;
            const unsigned here = __ballot_sync(kFullWarp, id >= 0) & 0xfu;
            const float ks_now = ks, vs_now = vs;
            id = next_id;
            ks = scale_of(c.k_scale, id);
            vs = scale_of(c.v_scale, id);
            next_id = piece_block(step + 2);
            // the largest value scale among the pieces that are there
            int e = lane < 4 && ((here >> lane) & 1u) ? exponent_of(vs_now) : -200;
            e = max(e, __shfl_xor_sync(kFullWarp, e, 1));
            e = max(e, __shfl_xor_sync(kFullWarp, e, 2));
            e = __shfl_sync(kFullWarp, e, 0);
            float kf[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) kf[i] = fminf(__shfl_sync(kFullWarp, ks_now, i) * undo, 3.0e38f);
            ok = mbar_wait_or_fail(smem_addr(&s_full[tile][b]), (step / kBuffers) & 1, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            tcgen05_fence_after();
            uint32_t raw_s[2][32];
            tmem_load32(tmem + lanes + Tile::s(tile, b), raw_s[0]);
            tmem_load32(tmem + lanes + Tile::s(tile, b) + 32, raw_s[1]);
            tmem_load_wait();
            float s[64];
            const int token0 = (first + step) * kStep;
#pragma unroll
            for (int j = 0; j < 64; ++j) s[j] = __uint_as_float(raw_s[j >> 5][j & 31]) * kf[j >> 4];
            if (here != 0xfu || token0 + kStep > all_see) {
#pragma unroll
                for (int j = 0; j < 64; ++j)
                    if (token0 + j > limit || !((here >> (j >> 4)) & 1u)) s[j] = -INFINITY;
            }
            float top = s[0];
#pragma unroll
            for (int j = 1; j < 64; ++j) top = fmaxf(top, s[j]);
            if (__any_sync(kFullWarp, top > m + kRaise) || e > reference + kRaiseScale) {
                const float most = fmaxf(m, top), f = exp2_fast(m - most);
                const int to = max(reference, e);
                m = most;
                l *= f;
                if (step > 0) {
                    ok = mbar_wait_or_fail(smem_addr(&pv_done[tile]), (step - 1) & 1, &failed);
                    if (!__all_sync(kFullWarp, ok)) break;
                    tcgen05_fence_after();
                    const float by = f * pow2(reference - to);
#pragma unroll 1
                    for (int d = 0; d < D; d += 32) {
                        uint32_t v[32];
                        tmem_load32(tmem + lanes + Tile::o(tile) + d, v);
                        tmem_load_wait();
#pragma unroll
                        for (int j = 0; j < 32; ++j) v[j] = __float_as_uint(__uint_as_float(v[j]) * by);
                        tmem_store32(tmem + lanes + Tile::o(tile) + d, v);
                    }
                }
                reference = to;
            }
            float vf[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {  // relative to the reference, at most 2^40
                const float scale = __shfl_sync(kFullWarp, vs_now, i);
                const int down = -reference;
                vf[i] = scale * pow2(down / 2) * pow2(down - down / 2);
            }
            uint32_t hi[32], lo[32];
            float sum0 = 0.0f, sum1 = 0.0f;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                const float p0 = exp2_fast(s[2 * j] - m), p1 = exp2_fast(s[2 * j + 1] - m);
                sum0 += p0;
                sum1 += p1;
                const float x0 = p0 * vf[j >> 3], x1 = p1 * vf[j >> 3];
                hi[j] = pack_bf16(x0, x1);
                lo[j] = pack_bf16(x0 - __uint_as_float(hi[j] << 16), x1 - __uint_as_float(hi[j] & 0xffff0000u));
            }
            l += sum0 + sum1;
            tmem_store32(tmem + lanes + Tile::s(tile, b), hi);
            tmem_store32(tmem + lanes + Tile::s(tile, b) + 32, lo);
            tmem_store_wait();
            tcgen05_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&p_full[tile][b]));
        }
        // the sums
        if (count > 0) {
            ok = ok && mbar_wait_or_fail(smem_addr(&pv_done[tile]), (count - 1) & 1, &failed);
            ok = __all_sync(kFullWarp, ok);
        }
        tcgen05_fence_after();
        const int64_t pair = (g.begin + row / a.rows) * c.n_kv_heads + head;
        const int64_t part = (pair * a.parts.splits + blockIdx.x) * a.rows + row % a.rows;
        if (count > 0 && ok) {
            const float inverse = l == 0.0f ? 0.0f : 1.0f / l, back = pow2(max(reference, -126));
#pragma unroll 1
            for (int d = 0; d < D; d += 32) {
                uint32_t v[32];
                tmem_load32(tmem + lanes + Tile::o(tile) + d, v);
                tmem_load_wait();
                if (row < rows) {
                    float4 *to = reinterpret_cast<float4 *>(a.parts.o + part * D + d);
#pragma unroll
                    for (int j = 0; j < 8; ++j) {
                        float y[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            y[k] = __uint_as_float(v[j * 4 + k]) * inverse * back;
                            if (nan_from[d + j * 4 + k] <= limit) y[k] = __uint_as_float(0x7fc00000u);
                        }
                        to[j] = make_float4(y[0], y[1], y[2], y[3]);
                    }
                }
                __syncwarp();
            }
        }
        if (row < rows && tokens > 0) a.parts.ml[part] = make_float2(m, l);
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
