// Attention of a few query tokens over the 8-bit cache.
//
// Mathematics: s_j = scale * q . k_j,  o = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m) with the
// running maximum m of an online softmax, in one pass over the cache; the splits of a long cache
// are joined afterwards by the same rule.  Accumulated weights need the final maximum and sum, so
// the pass leaves the scores (4 bytes a row and token, against 2 * head_dim of cache) and they are
// turned into weights at the end.  Up to 8 splits are a cluster and finish in the kernel, through
// distributed shared memory, each block with the scores it left itself; more splits (few sequences,
// long caches), or weights summed over several tiles of rows, take a second kernel.
//
// Bound by memory: 2 * head_dim bytes per token and kv head.  The heads of a group and the query
// tokens form the rows that share a pass, 8 (or 16) at a time.  Tokens are the long side of both
// tensor-core products (m16n8k16 on binary16, to which e4m3 converts exactly), so that 8 rows
// cost no padding to 16 and no operand is rearranged:
//   S^T [16 tokens x 8 rows] = K [16 x D] Q^T: a lane takes D/4 consecutive bytes of two tokens'
//     keys - the order of the inner dimension is free as long as Q agrees - and uses them as they lie;
//   O^T [D x 8 rows] += V^T [D x 16] P^T: a lane takes D/8 consecutive bytes of four tokens'
//     values and interleaves pairs of tokens bytewise before converting; P^T is S^T transposed
//     8x8 by movmatrix.
// The block scale of K goes onto the scores and that of V onto the 16-token partial product, in
// binary32.  The cache arrives by TMA, two stages of 64 tokens ahead (128 KB in flight on an SM; the
// swizzle keeps both access patterns free of bank conflicts).  P goes into the product in two
// binary16 parts: with one, a weight is off by up to 2^-12 of itself, which outputs far smaller than
// their values show in either type.  The maximum is raised only when a score exceeds it by more than
// 2^8, which saves the reductions of nearly all steps.  P is kept relative to 2^-7 of the maximum, so
// that it reaches 2^15 and uses binary16's range, and its second part is multiplied by 2^12: together
// they hold a weight to 2^-22 of itself down to 2^-22 of the largest, and to 2^-44 of the largest
// below.  (A token with most of the attention and a value near 0 leaves an output that is made of
// small weights.)  Against one part for bf16 outputs, and two parts that ended at 2^-25 of the
// largest for f16, this costs nothing up to 4 rows, and more above: 32 x 8191 tokens of 8 heads without weights
// take 85 us with 4 rows, 98 with 8 (93), 164 with 16 (139 and 157).
#include <algorithm>

#include "cache_common.cuh"
#include "sp_tma.cuh"

namespace sp {

namespace {

constexpr int kAttnWarps = 4;
constexpr int kRing = 3;           // stages of 16 tokens for every warp
constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLowest = -3.4028234663852886e38f;  // running maximum before any score: no finite score lies below
constexpr float kLift = 7.0f;   // the reference lies this far (in powers of two) below the running maximum
constexpr float kRaise = 8.0f;  // how far a score may exceed the running maximum
constexpr float kRest = 4096.0f;  // factor of a weight's second part
constexpr float kQueryRest = 1099511627776.0f;  // 2^40, of a query's

struct AttnArgs {
    sp_cache cache;
    const uint16_t *Q;
    sp_strides q, o;
    int64_t n_q, max_len;
    int n_heads, group, rows;  // rows = n_q * group
    int row_tiles, splits, block_shift;  // block_tokens = 1 << block_shift
    const int32_t *lens;
    float scale_log2;
    uint16_t *O;
    float *lse;
    float *part_o;   // [seq, kv head, split, row, D] unnormalised, relative to part_m
    float2 *part_ml; // [seq, kv head, split, row] maximum (log2) and sum
    float *scores;   // [seq, kv head, max_len, rows], log2; nullable
    const float *acc_in;  // accumulated weights; acc_out is null where a second kernel joins the splits
    float *acc_out;
    int64_t ld_acc;
};

__device__ __forceinline__ void mma_f16(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void mma_f16_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.0f));
}
// (d0, d1) += a * (b0, b1), two multiply-adds in one instruction.
__device__ __forceinline__ void add_scaled2(float &d0, float &d1, float a, float b0, float b1) {
    asm("{\n\t.reg .b64 a, b, d;\n\t"
        "mov.b64 a, {%2, %2};\n\tmov.b64 b, {%3, %4};\n\tmov.b64 d, {%0, %1};\n\t"
        "fma.rn.f32x2 d, a, b, d;\n\t"
        "mov.b64 {%0, %1}, d;\n\t}"
        : "+f"(d0), "+f"(d1) : "f"(a), "f"(b0), "f"(b1));
}
__device__ __forceinline__ uint32_t transpose8x8(uint32_t v) {
    uint32_t r;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
    return r;
}
__device__ __forceinline__ uint32_t pack_f16(float a, float b) {
    const __half2 h = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float2 unpack_f16(uint32_t u) { return unpack2<false>(u); }

__device__ __forceinline__ float exp2_fast(float x) {  // what is below 2^-126 counts as 0
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// A row's weights are 2^(s - reference) / sum: (reference, 1 / sum), 0 where a row sees nothing.
// (Their logarithm in one number would lose the sum's bits beside a large reference.)
__device__ __forceinline__ float2 norm_of(float reference, float sum) {
    return make_float2(reference, sum == 0.0f ? 0.0f : 1.0f / sum);
}
__device__ __forceinline__ float weight(float s, float2 norm) { return exp2_fast(s - norm.x) * norm.y; }

__device__ __forceinline__ void copy_scale(uint32_t dst, const float *src) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
template <int N>
__device__ __forceinline__ void read_piece(uint32_t src, uint32_t *w) {
    if constexpr (N == 4)
        asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(src));
    else
        asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "r"(src));
}

// A peer block's value.
__device__ __forceinline__ float load_remote(const float *p, int rank) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(remote_address(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ float2 load_remote(const float2 *p, int rank) {
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(remote_address(p, rank)) : "memory");
    return v;
}

// Place of a row's query token in its sequence, at most the last cached token; < 0: sees nothing.
__device__ __forceinline__ int row_limit(const AttnArgs &a, int64_t seq, int row, int64_t len) {
    if (row >= a.rows) return -1;
    return static_cast<int>(min(int64_t(a.lens[seq]) - a.n_q + row / a.group, len - 1));
}

}  // namespace

// What a block keeps in shared memory beside the ring, for the two functions that work on it.  (Single
// variables: as members of one object they cost the loop registers, and the long decoding case 2 %.)
template <int D, int NT>
struct AttnShared {
    float (&m)[kAttnWarps][NT * 8], (&l)[kAttnWarps][NT * 8];  // of the warps
    float2 (&block_ml)[NT * 8], (&row_norm)[NT * 8];
    uint64_t (&full)[kRing], (&empty)[kRing];
    float2 (&scales)[kRing][kAttnWarps];                       // of K and V
    uint32_t (&present)[kRing][kAttnWarps];                    // whether the table names a block there
    uint32_t &failed, &queries_rest;
    int (&nan_from)[D];                                        // first token among the call's own whose value is NaN, by column
    uint2 (&query_rest)[NT][D / 16][32];                       // the queries' second parts, as the operand registers lie
};
template <int D, int NT>
__device__ __forceinline__ AttnShared<D, NT> attention_shared() {
    __shared__ float m[kAttnWarps][NT * 8], l[kAttnWarps][NT * 8];
    __shared__ float2 block_ml[NT * 8], row_norm[NT * 8];
    __shared__ uint64_t full[kRing], empty[kRing];
    __shared__ float2 scales[kRing][kAttnWarps];
    __shared__ uint32_t present[kRing][kAttnWarps];
    __shared__ uint32_t failed, queries_rest;
    __shared__ int nan_from[D];
    __shared__ uint2 query_rest[NT][D / 16][32];
    return {m, l, block_ml, row_norm, full, empty, scales, present, failed, queries_rest, nan_from, query_rest};
}

template <bool BF16, int D, int NT, bool TWICE>
__device__ __noinline__ void attention_block_rest(const CUtensorMap &k_map, const CUtensorMap &v_map, const AttnArgs &a,
                                                  int next_block);

// NT: tiles of 8 rows.  TWICE (at most 4 rows): the rows stand twice in their tile, and the second
// time take their weights' second parts, so that one product serves both parts.  REST: the queries
// have second parts as well; a block that finds so once it has started goes on in a function of its
// own, so that the ordinary loop keeps the registers (inlined, that cost it 2 %).
template <bool BF16, int D, int NT, bool TWICE, bool REST>
__device__ __forceinline__ void attention_block(const CUtensorMap &k_map, const CUtensorMap &v_map, const AttnArgs &a,
                                                int next_block) {
    constexpr int KW = D / 16;  // words of keys a lane holds of one token, inner steps of the score product
    constexpr int VW = D / 32;  // words of values a lane holds of one token
    constexpr int MT = D / 16;  // 16-wide pieces of the head in the output product
    constexpr int kStep = 2 * 16 * D;  // bytes: 16 tokens' keys, 16 tokens' values
    extern __shared__ __align__(1024) uint8_t ring[];  // [kRing][warp][kStep]; afterwards the warps' sums
    const AttnShared<D, NT> sh = attention_shared<D, NT>();
    float(*sh_o)[NT * 8][D] = reinterpret_cast<float(*)[NT * 8][D]>(ring);
    float(*block_o)[D] = sh_o[kAttnWarps];             // the block's sum of them
    auto &sh_m = sh.m, &sh_l = sh.l;
    auto &block_ml = sh.block_ml, &row_norm = sh.row_norm;
    auto &full = sh.full, &empty = sh.empty;
    auto &scales = sh.scales;
    auto &present = sh.present;
    auto &nan_from = sh.nan_from;
    auto &query_rest = sh.query_rest;
    uint32_t &failed = sh.failed, &queries_rest = sh.queries_rest;
    const sp_cache &c = a.cache;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, g = lane >> 2, t = lane & 3;
    const int64_t seq = blockIdx.z;
    const int head = blockIdx.y / a.row_tiles, row0 = blockIdx.y % a.row_tiles * NT * 8;
    const int H = c.n_kv_heads, shift = a.block_shift;
    if constexpr (!REST) {
        pdl_launch_dependents();
        for (int d = threadIdx.x; d < D; d += kAttnWarps * 32) nan_from[d] = 0x7fffffff;
        if (threadIdx.x == 0) {
            if (c.n_blocks > 0) {
                tma_prefetch_map(&k_map);
                tma_prefetch_map(&v_map);
            }
            for (int i = 0; i < kRing; ++i) {
                mbar_init(smem_addr(&full[i]), 2 * kAttnWarps);  // a step's copies: the two of TMA, and the scales
                mbar_init(smem_addr(&empty[i]), kAttnWarps);
            }
            failed = queries_rest = 0u;
            mbar_fence_init();
        }
        __syncthreads();
        pdl_wait();
    }
    const int len = static_cast<int>(max(int64_t(0), min(min(int64_t(a.lens[seq]), a.max_len), c.table_cols << shift)));
    const int own_from = a.n_q > 1 ? static_cast<int>(min(int64_t(len), max(int64_t(0), a.lens[seq] - a.n_q))) : len;
    // the tokens before this one are seen by every query
    const int all_see = static_cast<int>(max(int64_t(0), min(int64_t(len), a.lens[seq] - a.n_q + 1)));
    const int steps = (len + 15) / 16;
    const int first = static_cast<int>(int64_t(steps) * blockIdx.x / a.splits);
    const int last = static_cast<int>(int64_t(steps) * (blockIdx.x + 1) / a.splits);

    // A stage holds a step of 16 tokens for every warp.  The warps take turns in filling stages, two
    // ahead: four lanes copy a step each, scales included (4-byte copies on the same barrier).  The
    // blocks are looked up a turn before they are wanted.
    const int32_t *table = c.table + seq * c.ld_table;
    const uint32_t n_blocks = static_cast<uint32_t>(c.n_blocks), ring_at = smem_addr(ring);
    const int stages = (last - first + kAttnWarps - 1) / kAttnWarps;
    const uint64_t policy = l2_evict_first();  // leaves the L2 to the scores, which the joining kernel reads
    auto block_of = [&](int stage) {
        const int step = first + stage * kAttnWarps + lane;
        return lane < kAttnWarps && step < last ? table[step >> (shift - 4)] : -1;
    };
    auto fill = [&](int stage, int slot, int block) {
        if (lane < kAttnWarps) {
            const int step = first + stage * kAttnWarps + lane;
            const uint32_t bar = smem_addr(&full[slot]);
            const bool here = uint32_t(block) < n_blocks;
            present[slot][lane] = here;
            if (here) {
                const int tile = block * H + head;
                const uint32_t to = ring_at + (slot * kAttnWarps + lane) * kStep;
                const int row = (tile << shift) + ((step << 4) & ((1 << shift) - 1));
                mbar_expect_tx(bar, kStep);
                tma_load_2d(to, &k_map, 0, row, bar, policy);
                tma_load_2d(to + kStep / 2, &v_map, 0, row, bar, policy);
                copy_scale(smem_addr(&scales[slot][lane].x), c.k_scale + tile);
                copy_scale(smem_addr(&scales[slot][lane].y), c.v_scale + tile);
                asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(bar) : "memory");
            } else {
                mbar_arrive(bar);
                mbar_arrive(bar);
            }
        }
        __syncwarp();
    };
    // next_block: of the stage this warp fills next
    static_assert(kRing - 1 <= kAttnWarps, "the first stages are filled by different warps");
    if constexpr (!REST) {
        next_block = block_of(warp);
        if (warp < kRing - 1) {
            if (warp < stages) fill(warp, warp, next_block);
            next_block = block_of(warp + kAttnWarps);
        }
    }
    RingPlace<kRing> place;

    // queries: operand registers, and the factor that undoes their scaling
    uint32_t qf[NT][KW][2];
    float qscale[NT][2], m[NT][2], l[NT][2], o[NT][MT][4];
    int limit[NT][2];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
        const int row = row0 + n * 8 + (TWICE ? g & 3 : g);
        float undo = a.scale_log2;
        [[maybe_unused]] uint32_t rest[KW][2] = {}, any_rest = 0u;
        if (row < a.rows) {
            const uint16_t *q = a.Q + seq * a.q.seq + (row / a.group) * a.q.token +
                                (head * a.group + row % a.group) * a.q.head + t * (D / 4);
            uint32_t raw[KW][2];
#pragma unroll
            for (int s = 0; s < KW; ++s) {
                const uint16_t *at = q + s * 4;  // as the lane's words of K lie
                raw[s][0] = at[0] | (uint32_t(at[1]) << 16);
                raw[s][1] = at[2] | (uint32_t(at[3]) << 16);
            }
            if constexpr (BF16) {
                // binary16 holds a row scaled by a power of two: its largest magnitude comes to
                // [2^14, 2^15).  What lies more than 2^30 below that loses bits; what is lost, 2^40
                // times, is a second operand, which a block takes only if it has one (down to 2^70
                // below the largest)
                uint32_t top = 0;
#pragma unroll
                for (int s = 0; s < KW; ++s)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const uint32_t lo = (raw[s][i] << 16) & 0x7fffffffu, hi = raw[s][i] & 0x7fff0000u;
                        if (lo < 0x7f800000u) top = max(top, lo);
                        if (hi < 0x7f800000u) top = max(top, hi);
                    }
                const unsigned quad = 0xfu << (lane & 28);
                top = max(top, __shfl_xor_sync(quad, top, 1));
                top = max(top, __shfl_xor_sync(quad, top, 2));
                const int up = min(141 - max(static_cast<int>(top >> 23), 1), 126);
                const float f = pow2(up);
                undo *= pow2(-up);
#pragma unroll
                for (int s = 0; s < KW; ++s)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        const float2 v = unpack2<true>(raw[s][i]);
                        raw[s][i] = pack_f16(v.x * f, v.y * f);
                        const float2 h = unpack_f16(raw[s][i]);
                        // 0 for what is not finite
                        const float lo = fabsf(h.x) <= 65504.0f ? v.x * f - h.x : 0.0f, hi = fabsf(h.y) <= 65504.0f ? v.y * f - h.y : 0.0f;
                        if constexpr (REST) rest[s][i] = pack_f16(lo * kQueryRest, hi * kQueryRest);
                        else any_rest |= __float_as_uint(lo) | __float_as_uint(hi);
                    }
            }
#pragma unroll
            for (int s = 0; s < KW; ++s) {
                qf[n][s][0] = raw[s][0];
                qf[n][s][1] = raw[s][1];
            }
        } else {
#pragma unroll
            for (int s = 0; s < KW; ++s) qf[n][s][0] = qf[n][s][1] = 0u;
        }
        if constexpr (REST) {
            if (warp == 0)
#pragma unroll
                for (int s = 0; s < KW; ++s) query_rest[n][s][lane] = make_uint2(rest[s][0], rest[s][1]);
        } else if (any_rest != 0u) {
            queries_rest = 1u;
        }
        // the scores' columns are rows 2t and 2t + 1
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            qscale[n][i] = __shfl_sync(kFullWarp, undo, (2 * t + i) * 4);
            limit[n][i] = row_limit(a, seq, row0 + n * 8 + (TWICE ? (2 * t + i) & 3 : 2 * t + i), len);
            m[n][i] = kLowest;
            l[n][i] = 0.0f;
        }
#pragma unroll
        for (int k = 0; k < MT; ++k)
#pragma unroll
            for (int i = 0; i < 4; ++i) o[n][k][i] = 0.0f;
    }
    __syncthreads();
    if constexpr (BF16 && !REST) {
        if (queries_rest != 0u) {
            attention_block_rest<BF16, D, NT, TWICE>(k_map, v_map, a, next_block);
            return;
        }
    }

    // of token g, row 2t of this tile; 8-byte aligned where rows is even
    float *const scores = a.scores + ((seq * H + head) * a.max_len + g) * a.rows + row0 + 2 * t;
    for (int stage = 0; stage < stages; ++stage, place.next()) {
        const int step = first + stage * kAttnWarps + warp, j0 = step * 16, slot = place.slot;
        const int ahead = stage + kRing - 1;
        bool ok = true;
        if ((ahead & (kAttnWarps - 1)) == warp && ahead < stages) {
            // the slot was last used by the stage before this one
            const int free_slot = slot == 0 ? kRing - 1 : slot - 1;
            if (ahead >= kRing) ok = mbar_wait_or_fail(smem_addr(&empty[free_slot]), slot == 0 ? place.parity ^ 1u : place.parity, &failed);
            if (!__all_sync(kFullWarp, ok)) break;
            fill(ahead, free_slot, next_block);
            next_block = block_of(ahead + kAttnWarps);
        }
        ok = mbar_wait_or_fail(smem_addr(&full[slot]), place.parity, &failed);
        if (!__all_sync(kFullWarp, ok)) break;
        if (step >= last) break;  // only in the last stage
        if (!present[slot][warp]) {
            if (a.scores != nullptr)
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int j = j0 + g + (i >> 1) * 8, row = row0 + n * 8 + 2 * t + (i & 1);
                        if (j < len && row < a.rows)
                            a.scores[((seq * H + head) * a.max_len + j) * a.rows + row] = -INFINITY;
                    }
            __syncwarp();
            if (lane == 0) mbar_arrive(smem_addr(&empty[slot]));
            continue;
        }
        const float k_scale = scales[slot][warp].x;
        const float v_scale = scales[slot][warp].y * (TWICE && t >= 2 ? 1.0f / kRest : 1.0f);
        uint32_t kw[2][KW], vw[4][VW];
        {
            // 16-byte chunk x of row r lies at x ^ (r & 7) (128-byte rows) or x ^ (r / 2 & 3)
            const uint32_t k_at = ring_at + (slot * kAttnWarps + warp) * kStep, v_at = k_at + kStep / 2;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int r = g + 8 * i, swap = D == 128 ? r & 7 : (r >> 1) & 3;
#pragma unroll
                for (int x = 0; x < D / 64; ++x) read_piece<4>(k_at + r * D + (((t * (D / 64) + x) ^ swap) << 4), &kw[i][x * 4]);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int r = 2 * t + (i & 1) + (i >> 1) * 8, swap = D == 128 ? r & 7 : (r >> 1) & 3;
                if constexpr (D == 128) read_piece<4>(v_at + r * D + ((g ^ swap) << 4), vw[i]);
                else read_piece<2>(v_at + r * D + (((g >> 1) ^ swap) << 4) + (g & 1) * 8, vw[i]);
            }
        }
        __syncwarp();  // the step is in registers
        if (lane == 0) mbar_arrive(smem_addr(&empty[slot]));

        // scores
        float s[NT][4];
        {
            float s2[NT][2][4];
            if constexpr (REST) {
#pragma unroll
                for (int k = 0; k < KW; ++k) {
                    uint32_t f[4];
                    e4m3_to_f16(kw[0][k], f[0], f[2]);
                    e4m3_to_f16(kw[1][k], f[1], f[3]);
#pragma unroll
                    for (int n = 0; n < NT; ++n) {
                        const uint2 b = query_rest[n][k][lane];
                        if (k == 0) mma_f16_first(s2[n][0], f, b.x, b.y);
                        else mma_f16(s2[n][0], f, b.x, b.y);
                    }
                }
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i) s2[n][0][i] *= 1.0f / kQueryRest;
            }
#pragma unroll
            for (int k = 0; k < KW; ++k) {
                uint32_t f[4];
                e4m3_to_f16(kw[0][k], f[0], f[2]);
                e4m3_to_f16(kw[1][k], f[1], f[3]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    if (k < 2 && !(REST && k == 0)) mma_f16_first(s2[n][k], f, qf[n][k][0], qf[n][k][1]);
                    else mma_f16(s2[n][k & 1], f, qf[n][k][0], qf[n][k][1]);
                }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 4; ++i) s[n][i] = (s2[n][0][i] + s2[n][1][i]) * (k_scale * qscale[n][i & 1]);
            if (j0 + 16 > all_see) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (j0 + g + (i >> 1) * 8 > limit[n][i & 1]) s[n][i] = -INFINITY;
            }
            bool raise = false;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int i = 0; i < 2; ++i) raise |= fmaxf(s[n][i], s[n][i + 2]) > m[n][i] + (kLift + kRaise);
            if (a.scores != nullptr) {
                // rows 2t, 2t + 1 of tokens g and g + 8
                float *to = scores + int64_t(j0) * a.rows;
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        const int row = row0 + n * 8 + 2 * t;
                        if (j0 + g + h * 8 < len && row < a.rows) {
                            float *at = to + (h * 8) * a.rows + n * 8;
                            if ((a.rows & 1) == 0) {
                                *reinterpret_cast<float2 *>(at) = make_float2(s[n][2 * h], s[n][2 * h + 1]);
                            } else {
                                at[0] = s[n][2 * h];
                                if (row + 1 < a.rows) at[1] = s[n][2 * h + 1];
                            }
                        }
                    }
            }
            if (__any_sync(kFullWarp, raise)) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        float top = fmaxf(s[n][i], s[n][i + 2]);
                        top = fmaxf(top, __shfl_xor_sync(kFullWarp, top, 4));
                        top = fmaxf(top, __shfl_xor_sync(kFullWarp, top, 8));
                        top = fmaxf(top, __shfl_xor_sync(kFullWarp, top, 16));
                        top = fmaxf(top - kLift, m[n][i]);
                        const float f = exp2_fast(m[n][i] - top);
                        m[n][i] = top;
                        l[n][i] *= f;
#pragma unroll
                        for (int k = 0; k < MT; ++k) {
                            o[n][k][i] *= f;
                            o[n][k][i + 2] *= f;
                        }
                    }
            }
        }
        // weights, as the operand of the output product
        uint32_t ph[NT][2], pl[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
            float p[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                p[i] = exp2_fast(s[n][i] - m[n][i & 1]);
                l[n][i & 1] += p[i];
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const uint32_t hi = pack_f16(p[2 * h], p[2 * h + 1]);
                const float2 r = unpack_f16(hi);
                const uint32_t rest = pack_f16((p[2 * h] - r.x) * kRest, (p[2 * h + 1] - r.y) * kRest);
                ph[n][h] = transpose8x8(TWICE && t >= 2 ? rest : hi);
                if constexpr (!TWICE) pl[n][h] = transpose8x8(rest);
            }
        }
        // values past the end, and NaN of the call's own tokens, which some rows do not see
        if (j0 + 16 > own_from) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int j = j0 + 2 * t + (i & 1) + (i >> 1) * 8;
#pragma unroll
                for (int w = 0; w < VW; ++w) {
                    if (j >= len) vw[i][w] = 0u;
                    else if (j >= own_from) {
#pragma unroll
                        for (int k = 0; k < 4; ++k)
                            if (((vw[i][w] >> (8 * k)) & 0x7fu) == 0x7fu) {
                                atomicMin(&nan_from[g * (D / 8) + w * 4 + k], j);
                                vw[i][w] &= ~(0xffu << (8 * k));
                            }
                    }
                }
            }
            __syncwarp();
        }
#pragma unroll
        for (int w = 0; w < VW; ++w) {
#pragma unroll
            for (int half = 0; half < 2; ++half) {
                // two columns of four tokens: (column, token pair)
                const uint32_t sel = half == 0 ? 0x5140u : 0x7362u;
                uint32_t f[4];
                e4m3_to_f16(prmt(vw[0][w], vw[1][w], sel), f[0], f[1]);
                e4m3_to_f16(prmt(vw[2][w], vw[3][w], sel), f[2], f[3]);
#pragma unroll
                for (int n = 0; n < NT; ++n) {
                    float x[4];
                    mma_f16_first(x, f, ph[n][0], ph[n][1]);
                    if constexpr (!TWICE) {
                        float rest[4];
                        mma_f16_first(rest, f, pl[n][0], pl[n][1]);
                        add_scaled2(x[0], x[1], 1.0f / kRest, rest[0], rest[1]);
                        add_scaled2(x[2], x[3], 1.0f / kRest, rest[2], rest[3]);
                    }
                    float(&to)[4] = o[n][2 * w + half];
                    add_scaled2(to[0], to[1], v_scale, x[0], x[1]);
                    add_scaled2(to[2], to[3], v_scale, x[2], x[3]);
                }
            }
        }
    }

    // the warps' parts meet in shared memory (the ring's: every copy has been waited for)
    __syncthreads();
    if (failed != 0u) {  // a block that gave up still has copies in flight; no warp starts any more
        if (threadIdx.x == 0)
            for (int i = 0; i < 2 * kRing; ++i) mbar_wait(smem_addr(&full[i % kRing]), i / kRing);
        __syncthreads();
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int row = n * 8 + 2 * t + i;
            float sum = l[n][i];
            sum += __shfl_xor_sync(kFullWarp, sum, 4);
            sum += __shfl_xor_sync(kFullWarp, sum, 8);
            sum += __shfl_xor_sync(kFullWarp, sum, 16);
            if (g == 0) {
                sh_m[warp][row] = m[n][i];
                sh_l[warp][row] = sum;
            }
#pragma unroll
            for (int k = 0; k < MT; ++k) {
                sh_o[warp][row][g * (D / 8) + 2 * k] = o[n][k][i];
                sh_o[warp][row][g * (D / 8) + 2 * k + 1] = o[n][k][i + 2];
            }
        }
    __syncthreads();
    for (int at = threadIdx.x; at < NT * 8 * D; at += kAttnWarps * 32) {
        const int r = at / D, d = at % D, row = row0 + r;
        if (row >= a.rows) break;
        float top = sh_m[0][r];
#pragma unroll
        for (int w = 1; w < kAttnWarps; ++w) top = fmaxf(top, sh_m[w][r]);
        float sum = 0.0f, out = 0.0f;
#pragma unroll
        for (int w = 0; w < kAttnWarps; ++w) {
            const float f = exp2_fast(sh_m[w][r] - top);
            sum = fmaf(f, sh_l[w][r], sum);
            out = fmaf(f, TWICE ? sh_o[w][r][d] + sh_o[w][r + 4][d] : sh_o[w][r][d], out);
        }
        if (nan_from[d] <= row_limit(a, seq, row, len)) out = __uint_as_float(0x7fc00000u);
        if (a.part_o != nullptr) {
            const int64_t p = ((seq * H + head) * a.splits + blockIdx.x) * a.rows + row;
            a.part_o[p * D + d] = out;
            if (d == 0) a.part_ml[p] = make_float2(top, sum);
        } else {
            block_o[r][d] = out;
            if (d == 0) block_ml[r] = make_float2(top, sum);
        }
    }
    if (a.part_o != nullptr) return;

    // the cluster's blocks share the output's elements
    const int ranks = a.splits, rank = blockIdx.x;
    if (ranks > 1) cluster_sync();
    else __syncthreads();
    const int share = NT * 8 * D / ranks;
    for (int at = rank * share + threadIdx.x; at < (rank + 1) * share; at += kAttnWarps * 32) {
        const int r = at / D, d = at % D, row = row0 + r;
        if (row >= a.rows) break;
        float top = kLowest, sum = 0.0f, out = 0.0f;
        for (int k = 0; k < ranks; ++k) {
            const float2 ml = load_remote(&block_ml[r], k);
            const float v = load_remote(&block_o[r][d], k), most = fmaxf(top, ml.x);
            const float f = exp2_fast(top - most), h = exp2_fast(ml.x - most);
            sum = fmaf(sum, f, ml.y * h);
            out = fmaf(out, f, v * h);
            top = most;
        }
        const int i = row / a.group, hq = head * a.group + row % a.group;
        const float y = sum == 0.0f ? 0.0f : out / sum;
        uint16_t bits;
        if constexpr (BF16) bits = __bfloat16_as_ushort(__float2bfloat16_rn(y));
        else bits = __half_as_ushort(__float2half_rn(y));
        a.O[seq * a.o.seq + i * a.o.token + hq * a.o.head + d] = bits;
        if (d == 0 && a.lse != nullptr) a.lse[(seq * a.n_q + i) * a.n_heads + hq] = (top + log2f(sum)) * 0.6931471805599453f;
    }
    if (a.acc_out != nullptr) {
        if (threadIdx.x < NT * 8) {
            float top = kLowest, sum = 0.0f;
            for (int k = 0; k < ranks; ++k) {
                const float2 ml = load_remote(&block_ml[threadIdx.x], k);
                const float most = fmaxf(top, ml.x);
                sum = fmaf(sum, exp2_fast(top - most), ml.y * exp2_fast(ml.x - most));
                top = most;
            }
            row_norm[threadIdx.x] = norm_of(top, sum);
        }
        __syncthreads();
        const int64_t pair = seq * H + head;
        const int own = static_cast<int>(max(int64_t(-1), min(a.lens[seq] - a.n_q, a.max_len)));
        const int end = min(last * 16, len);
        for (int j = first * 16 + threadIdx.x; j < end; j += kAttnWarps * 32) {
            const float *x = a.scores + (pair * a.max_len + j) * a.rows;
            float sum = a.acc_in != nullptr && j < own ? a.acc_in[pair * a.ld_acc + j] : 0.0f, add = 0.0f;
            if ((a.rows & 3) == 0) {
                for (int r = 0; r < a.rows; r += 4) {
                    const float4 v = *reinterpret_cast<const float4 *>(x + r);
                    add += weight(v.x, row_norm[r]) + weight(v.y, row_norm[r + 1]) + weight(v.z, row_norm[r + 2]) +
                           weight(v.w, row_norm[r + 3]);
                }
            } else {
                for (int r = 0; r < a.rows; ++r) add += weight(x[r], row_norm[r]);
            }
            a.acc_out[pair * a.ld_acc + j] = sum + add;
        }
        for (int64_t j = len + rank * (kAttnWarps * 32) + threadIdx.x; j < a.max_len; j += ranks * kAttnWarps * 32)
            a.acc_out[pair * a.ld_acc + j] = 0.0f;
    }
    if (ranks > 1) cluster_sync();  // no block leaves while its sums are read
}

template <bool BF16, int D, int NT, bool TWICE>
__device__ __noinline__ void attention_block_rest(const CUtensorMap &k_map, const CUtensorMap &v_map, const AttnArgs &a,
                                                  int next_block) {
    attention_block<BF16, D, NT, TWICE, true>(k_map, v_map, a, next_block);
}

template <bool BF16, int D, int NT, bool TWICE>
__global__ void __launch_bounds__(kAttnWarps * 32, NT == 1 ? 4 : 2)
cache_attention_kernel(const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                       const __grid_constant__ AttnArgs a) {
    attention_block<BF16, D, NT, TWICE, false>(k_map, v_map, a, 0);
}

// Joins the splits; turns the scores into accumulated weights.  Block x of a (sequence, kv head)
// takes the rows x, x + gridDim.x, ... of the output and the x-th stretch of kJoinTokens tokens.
// ROWS: rows where they are 1, 2, 4 or 8 (a token's scores are one load), else 0.
constexpr int kJoinThreads = 256, kJoinEach = 4, kJoinTokens = kJoinThreads * kJoinEach;

template <bool BF16, int ROWS>
__global__ void __launch_bounds__(kJoinThreads)
cache_join_kernel(const AttnArgs a, const float *acc_in, float *acc_out, int64_t ld_acc) {
    extern __shared__ float2 join_norm[];
    const sp_cache &c = a.cache;
    const int H = c.n_kv_heads, D = c.head_dim, head = blockIdx.y;
    const int64_t seq = blockIdx.z, pair = seq * H + head;
    const int rows = ROWS != 0 ? ROWS : a.rows;
    pdl_launch_dependents();
    pdl_wait();
    const float2 *ml = a.part_ml + pair * a.splits * rows;
    const float *part = a.part_o + pair * a.splits * rows * D;
    const int j0 = blockIdx.x * kJoinTokens + threadIdx.x;
    if (acc_out != nullptr && int64_t(blockIdx.x) * kJoinTokens < a.max_len) {
        const int len = static_cast<int>(max(int64_t(0), min(min(int64_t(a.lens[seq]), a.max_len), c.table_cols * c.block_tokens)));
        const int own = static_cast<int>(max(int64_t(-1), min(a.lens[seq] - a.n_q, a.max_len)));
        // the scores and the old sums are on their way before the rows' sums are joined
        float s[kJoinEach][ROWS != 0 ? ROWS : 1], sum[kJoinEach];
        const float *scores = a.scores + (pair * a.max_len + j0) * rows;
#pragma unroll
        for (int i = 0; i < kJoinEach; ++i) {
            const int j = j0 + i * kJoinThreads;
            sum[i] = acc_in != nullptr && j < own ? acc_in[pair * ld_acc + j] : 0.0f;
            if constexpr (ROWS != 0) {
                const float *at = scores + int64_t(i) * kJoinThreads * ROWS;
                if (j >= len) {
#pragma unroll
                    for (int r = 0; r < ROWS; ++r) s[i][r] = -INFINITY;
                } else if constexpr (ROWS == 1) {
                    s[i][0] = __ldcs(at);
                } else if constexpr (ROWS == 2) {
                    const float2 v = __ldcs(reinterpret_cast<const float2 *>(at));
                    s[i][0] = v.x; s[i][1] = v.y;
                } else {
#pragma unroll
                    for (int r = 0; r < ROWS; r += 4) {
                        const float4 v = __ldcs(reinterpret_cast<const float4 *>(at + r));
                        s[i][r] = v.x; s[i][r + 1] = v.y; s[i][r + 2] = v.z; s[i][r + 3] = v.w;
                    }
                }
            }
        }
        // a warp joins a row, a lane reads a split
        const int lane = threadIdx.x & 31;
        for (int row = threadIdx.x >> 5; row < rows; row += kJoinThreads / 32) {
            float top = -INFINITY, total = 0.0f;
            for (int k0 = 0; k0 < a.splits; k0 += 32) {
                const float2 v = k0 + lane < a.splits ? ml[(k0 + lane) * rows + row] : make_float2(-INFINITY, 0.0f);
                float most = v.x;
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) most = fmaxf(most, __shfl_xor_sync(kFullWarp, most, o));
                most = fmaxf(most, top);
                float part_sum = v.y * exp2_fast(v.x - most);
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) part_sum += __shfl_xor_sync(kFullWarp, part_sum, o);
                total = fmaf(total, exp2_fast(top - most), part_sum);
                top = most;
            }
            if (lane == 0) join_norm[row] = norm_of(top, total);
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kJoinEach; ++i) {
            const int j = j0 + i * kJoinThreads;
            if (j >= a.max_len) break;
            float add = 0.0f;
            if constexpr (ROWS != 0) {
#pragma unroll
                for (int r = 0; r < ROWS; ++r) add += weight(s[i][r], join_norm[r]);
            } else if (j < len) {
                const float *at = scores + int64_t(i) * kJoinThreads * rows;
                for (int r = 0; r < rows; ++r) {
                    const float x = __ldcs(at + r);
                    add += weight(x, join_norm[r]);
                }
            }
            acc_out[pair * ld_acc + j] = j < len ? sum[i] + add : 0.0f;
        }
    }
    for (int row = blockIdx.x; row < rows; row += gridDim.x) {
        const int i = row / a.group, hq = head * a.group + row % a.group;
        float top = -INFINITY;
        for (int s = 0; s < a.splits; ++s) top = fmaxf(top, ml[s * rows + row].x);
        for (int d = threadIdx.x; d < D; d += kJoinThreads) {
            float sum = 0.0f, out = 0.0f;
#pragma unroll 4
            for (int s = 0; s < a.splits; ++s) {
                const float2 v = ml[s * rows + row];
                const float f = exp2_fast(v.x - top);
                sum = fmaf(f, v.y, sum);
                out = fmaf(f, part[(s * rows + row) * int64_t(D) + d], out);
            }
            const float y = sum == 0.0f ? 0.0f : out / sum;
            uint16_t bits;
            if constexpr (BF16) bits = __bfloat16_as_ushort(__float2bfloat16_rn(y));
            else bits = __half_as_ushort(__float2half_rn(y));
            a.O[seq * a.o.seq + i * a.o.token + hq * a.o.head + d] = bits;
            if (d == 0 && a.lse != nullptr)
                a.lse[(seq * a.n_q + i) * a.n_heads + hq] = (top + log2f(sum)) * 0.6931471805599453f;
        }
    }
}

// How many blocks share a (sequence, kv head, row tile), none with less than 64 tokens, and whether
// they finish together.  Where that gives a few blocks (short caches, few heads), a cluster of up
// to 8 spares the second kernel: 517 tokens of 16 heads take 6.7 us against 7.6.  Otherwise all
// blocks run at once, 4 an SM, and the second kernel has the device to itself: 32 x 8191 tokens of
// 8 heads with weights take 102 us (5.0 TB/s), in clusters 115 to 117 (blocks of a cluster start and end
// together).
// The counts are those of a B200's 148 SMs: the workspace is asked for without a device.
struct AttentionPlan {
    int row_tiles, splits;
    bool join;  // a second kernel joins the splits
};
static AttentionPlan attention_plan(const sp_cache &c, int64_t rows, int64_t max_len, bool want_acc) {
    AttentionPlan p;
    p.row_tiles = static_cast<int>(rows <= 8 ? 1 : (rows + 15) / 16);
    const int64_t units = std::max(int64_t(1), c.n_seqs * c.n_kv_heads * p.row_tiles);
    const int64_t most = std::max(int64_t(1), (max_len + 63) / 64);
    const int64_t want = std::max(int64_t(1), std::min(std::min(most, int64_t(256)), 148 * 4 / units));
    p.splits = static_cast<int>(want);
    if (want <= 15 && units * 8 <= 148 * 2 && (!want_acc || p.row_tiles == 1)) {
        p.splits = 1;
        while (p.splits < 8 && p.splits * 2 <= want) p.splits *= 2;
        p.join = false;
    } else {
        p.join = p.splits > 1 || want_acc;
    }
    return p;
}

int64_t cache_attention_workspace(const sp_cache &c, int64_t n_q, int n_heads, int64_t max_len, bool want_acc) {
    const int64_t rows = n_q * (n_heads / c.n_kv_heads), pairs = c.n_seqs * c.n_kv_heads;
    if (pairs == 0 || rows == 0) return 0;
    const AttentionPlan plan = attention_plan(c, rows, max_len, want_acc);
    int64_t bytes = want_acc ? (pairs * max_len * rows + 3) / 4 * 16 : 0;
    if (plan.join) bytes += pairs * plan.splits * rows * (c.head_dim * 4 + 8);
    return bytes;
}

sp_status launch_cache_attention(const sp_cache &c, const void *Q, const sp_strides &q, sp_dtype dtype, int64_t n_q,
                                 int n_heads, const int32_t *lens, int64_t max_len, float scale, void *O,
                                 const sp_strides &o, float *lse, const float *acc_in, float *acc_out, int64_t ld_acc,
                                 void *workspace, cudaStream_t stream) {
    AttnArgs a = {};
    a.cache = c;
    a.Q = static_cast<const uint16_t *>(Q);
    a.q = q;
    a.o = o;
    a.n_q = n_q;
    a.max_len = max_len;
    a.n_heads = n_heads;
    a.group = n_heads / c.n_kv_heads;
    a.rows = static_cast<int>(n_q * a.group);
    const AttentionPlan plan = attention_plan(c, a.rows, max_len, acc_out != nullptr);
    a.row_tiles = plan.row_tiles;
    a.splits = plan.splits;
    a.block_shift = c.block_tokens == 16 ? 4 : c.block_tokens == 32 ? 5 : 6;
    a.lens = lens;
    a.scale_log2 = scale * kLog2e;
    a.O = static_cast<uint16_t *>(O);
    a.lse = lse;
    const bool no_rows = a.rows == 0;  // the second kernel moves the accumulated weights alone
    const int64_t pairs = c.n_seqs * c.n_kv_heads;
    // scores first: their loads want 16-byte boundaries
    float *at = static_cast<float *>(workspace);
    if (acc_out != nullptr) {
        a.scores = at;
        at += (pairs * max_len * a.rows + 3) / 4 * 4;
    }
    if (!plan.join) {
        a.acc_in = acc_in;
        a.acc_out = acc_out;
        a.ld_acc = ld_acc;
    } else {
        a.part_o = at;
        a.part_ml = reinterpret_cast<float2 *>(at + pairs * a.splits * a.rows * c.head_dim);
    }
    ClusterPdlConfig pdl(plan.join ? 1 : a.splits, dim3(a.splits, c.n_kv_heads * a.row_tiles, static_cast<unsigned>(c.n_seqs)), dim3(kAttnWarps * 32), stream);
    CUtensorMap k_map = {}, v_map = {};
    cudaError_t e = cudaSuccess;
    if (c.n_blocks > 0 && !no_rows) {
        const int64_t pool_rows = c.n_blocks * c.n_kv_heads * c.block_tokens;
        if (c.n_blocks > 0x7fffffff || pool_rows > 0x7fffffff) return SP_ERR_SHAPE;
        e = encode_byte_rows(&k_map, c.k, pool_rows, c.head_dim, 16);
        if (e == cudaSuccess) e = encode_byte_rows(&v_map, c.v, pool_rows, c.head_dim, 16);
    }
    if (e != cudaSuccess) return cuda_fail(e);
    pdl.cfg.dynamicSmemBytes = kAttnWarps * kRing * c.head_dim * 32;
#define SP_LAUNCH(B, DD, N, TWICE)                                                                       \
    do {                                                                                                 \
        static DynamicSmem limit;                                                                        \
        auto *kernel = cache_attention_kernel<B, DD, N, TWICE>;                                          \
        e = limit.allow(reinterpret_cast<const void *>(kernel));                                         \
        if (e == cudaSuccess) e = cudaLaunchKernelEx(&pdl.cfg, kernel, k_map, v_map, a);                 \
    } while (0)
#define SP_ROWS(B, DD)                                    \
    do {                                                  \
        if (a.rows <= 4) SP_LAUNCH(B, DD, 1, true);       \
        else if (a.rows <= 8) SP_LAUNCH(B, DD, 1, false); \
        else SP_LAUNCH(B, DD, 2, false);                  \
    } while (0)
#define SP_PICK(B) \
    if (c.head_dim == 64) SP_ROWS(B, 64); else SP_ROWS(B, 128);
    if (no_rows) {}
    else if (dtype == SP_BF16) { SP_PICK(true) }
    else { SP_PICK(false) }
#undef SP_PICK
#undef SP_ROWS
#undef SP_LAUNCH
    if (e != cudaSuccess) return cuda_fail(e);
    if (!no_rows) {
        sp_status st = check_launch();
        if (st != SP_OK || !plan.join) return st;
    }
    const int64_t blocks = std::max(acc_out != nullptr ? (max_len + kJoinTokens - 1) / kJoinTokens : 1, std::min(int64_t(a.rows), int64_t(8)));
    if (blocks == 0) return SP_OK;
    PdlConfig second(dim3(static_cast<unsigned>(blocks), c.n_kv_heads, static_cast<unsigned>(c.n_seqs)), dim3(kJoinThreads), stream);
    second.cfg.dynamicSmemBytes = a.rows * sizeof(float2);
#define SP_LAUNCH(R)                                                                                                 \
    do {                                                                                                             \
        auto *kernel = dtype == SP_BF16 ? cache_join_kernel<true, R> : cache_join_kernel<false, R>;                  \
        static DynamicSmem limit[2];                                                                                 \
        if (second.cfg.dynamicSmemBytes > 48 * 1024)                                                                 \
            e = limit[dtype == SP_BF16].allow(reinterpret_cast<const void *>(kernel));                               \
        if (e == cudaSuccess) e = cudaLaunchKernelEx(&second.cfg, kernel, a, acc_in, acc_out, ld_acc);               \
    } while (0)
    switch (a.rows) {
        case 1: SP_LAUNCH(1); break;
        case 2: SP_LAUNCH(2); break;
        case 4: SP_LAUNCH(4); break;
        case 8: SP_LAUNCH(8); break;
        default: SP_LAUNCH(0); break;
    }
#undef SP_LAUNCH
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

}  // namespace sp
