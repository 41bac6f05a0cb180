// Eviction from the 8-bit cache by accumulated attention weight.
//
// Two launches.  Selection: for each (sequence, kv head) the need-th largest of the accumulated
// weights is found digit by digit (11, 11 and 10 bits, from the top, over an order-preserving
// integer image of the floats; the rest is skipped when a digit's keys are all needed); then the
// places of what is kept are written in token order: all above that value, and of its equals the
// first ones.  A row is spread over the blocks of a
// cluster, which hold its weights in registers - one read - and add up their digit counts through
// distributed shared memory; a row longer than a cluster's registers is read again in each of the
// passes.  Gathering: a block of threads lays block_tokens kept tokens of one head into a new
// cache block, K and V, the scales found from the codes it already holds in registers.  Bound by
// memory: 4 bytes read per token, and 2 * head_dim read and written per kept one.  Measured: 8 x 32768
// tokens of 8 heads to 4096 47.0 us, of which some 20 are the selection's chain of barriers and
// remote counts (several copies of the first digit's counts did not shorten it).
#include <algorithm>

#include "cache_common.cuh"

namespace sp {

namespace {

constexpr int kBins = 2048;
constexpr int kMostBlocks = 8;  // of a cluster

struct SelectArgs {
    const int32_t *lens;
    const float *acc;
    int64_t ld_acc, budget, recent, max_len;
    int32_t *kept;
    float *acc_out;
    int64_t ld_acc_out;
    int32_t *lens_out;
    int n_kv_heads;
};

// Integer image that orders like the value: NaN above everything, -0 equal to +0.
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t u = __float_as_uint(x + 0.0f);
    if ((u & 0x7fffffffu) > 0x7f800000u) return 0xffffffffu;
    return u & 0x80000000u ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ uint32_t load_remote(const uint32_t *p, int rank) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(remote_address(p, rank)) : "memory");
    return v;
}
__device__ __forceinline__ uint4 load_remote4(const uint32_t *p, int rank) {
    uint4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(remote_address(p, rank)) : "memory");
    return v;
}
// Sum over the threads before this one; `total` over all.
template <int THREADS>
__device__ __forceinline__ uint32_t block_prefix(uint32_t mine, uint32_t *warp_sum, uint32_t &total) {
    constexpr int kWarps = THREADS / 32;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    uint32_t sum = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint32_t up = __shfl_up_sync(kFullWarp, sum, o);
        if (lane >= o) sum += up;
    }
    __syncthreads();  // the last call's sums have been read
    if (lane == 31) warp_sum[warp] = sum;
    __syncthreads();
    uint32_t before = lane < kWarps ? warp_sum[lane] : 0u;
    const uint32_t own = before;
#pragma unroll
    for (int o = 1; o < kWarps; o <<= 1) {
        const uint32_t up = __shfl_up_sync(kFullWarp, before, o);
        if (lane >= o) before += up;
    }
    total = __shfl_sync(kFullWarp, before, kWarps - 1);
    return __shfl_sync(kFullWarp, before - own, warp) + sum - mine;
}

}  // namespace

// One cluster (of gridDim.x blocks) for a row; a warp has 32 * KEYS consecutive tokens of a stretch,
// a lane every 32nd of them.  The row is cut into stretches of gridDim.x * THREADS * KEYS tokens;
// HELD: there is one, kept in registers.
template <int THREADS, int KEYS, bool HELD>
__global__ void __launch_bounds__(THREADS, 2) cache_select_kernel(const SelectArgs a) {
    __shared__ __align__(16) uint32_t hist[2][kBins];
    __shared__ uint32_t warp_sum[32], found[3], counts[2];
    __shared__ uint2 warp_counts[32];
    const int64_t row = blockIdx.y + int64_t(blockIdx.z) * gridDim.y;
    const int64_t seq = row / a.n_kv_heads;
    const int tid = threadIdx.x, rank = blockIdx.x, ranks = gridDim.x;
    for (int i = tid; i < 2 * kBins; i += THREADS) (&hist[0][0])[i] = 0;
    __syncthreads();
    pdl_launch_dependents();
    pdl_wait();
    const int n = static_cast<int>(max(int64_t(0), min(int64_t(a.lens[seq]), a.max_len)));
    const int m = static_cast<int>(min(int64_t(n), a.budget)), last = static_cast<int>(min(a.recent, int64_t(m)));
    const int free = n - last, need = m - last;
    const float *acc = a.acc + row * a.ld_acc;
    int32_t *kept = a.kept + row * a.budget;
    const int per_block = THREADS * KEYS, stretch = ranks * per_block;
    const int lane = tid & 31, warp = tid >> 5;
    const int mine = rank * per_block + warp * (32 * KEYS) + lane;  // this thread's first token of a stretch

    float x[KEYS];
    auto load = [&](int j0) {
#pragma unroll
        for (int i = 0; i < KEYS; ++i) x[i] = j0 + mine + i * 32 < n ? __ldg(acc + j0 + mine + i * 32) : 0.0f;
    };
    if constexpr (HELD) load(0);

    // cut: keys above it are kept, and the first `ties` of those equal to it
    uint32_t cut = 0xffffffffu, ties = 0;
    if (need >= free) {
        cut = 0;
        ties = 0xffffffffu;
    } else if (need > 0) {
        uint32_t prefix = 0, left = static_cast<uint32_t>(need);
#pragma unroll 1
        for (int pass = 0; pass < 3; ++pass) {
            const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
            const uint32_t bins = pass == 2 ? 1024u : 2048u;
            const uint32_t above_mask = pass == 0 ? 0u : ~0u << (pass == 1 ? 21 : 10);
            uint32_t *h = hist[pass & 1];
            for (int j0 = 0; j0 < free; j0 += stretch) {
                if constexpr (!HELD) load(j0);
#pragma unroll
                for (int i = 0; i < KEYS; ++i) {
                    const uint32_t k = order_key(x[i]);
                    if (j0 + mine + i * 32 < free && (k & above_mask) == prefix) atomicAdd(&h[(k >> shift) & (bins - 1u)], 1u);
                }
            }
            if (ranks > 1) cluster_sync();
            else __syncthreads();
            // digits from the top, kPer a thread; all blocks come to the same answer
            constexpr int kPer = kBins / THREADS > 4 ? kBins / THREADS : 4;
            uint32_t c[kPer], sum = 0;
#pragma unroll
            for (int i = 0; i < kPer; ++i) c[i] = 0u;
            if (tid * kPer < kBins) {
#pragma unroll
                for (int i = 0; i < kPer; i += 4) {
                    const uint32_t *at = &h[kBins - 4 - (tid * kPer + i)];
#pragma unroll 1
                    for (int r0 = 0; r0 < ranks; r0 += 4) {
                        uint4 v[4];
#pragma unroll
                        for (int r = 0; r < 4; ++r)  // all on their way before the first is used
                            if (r0 + r < ranks) v[r] = ranks > 1 ? load_remote4(at, r0 + r) : *reinterpret_cast<const uint4 *>(at);
#pragma unroll
                        for (int r = 0; r < 4; ++r)
                            if (r0 + r < ranks) {
                                c[i] += v[r].w;
                                c[i + 1] += v[r].z;
                                c[i + 2] += v[r].y;
                                c[i + 3] += v[r].x;
                            }
                    }
                }
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) sum += c[i];
            uint32_t total, above = block_prefix<THREADS>(sum, warp_sum, total);
            if (above < left && above + sum >= left) {
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    if (above < left && above + c[i] >= left) {
                        found[0] = kBins - 1 - (tid * kPer + i);
                        found[1] = left - above;
                        found[2] = c[i];
                    }
                    above += c[i];
                }
            }
            // the other counts were last read before this pass's barrier
            if (pass == 1)
                for (int i = tid; i < kBins; i += THREADS) hist[0][i] = 0;
            __syncthreads();
            prefix |= found[0] << shift;
            left = found[1];
            if (left == found[2]) {  // every key that begins like this is kept
                left = prefix == 0u ? 0xffffffffu : 0u;
                prefix = prefix == 0u ? 0u : prefix - 1u;
                break;
            }
        }
        cut = prefix;
        ties = left;
    }

    // in token order: a kept token's place is the number of kept ones before it
    uint32_t over_before = 0, equal_before = 0;
    for (int j0 = 0; j0 < n; j0 += stretch) {
        if constexpr (!HELD) load(j0);
        uint32_t over = 0, equal = 0;  // bit i: of this lane's token i
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const int j = j0 + mine + i * 32;
            const uint32_t k = order_key(x[i]);
            if (j >= free ? j < n : need > 0 && k > cut) over |= 1u << i;
            if (j < free && need > 0 && k == cut) equal |= 1u << i;
        }
        const uint32_t warp_over = __reduce_add_sync(kFullWarp, __popc(over));
        const uint32_t warp_equal = __reduce_add_sync(kFullWarp, __popc(equal));
        // kept ones before this warp, before this block, and in all
        __syncthreads();
        if (lane == 0) warp_counts[warp] = make_uint2(warp_over, warp_equal);
        __syncthreads();
        uint2 own = lane < THREADS / 32 ? warp_counts[lane] : make_uint2(0u, 0u);
        uint32_t total_over = __reduce_add_sync(kFullWarp, own.x), total_equal = __reduce_add_sync(kFullWarp, own.y);
        uint32_t o_at = __reduce_add_sync(kFullWarp, lane < warp ? own.x : 0u);
        uint32_t e_at = __reduce_add_sync(kFullWarp, lane < warp ? own.y : 0u);
        if (ranks > 1) {
            if (tid == 0) {
                counts[0] = total_over;
                counts[1] = total_equal;
            }
            cluster_sync();
            own = make_uint2(0u, 0u);
            if (lane < ranks) own = make_uint2(load_remote(&counts[0], lane), load_remote(&counts[1], lane));
            total_over = __reduce_add_sync(kFullWarp, own.x);
            total_equal = __reduce_add_sync(kFullWarp, own.y);
            o_at += __reduce_add_sync(kFullWarp, lane < rank ? own.x : 0u);
            e_at += __reduce_add_sync(kFullWarp, lane < rank ? own.y : 0u);
            if (!HELD) cluster_sync();
        }
        o_at += over_before;
        e_at += equal_before;
        const uint32_t lower = (1u << lane) - 1u;
        float *acc_out = a.acc_out != nullptr ? a.acc_out + row * a.ld_acc_out : nullptr;
#pragma unroll
        for (int i = 0; i < KEYS; ++i) {
            const bool is_over = (over >> i) & 1u;
            const uint32_t overs = __ballot_sync(kFullWarp, is_over);
            if (warp_equal == 0u || ties == 0u) {  // nearly always: the values are all different
                if (is_over) {
                    const uint32_t at = o_at + min(e_at, ties) + __popc(overs & lower);
                    kept[at] = j0 + mine + i * 32;
                    if (acc_out != nullptr) acc_out[at] = x[i];
                }
            } else {
                const bool is_equal = (equal >> i) & 1u;
                const uint32_t equals = __ballot_sync(kFullWarp, is_equal);
                const uint32_t e_mine = e_at + __popc(equals & lower);
                if (is_over || (is_equal && e_mine < ties)) {
                    const uint32_t at = o_at + __popc(overs & lower) + min(e_mine, ties);
                    kept[at] = j0 + mine + i * 32;
                    if (acc_out != nullptr) acc_out[at] = x[i];
                }
                e_at += __popc(equals);
            }
            o_at += __popc(overs);
        }
        over_before += total_over;
        equal_before += total_equal;
    }
    for (int64_t at = m + rank * THREADS + tid; at < a.budget; at += ranks * THREADS) {
        kept[at] = -1;
        if (a.acc_out != nullptr) a.acc_out[row * a.ld_acc_out + at] = 0.0f;
    }
    if (a.lens_out != nullptr && row % a.n_kv_heads == 0 && rank == 0 && tid == 0) a.lens_out[seq] = m;
    if (ranks > 1) cluster_sync();  // no block leaves while its counts are read
}

template <int THREADS, int KEYS, bool HELD>
static cudaError_t launch_select(const SelectArgs &a, int64_t rows, int ranks, cudaStream_t stream) {
    ClusterPdlConfig pdl(ranks, dim3(ranks, static_cast<unsigned>(a.n_kv_heads), static_cast<unsigned>(rows / a.n_kv_heads)),
                         dim3(THREADS), stream);
    return cudaLaunchKernelEx(&pdl.cfg, cache_select_kernel<THREADS, KEYS, HELD>, a);
}

static cudaError_t launch_select(const SelectArgs &a, int64_t rows, cudaStream_t stream) {
    if (a.max_len <= 2048) return launch_select<256, 8, true>(a, rows, 1, stream);
    // blocks of a row's cluster: as many as the row fills at 16 tokens a thread
    int ranks = 1;
    while (ranks < kMostBlocks && ranks * 8192 < a.max_len) ranks *= 2;
    if (ranks * 8192 >= a.max_len) return launch_select<512, 16, true>(a, rows, ranks, stream);
    return launch_select<512, 16, false>(a, rows, ranks, stream);
}

template <int D, int T>
__global__ void __launch_bounds__(128)
cache_gather_kernel(const sp_cache src, const sp_cache dst, const int32_t *__restrict__ kept, int budget) {
    constexpr int kRowPieces = D / 16;                        // pieces of 16 codes of a token
    constexpr int kThreads = T * kRowPieces < 128 ? T * kRowPieces : 128;  // that have a piece
    constexpr int kPieces = T * kRowPieces / kThreads;        // of the tile, for a thread
    constexpr int kRowStep = kThreads / kRowPieces;
    __shared__ uint32_t warp_amax[2][4];
    const int head = blockIdx.y, H = src.n_kv_heads;
    const int64_t seq = blockIdx.z;
    pdl_launch_dependents();
    pdl_wait();
    const bool active = kThreads == 128 || threadIdx.x < kThreads;
    const int d = threadIdx.x % kRowPieces, row = threadIdx.x / kRowPieces;
    const int32_t *k = kept + (seq * H + head) * budget;
    const int32_t *table = src.table + seq * src.ld_table;
    const int64_t to = cache_block(dst, seq, blockIdx.x);
    if (to < 0) return;
    uint4 w[2][kPieces];
    float scale[2][kPieces];
    int j[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        const int64_t slot = int64_t(blockIdx.x) * T + row + i * kRowStep;
        j[i] = active && slot < budget ? k[slot] : -1;
    }
    int block[kPieces];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) block[i] = j[i] >= 0 && unsigned(j[i]) / T < src.table_cols ? table[unsigned(j[i]) / T] : -1;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
        w[0][i] = w[1][i] = make_uint4(0u, 0u, 0u, 0u);
        scale[0][i] = scale[1][i] = 0.0f;
        if (block[i] >= 0 && block[i] < src.n_blocks) {
            const int64_t tile = int64_t(block[i]) * H + head;
            const int64_t piece = (tile * T + unsigned(j[i]) % T) * kRowPieces + d;
            w[0][i] = __ldg(static_cast<const uint4 *>(src.k) + piece);
            w[1][i] = __ldg(static_cast<const uint4 *>(src.v) + piece);
            scale[0][i] = src.k_scale[tile];
            scale[1][i] = src.v_scale[tile];
        }
    }
    // the largest finite code of a piece (codes order like their magnitudes), times its token's scale
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        uint32_t amax = 0;
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            const uint4 &c = w[which][i];
            constexpr uint32_t kBare = 0x7f7f7f7fu;
            uint32_t m = __vmaxu4(__vmaxu4(c.x & kBare, c.y & kBare), __vmaxu4(c.z & kBare, c.w & kBare));
            m = __vmaxu4(m, m >> 16);
            m = max(m & 0xffu, (m >> 8) & 0xffu);
            float top;
            if (m != 0x7fu) {
                uint32_t lo, hi;
                e4m3_to_f16(m, lo, hi);
                top = unpack2<false>(lo).x;
            } else {
                float v[8];
                e4m3_unpack8(make_uint2(c.x, c.y), v);
                uint32_t bits = finite_amax8(v);
                e4m3_unpack8(make_uint2(c.z, c.w), v);
                bits = max(bits, finite_amax8(v));
                top = __uint_as_float(bits);
            }
            amax = max(amax, __float_as_uint(top * scale[which][i]));
        }
        amax = __reduce_max_sync(kFullWarp, amax);
        if ((threadIdx.x & 31) == 0) warp_amax[which][threadIdx.x >> 5] = amax;
    }
    __syncthreads();
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        const uint32_t *m = warp_amax[which];
        const int e = cache_exponent(max(max(m[0], m[1]), max(m[2], m[3])));
        uint4 *out = static_cast<uint4 *>(which == 0 ? dst.k : dst.v) + (to * H + head) * (T * kRowPieces);
#pragma unroll
        for (int i = 0; i < kPieces; ++i) {
            // between scales further apart than binary32 reaches, a code is 0 or NaN: any factor serves
            const float f = pow2(min(exponent_of(scale[which][i]) - e, 127));
            uint4 y = w[which][i];
            if (f != 1.0f) {  // most tokens keep their scale, and so their codes
                float v[8];
                e4m3_unpack8(make_uint2(y.x, y.y), v);
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] *= f;
                const uint2 lo = e4m3_pack8_finite(v);
                e4m3_unpack8(make_uint2(y.z, y.w), v);
#pragma unroll
                for (int q = 0; q < 8; ++q) v[q] *= f;
                const uint2 hi = e4m3_pack8_finite(v);
                y = make_uint4(lo.x, lo.y, hi.x, hi.y);
            }
            if (active) out[threadIdx.x + i * kThreads] = y;
        }
        if (threadIdx.x == 0) (which == 0 ? dst.k_scale : dst.v_scale)[to * H + head] = pow2(e);
    }
}

sp_status launch_cache_evict(const sp_cache &src, const int32_t *lens, int64_t max_len, const float *acc, int64_t ld_acc,
                             int64_t budget, int64_t recent, const sp_cache &dst, int32_t *kept, float *acc_out,
                             int64_t ld_acc_out, int32_t *lens_out, cudaStream_t stream) {
    const int64_t rows = src.n_seqs * src.n_kv_heads;
    const int64_t places = (budget + src.block_tokens - 1) / src.block_tokens;
    if (rows > 0x7fffffff) return SP_ERR_SHAPE;
    SelectArgs a = {};
    a.lens = lens;
    a.acc = acc;
    a.ld_acc = ld_acc;
    a.budget = budget;
    a.recent = recent;
    a.max_len = std::min(max_len, src.table_cols * src.block_tokens);
    a.kept = kept;
    a.acc_out = acc_out;
    a.ld_acc_out = ld_acc_out;
    a.lens_out = lens_out;
    a.n_kv_heads = src.n_kv_heads;
    cudaError_t e = launch_select(a, rows, stream);
    if (e != cudaSuccess) return cuda_fail(e);
    sp_status st = check_launch();
    if (st != SP_OK) return st;
    if (places == 0) return SP_OK;
    PdlConfig pdl(dim3(static_cast<unsigned>(places), src.n_kv_heads, static_cast<unsigned>(src.n_seqs)), dim3(128), stream);
    const int kept_budget = static_cast<int>(budget);
    e = cudaErrorInvalidValue;
#define SP_LAUNCH(D, T)                                      \
    if (src.head_dim == D && src.block_tokens == T)          \
        e = cudaLaunchKernelEx(&pdl.cfg, cache_gather_kernel<D, T>, src, dst, kept, kept_budget);
    SP_LAUNCH(64, 16)
    SP_LAUNCH(64, 32)
    SP_LAUNCH(64, 64)
    SP_LAUNCH(128, 16)
    SP_LAUNCH(128, 32)
    SP_LAUNCH(128, 64)
#undef SP_LAUNCH
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

}  // namespace sp
