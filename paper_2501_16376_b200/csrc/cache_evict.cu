// Eviction from the 8-bit cache by accumulated attention weight.
//
// Two launches.  Selection: for each (sequence, kv head) the need-th largest of the accumulated
// weights is found digit by digit (8 bits a pass, from the top, over an order-preserving integer
// image of the floats); then one pass in token order writes the places of what is kept: all above
// that value, and of its equals the first ones.  Gathering: a block of threads lays block_tokens
// kept tokens of one head into a new cache block, its scale found from the codes it already holds
// in registers.  Bound by memory: 4 bytes read per token, and 2 * head_dim moved twice per kept one.
#include <algorithm>

#include "cache_common.cuh"

namespace sp {

namespace {

constexpr int kSelectThreads = 1024;
constexpr int kPerThread = 4;

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

}  // namespace

__global__ void __launch_bounds__(kSelectThreads) cache_select_kernel(const SelectArgs a) {
    __shared__ uint32_t hist[256], warp_sum[32];
    __shared__ uint32_t found[2];
    const int64_t row = blockIdx.x, seq = row / a.n_kv_heads;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t n = max(int64_t(0), min(int64_t(a.lens[seq]), a.max_len));
    const int64_t m = min(n, a.budget), last = min(a.recent, m), free = n - last;
    const float *acc = a.acc + row * a.ld_acc;
    int32_t *kept = a.kept + row * a.budget;
    const int64_t need = m - last;

    // cut: keys above it are kept, and the first `ties` of those equal to it
    uint32_t cut = 0xffffffffu, ties = 0;
    if (need >= free) {
        cut = 0;
        ties = 0xffffffffu;
    } else if (need > 0) {
        uint32_t prefix = 0, left = static_cast<uint32_t>(need);
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) hist[tid] = 0;
            __syncthreads();
            for (int64_t j = tid; j < free; j += kSelectThreads) {
                const uint32_t k = order_key(acc[j]);
                if (shift == 24 || (k >> (shift + 8)) == (prefix >> (shift + 8))) atomicAdd(&hist[(k >> shift) & 255u], 1u);
            }
            __syncthreads();
            // the digit whose count, added to those above it, first reaches what is left
            if (warp == 0) {
                uint32_t mine = 0, c[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    c[i] = hist[255 - (lane * 8 + i)];
                    mine += c[i];
                }
                uint32_t above = mine;
                for (int o = 1; o < 32; o <<= 1) {
                    const uint32_t up = __shfl_up_sync(kFullWarp, above, o);
                    if (lane >= o) above += up;
                }
                above -= mine;
                if (above < left && above + mine >= left) {
                    int i = 0;
                    while (above + c[i] < left) above += c[i++];
                    found[0] = 255 - (lane * 8 + i);
                    found[1] = left - above;
                }
            }
            __syncthreads();
            prefix |= found[0] << shift;
            left = found[1];
            __syncthreads();
        }
        cut = prefix;
        ties = left;
    }

    // in token order: place of a kept token = kept ones before it
    uint32_t over_before = 0, equal_before = 0;
    for (int64_t j0 = 0; j0 < n; j0 += kSelectThreads * kPerThread) {
        uint32_t over = 0, equal = 0;  // of this thread's consecutive tokens, as bits
        float x[kPerThread];
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const int64_t j = j0 + tid * kPerThread + i;
            if (j < n) {
                x[i] = acc[j];
                const uint32_t k = order_key(x[i]);
                if (j >= free || (need > 0 && k > cut)) over |= 1u << i;
                else if (need > 0 && k == cut) equal |= 1u << i;
            }
        }
        // counts of both kinds share a word: at most 4096 of each in a tile
        const uint32_t mine = __popc(over) | (__popc(equal) << 16);
        uint32_t sum = mine;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(kFullWarp, sum, o);
            if (lane >= o) sum += up;
        }
        if (lane == 31) warp_sum[warp] = sum;
        __syncthreads();
        uint32_t total = warp_sum[lane], before = total;
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t up = __shfl_up_sync(kFullWarp, before, o);
            if (lane >= o) before += up;
        }
        total = __shfl_sync(kFullWarp, before, 31);
        before = __shfl_sync(kFullWarp, before, (warp + 31) & 31);
        if (warp == 0) before = 0;
        before += sum - mine;
        uint32_t o_at = over_before + (before & 0xffffu), e_at = equal_before + (before >> 16);
#pragma unroll
        for (int i = 0; i < kPerThread; ++i) {
            const bool is_over = (over >> i) & 1u, is_equal = (equal >> i) & 1u;
            if (is_over || (is_equal && e_at < ties)) {
                const int64_t at = o_at + min(e_at, ties);
                kept[at] = static_cast<int32_t>(j0 + tid * kPerThread + i);
                if (a.acc_out != nullptr) a.acc_out[row * a.ld_acc_out + at] = x[i];
            }
            o_at += is_over;
            e_at += is_equal;
        }
        over_before += total & 0xffffu;
        equal_before += total >> 16;
        __syncthreads();
    }
    for (int64_t at = m + tid; at < a.budget; at += kSelectThreads) {
        kept[at] = -1;
        if (a.acc_out != nullptr) a.acc_out[row * a.ld_acc_out + at] = 0.0f;
    }
    if (a.lens_out != nullptr && row % a.n_kv_heads == 0 && tid == 0) a.lens_out[seq] = static_cast<int32_t>(m);
}

template <int D, int T>
__global__ void __launch_bounds__(128)
cache_gather_kernel(const sp_cache src, const sp_cache dst, const int32_t *__restrict__ kept, int budget) {
    constexpr int kRowChunks = D / 8;               // pieces of 8 codes of a token
    constexpr int kChunks = T * kRowChunks / 128;   // of the tile, for a thread
    constexpr int kRowStep = 128 / kRowChunks;
    __shared__ uint32_t warp_amax[4];
    const int which = blockIdx.z & 1, head = blockIdx.y, H = src.n_kv_heads;
    const int64_t seq = blockIdx.z >> 1;
    pdl_launch_dependents();
    pdl_wait();
    const int d = threadIdx.x % kRowChunks, row = threadIdx.x / kRowChunks;
    const int32_t *k = kept + (seq * H + head) * budget;
    int j[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int64_t slot = int64_t(blockIdx.x) * T + row + i * kRowStep;
        j[i] = slot < budget ? k[slot] : -1;
    }
    const int64_t to = cache_block(dst, seq, blockIdx.x);
    if (to < 0) return;
    const uint8_t *from = static_cast<const uint8_t *>(which == 0 ? src.k : src.v);
    const float *from_scale = which == 0 ? src.k_scale : src.v_scale;
    uint2 w[kChunks];
    float scale[kChunks];
    int64_t at[kChunks];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) at[i] = j[i] >= 0 ? cache_block(src, seq, unsigned(j[i]) / T) * H + head : -1;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        w[i] = make_uint2(0u, 0u);
        scale[i] = 0.0f;
        if (at[i] >= 0) {
            w[i] = __ldg(reinterpret_cast<const uint2 *>(from + (at[i] * T + unsigned(j[i]) % T) * D) + d);
            scale[i] = from_scale[at[i]];
        }
    }
    // the largest finite code of a piece, times its token's scale
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        float v[8];
        e4m3_unpack8(w[i], v);
        amax = max(amax, __float_as_uint(__uint_as_float(finite_amax8(v)) * scale[i]));
    }
    amax = __reduce_max_sync(kFullWarp, amax);
    if ((threadIdx.x & 31) == 0) warp_amax[threadIdx.x >> 5] = amax;
    __syncthreads();
    amax = max(max(warp_amax[0], warp_amax[1]), max(warp_amax[2], warp_amax[3]));
    const int e = cache_exponent(amax);
    const float inv = pow2(-e);
    uint2 *out = reinterpret_cast<uint2 *>(static_cast<uint8_t *>(which == 0 ? dst.k : dst.v) + (to * H + head) * (T * D));
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const float f = scale[i] * inv;
        uint2 y = w[i];
        if (f != 1.0f) {  // most tokens keep their scale, and so their codes
            float v[8];
            e4m3_unpack8(w[i], v);
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] *= f;
            y = e4m3_pack8(v);
        }
        out[threadIdx.x + i * 128] = y;
    }
    if (threadIdx.x == 0) (which == 0 ? dst.k_scale : dst.v_scale)[to * H + head] = pow2(e);
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
    PdlConfig select(dim3(static_cast<unsigned>(rows)), dim3(kSelectThreads), stream);
    cudaError_t e = cudaLaunchKernelEx(&select.cfg, cache_select_kernel, a);
    if (e != cudaSuccess) return cuda_fail(e);
    sp_status st = check_launch();
    if (st != SP_OK) return st;
    if (places == 0) return SP_OK;
    PdlConfig pdl(dim3(static_cast<unsigned>(places), src.n_kv_heads, static_cast<unsigned>(src.n_seqs * 2)), dim3(128), stream);
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
