// Appending keys and values to the 8-bit cache.
//
// Mathematics: e = the least exponent with max|v| <= 448 * 2^e over the finite new values of a
// (block, head), and at least the block's old one where it already holds tokens; code = e4m3 of
// v / 2^e.  Codes already there are rescaled by 2^(e_old - e), exact but for what falls among
// e4m3's subnormals.  Bound by memory (2 bytes read, 1 written per value): one block of threads
// holds a cache block's tile of one head in registers, so the maximum costs no second read.  Measured:
// 4 x 2047 tokens of 32 heads in f16 33.5 us (6.0 TB/s).
#include "cache_common.cuh"

namespace sp {

namespace {

struct AppendArgs {
    sp_cache cache;
    const uint16_t *x[2];  // K, V
    sp_strides stride[2];
    int n_new;
    const int32_t *start, *count;
};

}  // namespace

template <bool BF16, int D, int T, bool VEC>
__global__ void __launch_bounds__(128) cache_append_kernel(const AppendArgs a) {
    constexpr int kRowChunks = D / 8;               // 16-byte pieces of a token's new values
    constexpr int kChunks = T * kRowChunks / 128;   // of the tile, for a thread
    __shared__ uint32_t warp_amax[4];
    const sp_cache &c = a.cache;
    const int which = blockIdx.z & 1, head = blockIdx.y;
    const int64_t seq = blockIdx.z >> 1;
    pdl_launch_dependents();
    pdl_wait();
    const int begin = a.start[seq];
    const int n = a.count != nullptr ? min(a.count[seq], a.n_new) : a.n_new;
    if (begin < 0 || n <= 0) return;
    const int64_t place = begin / T + int(blockIdx.x);
    const int64_t first = place * T - begin;        // the tile's first token among the new ones
    if (first >= n) return;

    // the new values are on their way before the table is looked up
    const uint16_t *x = a.x[which] + seq * a.stride[which].seq + head * a.stride[which].head;
    const int64_t pitch = a.stride[which].token;
    const int d = threadIdx.x % kRowChunks * 8, row = threadIdx.x / kRowChunks;
    constexpr int kRowStep = 128 / kRowChunks;
    uint32_t p[kChunks][4];
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int64_t token = first + row + i * kRowStep;
        if (token >= 0 && token < n) load8<VEC, true>(x + token * pitch, d, D, p[i]);
        else p[i][0] = p[i][1] = p[i][2] = p[i][3] = 0u;
    }
    const int64_t block = cache_block(c, seq, place);
    if (block < 0) return;
    uint8_t *codes = static_cast<uint8_t *>(which == 0 ? c.k : c.v) + (block * c.n_kv_heads + head) * (T * D);
    float *scale = (which == 0 ? c.k_scale : c.v_scale) + block * c.n_kv_heads + head;
    const int e_old = first < 0 ? exponent_of(*scale) : kMinCacheExponent;

    // bit patterns of magnitudes order like the magnitudes; only a tile that holds something not
    // finite looks again
    auto reduce = [&](uint32_t m) {
        m = __reduce_max_sync(kFullWarp, m);
        __syncthreads();
        if ((threadIdx.x & 31) == 0) warp_amax[threadIdx.x >> 5] = m;
        __syncthreads();
        return max(max(warp_amax[0], warp_amax[1]), max(warp_amax[2], warp_amax[3]));
    };
    uint32_t amax = 0;
#pragma unroll
    for (int i = 0; i < kChunks; ++i)
#pragma unroll
        for (int k = 0; k < 4; ++k) amax = __vmaxu2(amax, p[i][k] & 0x7fff7fffu);
    amax = max(amax & 0xffffu, amax >> 16);
    amax = reduce(__float_as_uint(unpack2<BF16>(amax).x));
    const bool finite = amax < 0x7f800000u;
    if (!finite) {
        amax = 0;
#pragma unroll
        for (int i = 0; i < kChunks; ++i) {
            float v[8];
            unpack8<BF16>(p[i], v);
            amax = max(amax, finite_amax8(v));
        }
        amax = reduce(amax);
    }
    const int e = max(cache_exponent(amax), e_old);
    const float inv = pow2(-e);
#pragma unroll
    for (int i = 0; i < kChunks; ++i) {
        const int64_t token = first + row + i * kRowStep;
        uint2 *out = reinterpret_cast<uint2 *>(codes) + threadIdx.x + i * 128;
        float v[8];
        if (token >= 0 && token < n) {
            unpack8<BF16>(p[i], v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= inv;
            *out = finite ? e4m3_pack8_finite(v) : e4m3_pack8(v);
        } else if (token < 0 && e != e_old) {
            e4m3_unpack8(*out, v);
            const float f = pow2(e_old - e);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= f;
            *out = e4m3_pack8(v);
        }
    }
    if (threadIdx.x == 0) *scale = pow2(e);
}

sp_status launch_cache_append(const sp_cache &cache, const void *K, const sp_strides &ks, const void *V,
                              const sp_strides &vs, sp_dtype dtype, int64_t n_new, const int32_t *start,
                              const int32_t *count, cudaStream_t stream) {
    AppendArgs a = {};
    a.cache = cache;
    a.x[0] = static_cast<const uint16_t *>(K);
    a.x[1] = static_cast<const uint16_t *>(V);
    a.stride[0] = ks;
    a.stride[1] = vs;
    a.n_new = static_cast<int>(n_new);
    a.start = start;
    a.count = count;
    bool vec = aligned16(K) && aligned16(V);
    for (const sp_strides &s : a.stride) vec = vec && s.seq % 8 == 0 && s.token % 8 == 0 && s.head % 8 == 0;
    // x: the cache blocks that a sequence's new tokens can touch
    const int64_t touched = (n_new + cache.block_tokens - 2) / cache.block_tokens + 1;
    PdlConfig pdl(dim3(static_cast<unsigned>(touched), cache.n_kv_heads, static_cast<unsigned>(cache.n_seqs * 2)), dim3(128),
                  stream);
    cudaError_t e = cudaErrorInvalidValue;
#define SP_LAUNCH(D, T)                                                                          \
    if (cache.head_dim == D && cache.block_tokens == T) {                                        \
        if (dtype == SP_BF16)                                                                    \
            e = vec ? cudaLaunchKernelEx(&pdl.cfg, cache_append_kernel<true, D, T, true>, a)     \
                    : cudaLaunchKernelEx(&pdl.cfg, cache_append_kernel<true, D, T, false>, a);   \
        else                                                                                     \
            e = vec ? cudaLaunchKernelEx(&pdl.cfg, cache_append_kernel<false, D, T, true>, a)    \
                    : cudaLaunchKernelEx(&pdl.cfg, cache_append_kernel<false, D, T, false>, a);  \
    }
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
