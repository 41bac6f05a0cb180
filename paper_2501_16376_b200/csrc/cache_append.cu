// Appending keys and values to the 8-bit cache.
//
// Mathematics: e = the least exponent with max|v| <= 448 * 2^e over the finite new values of a
// (block, head), and at least the block's old one where it already holds tokens; code = e4m3 of
// v / 2^e.  Codes already there are rescaled by 2^(e_old - e), exact but for what falls among
// e4m3's subnormals.  Bound by memory (2 bytes read, 1 written per value): one block of threads
// holds a cache block's tile of one head in registers, so the maximum costs no second read.
#include "cache_common.cuh"

namespace sp {

namespace {

struct AppendArgs {
    sp_cache cache;
    const uint16_t *x[2];  // K, V
    sp_strides stride[2];
    int64_t n_new;
    const int32_t *start, *count;
    int64_t touched;  // cache blocks a sequence's new tokens can touch
};

}  // namespace

// CHUNKS 16-byte pieces of the new values a thread: block_tokens * head_dim / 8 / 128
template <bool BF16, int CHUNKS, bool VEC>
__global__ void __launch_bounds__(128) cache_append_kernel(const AppendArgs a) {
    __shared__ uint32_t warp_amax[4];
    const sp_cache &c = a.cache;
    const int which = blockIdx.z, head = blockIdx.y;
    const int64_t seq = blockIdx.x / a.touched;
    const int D = c.head_dim, T = c.block_tokens, row_chunks = D / 8;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t begin = a.start[seq];
    const int64_t n = a.count != nullptr ? min(int64_t(a.count[seq]), a.n_new) : a.n_new;
    if (begin < 0 || n <= 0) return;
    const int64_t place = begin / T + blockIdx.x % a.touched;
    if (place * T >= begin + n) return;
    const int64_t block = cache_block(c, seq, place);
    if (block < 0) return;

    const uint16_t *x = a.x[which] + seq * a.stride[which].seq + head * a.stride[which].head;
    uint8_t *codes = static_cast<uint8_t *>(which == 0 ? c.k : c.v) + (block * c.n_kv_heads + head) * T * D;
    float *scale = (which == 0 ? c.k_scale : c.v_scale) + block * c.n_kv_heads + head;
    const bool has_old = begin > place * T;
    const int e_old = has_old ? exponent_of(*scale) : kMinCacheExponent;

    uint32_t p[CHUNKS][4], amax = 0;
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        const int at = threadIdx.x + i * 128;
        const int64_t token = place * T + at / row_chunks - begin;
        if (token >= 0 && token < n) {
            load8<VEC, true>(x + token * a.stride[which].token, at % row_chunks * 8, D, p[i]);
            float v[8];
            unpack8<BF16>(p[i], v);
            amax = max(amax, finite_amax8(v));
        }
    }
    amax = __reduce_max_sync(kFullWarp, amax);
    if ((threadIdx.x & 31) == 0) warp_amax[threadIdx.x >> 5] = amax;
    __syncthreads();
    amax = max(max(warp_amax[0], warp_amax[1]), max(warp_amax[2], warp_amax[3]));
    const int e = max(cache_exponent(amax), e_old);
    const float inv = pow2(-e);
#pragma unroll
    for (int i = 0; i < CHUNKS; ++i) {
        const int at = threadIdx.x + i * 128;
        const int64_t token = place * T + at / row_chunks - begin;
        uint2 *out = reinterpret_cast<uint2 *>(codes) + at;
        float v[8];
        if (token >= 0 && token < n) {
            unpack8<BF16>(p[i], v);
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] *= inv;
            *out = e4m3_pack8(v);
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
    a.n_new = n_new;
    a.start = start;
    a.count = count;
    a.touched = (n_new + cache.block_tokens - 2) / cache.block_tokens + 1;
    if (a.touched > 0x7fffffff / cache.n_seqs) return SP_ERR_SHAPE;
    bool vec = aligned16(K) && aligned16(V);
    for (const sp_strides &s : a.stride) vec = vec && s.seq % 8 == 0 && s.token % 8 == 0 && s.head % 8 == 0;
    PdlConfig pdl(dim3(static_cast<unsigned>(a.touched * cache.n_seqs), cache.n_kv_heads, 2), dim3(128), stream);
    const int chunks = cache.block_tokens * cache.head_dim / 1024;
    cudaError_t e = cudaErrorInvalidValue;
#define SP_LAUNCH(C)                                                                          \
    if (chunks == C) {                                                                        \
        if (dtype == SP_BF16)                                                                 \
            e = vec ? cudaLaunchKernelEx(&pdl.cfg, cache_append_kernel<true, C, true>, a)     \
                    : cudaLaunchKernelEx(&pdl.cfg, cache_append_kernel<true, C, false>, a);   \
        else                                                                                  \
            e = vec ? cudaLaunchKernelEx(&pdl.cfg, cache_append_kernel<false, C, true>, a)    \
                    : cudaLaunchKernelEx(&pdl.cfg, cache_append_kernel<false, C, false>, a);  \
    }
    SP_LAUNCH(1)
    SP_LAUNCH(2)
    SP_LAUNCH(4)
    SP_LAUNCH(8)
#undef SP_LAUNCH
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

}  // namespace sp
