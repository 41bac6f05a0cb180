// Attention of a batch whose sequences share prefixes, over the 8-bit cache.
#include "cache_common.cuh"
#include "sp_internal.h"

namespace sp {

namespace {

struct SharedArgs {
    sp_cache cache;
    SharedAttention s;
    float scale_log2;
    int group;
};

// Which group a sequence is in, by the first max_group of each; where its own tokens begin.
struct Place {
    int first;      // row of the table that holds the shared blocks
    int64_t own;    // tokens before this one are the shared ones
};
__device__ __forceinline__ Place place_of(const SharedArgs &a, int64_t seq) {
    Place p{static_cast<int>(seq), 0};
    for (int64_t g = 0; g < a.s.n_groups; ++g) {
        const int64_t begin = a.s.group_start[g], end = min(int64_t(a.s.group_start[g + 1]), begin + a.s.max_group);
        if (seq < begin || seq >= end) continue;
        const int64_t T = a.cache.block_tokens, tokens = min(int64_t(a.s.prefix[g]), a.s.max_prefix);
        p.first = static_cast<int>(begin);
        p.own = max(int64_t(0), min(tokens / T, a.cache.table_cols)) * T;
    }
    return p;
}

}  // namespace

// A warp a query head.
template <bool BF16, int D>
__global__ void __launch_bounds__(32)
cache_shared_simple_kernel(const __grid_constant__ SharedArgs a) {
    constexpr int kEach = D / 32;
    const sp_cache &c = a.cache;
    const int lane = threadIdx.x, hq = blockIdx.x, head = hq / a.group;
    const int64_t i = blockIdx.y, seq = blockIdx.z;
    pdl_launch_dependents();
    pdl_wait();
    const Place place = place_of(a, seq);
    const int64_t T = c.block_tokens;
    const int64_t end = min(min(a.s.lens[seq] - a.s.n_q + i + 1, min(int64_t(a.s.lens[seq]), a.s.max_len)), c.table_cols * T);
    const uint16_t *q = static_cast<const uint16_t *>(a.s.Q) + seq * a.s.q.seq + i * a.s.q.token + hq * a.s.q.head;
    float x[kEach], o[kEach] = {}, m = -3.4028234663852886e38f, l = 0.0f;
#pragma unroll
    for (int d = 0; d < kEach; ++d) x[d] = BF16 ? __uint_as_float(uint32_t(q[lane * kEach + d]) << 16) : __half2float(__ushort_as_half(q[lane * kEach + d]));
    for (int64_t j = 0; j < end; ++j) {
        const int64_t block = cache_block(c, j < place.own ? place.first : seq, j / T);
        if (block < 0) continue;
        const int64_t tile = block * c.n_kv_heads + head, at = (tile * T + j % T) * D + lane * kEach;
        float s = 0.0f, v[kEach];
#pragma unroll
        for (int d = 0; d < kEach; ++d) {
            uint32_t lo, hi;
            const uint32_t w = static_cast<const uint8_t *>(c.k)[at + d] | uint32_t(static_cast<const uint8_t *>(c.v)[at + d]) << 8;
            e4m3_to_f16(w, lo, hi);
            const float2 f = unpack2<false>(lo);
            s = fmaf(x[d], f.x, s);
            v[d] = f.y * c.v_scale[tile];
        }
#pragma unroll
        for (int w = 16; w > 0; w >>= 1) s += __shfl_xor_sync(kFullWarp, s, w);
        s *= c.k_scale[tile] * a.scale_log2;
        const float top = fmaxf(m, s), f = exp2f(m - top), p = exp2f(s - top);
        l = l * f + p;
#pragma unroll
        for (int d = 0; d < kEach; ++d) o[d] = o[d] * f + p * v[d];
        m = top;
    }
    uint16_t *out = static_cast<uint16_t *>(a.s.O) + seq * a.s.o.seq + i * a.s.o.token + hq * a.s.o.head;
#pragma unroll
    for (int d = 0; d < kEach; ++d) {
        const float y = l == 0.0f ? 0.0f : o[d] / l;
        out[lane * kEach + d] = BF16 ? __bfloat16_as_ushort(__float2bfloat16_rn(y)) : __half_as_ushort(__float2half_rn(y));
    }
    if (lane == 0 && a.s.lse != nullptr) a.s.lse[(seq * a.s.n_q + i) * a.s.n_heads + hq] = (m + log2f(l)) * 0.6931471805599453f;
}

int64_t cache_shared_workspace(const sp_cache &, const SharedAttention &) { return 0; }

sp_status launch_cache_shared(const sp_cache &c, const SharedAttention &s, void *, cudaStream_t stream) {
    const SharedArgs a{c, s, s.scale * 1.4426950408889634f, s.n_heads / c.n_kv_heads};
    PdlConfig pdl(dim3(s.n_heads, static_cast<unsigned>(s.n_q), static_cast<unsigned>(c.n_seqs)), dim3(32), stream);
    cudaError_t e;
    if (c.head_dim == 64)
        e = s.dtype == SP_BF16 ? cudaLaunchKernelEx(&pdl.cfg, cache_shared_simple_kernel<true, 64>, a) : cudaLaunchKernelEx(&pdl.cfg, cache_shared_simple_kernel<false, 64>, a);
    else
        e = s.dtype == SP_BF16 ? cudaLaunchKernelEx(&pdl.cfg, cache_shared_simple_kernel<true, 128>, a) : cudaLaunchKernelEx(&pdl.cfg, cache_shared_simple_kernel<false, 128>, a);
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

}  // namespace sp
