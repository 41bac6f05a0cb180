// Norms of queries and keys for each head and the rotation by position, in one pass.
//
// Mathematics: y = x * rsqrt(mean x^2 + eps) * w over a head's D values (where w is given), then the
// first `rotary` of them in pairs (a, b) -> (a cos - b sin, b cos + a sin), the angle being
// place * freq[pair].  Everything is binary32 between the 16-bit loads and the one rounding at the end.
// The angle's product and its reduction to a turn are binary64: at place 10^6 a binary32 product is
// off by up to 2^-5 radians, which an output in 16 bits shows.
//
// Bound by memory: 4 bytes a value, read once and written once.  All heads of a token turn by the
// same angles, so a block takes whole tokens, works their cosines out once into shared memory and
// uses them for every head; a head is D / 16 lanes of 16 values, whose two 16-byte pieces are the
// partners of one another (halves) or neighbours (pairs), so that no value changes lanes but in the
// sum of squares.
#include <algorithm>

#include "sp_device.cuh"
#include "sp_internal.h"

namespace sp {

namespace {

constexpr int kRotaryThreads = 256;
constexpr int kMostTokens = 8;  // of a block

struct RotaryArgs {
    const uint16_t *Q, *K, *q_weight, *k_weight;
    uint16_t *Q_out, *K_out;
    sp_strides q, k, q_out, k_out;
    const int32_t *start;
    const float *freq;
    int64_t n_tokens, total;  // of a sequence, of all
    int heads, kv_heads, head_dim, rotary;
    int tokens, head_share;  // of a block
    float eps;
    bool pairs;
};

// cos and sin of place * freq.
__device__ __forceinline__ float2 turn(int64_t place, float freq) {
    double t = static_cast<double>(place) * static_cast<double>(freq) * 0.15915494309189535;  // turns
    t -= rint(t);
    float2 cs;
    sincospif(static_cast<float>(2.0 * t), &cs.y, &cs.x);
    return cs;
}

template <bool BF16>
__device__ __forceinline__ uint32_t pack2(float a, float b) {
    if constexpr (BF16) {
        const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    } else {
        const __half2 h = __floats2half2_rn(a, b);
        return *reinterpret_cast<const uint32_t *>(&h);
    }
}
template <bool BF16>
__device__ __forceinline__ float widen(uint16_t v) {
    if constexpr (BF16) return __uint_as_float(uint32_t(v) << 16);
    else return __half2float(__ushort_as_half(v));
}
template <bool BF16>
__device__ __forceinline__ uint16_t narrow(float v) {
    if constexpr (BF16) return __bfloat16_as_ushort(__float2bfloat16_rn(v));
    else return __half_as_ushort(__float2half_rn(v));
}

}  // namespace

// Heads of D values whose pieces are 16-byte aligned; PAIRS, or halves with rotary a multiple of 16.
template <bool BF16, int D, bool PAIRS>
__global__ void __launch_bounds__(kRotaryThreads)
qk_rotary_kernel(const __grid_constant__ RotaryArgs a) {
    constexpr int kLanes = D / 16, kRows = kRotaryThreads / kLanes;
    __shared__ float2 angle[kMostTokens][D / 2];
    pdl_launch_dependents();
    pdl_wait();
    const int64_t token0 = int64_t(blockIdx.x) * a.tokens;
    const int tokens = static_cast<int>(min(int64_t(a.tokens), a.total - token0));
    const int lane = threadIdx.x % kLanes, row = threadIdx.x / kLanes;
    const int head0 = blockIdx.y * a.head_share, heads = min(a.head_share, a.heads + a.kv_heads - head0);
    const int items = tokens * heads;
    // where the lane's two pieces of 8 lie in a head
    const int half = a.rotary / 2, units = PAIRS ? 0 : half / 8;
    const bool halves = !PAIRS && lane < units;
    const int at0 = halves ? lane * 8 : lane * 16, at1 = halves ? at0 + half : at0 + 8;
    uint4 x0, x1;
    auto load = [&](int item) {
        const int t = item / heads, h = head0 + item % heads;
        const int64_t token = token0 + t, seq = token / a.n_tokens, i = token % a.n_tokens;
        const uint16_t *p = h < a.heads ? a.Q + seq * a.q.seq + i * a.q.token + h * a.q.head
                                        : a.K + seq * a.k.seq + i * a.k.token + (h - a.heads) * a.k.head;
        x0 = *reinterpret_cast<const uint4 *>(p + at0);
        x1 = *reinterpret_cast<const uint4 *>(p + at1);
    };
    if (row < items) load(row);
    for (int at = threadIdx.x; at < tokens * (D / 2); at += kRotaryThreads) {
        const int t = at / (D / 2), k = at % (D / 2);
        const int64_t token = token0 + t, seq = token / a.n_tokens;
        if (k < half) angle[t][k] = turn(a.start[seq] + token % a.n_tokens, a.freq[k]);
    }
    __syncthreads();
    for (int item = row; item < items; item += kRows) {
        const int t = item / heads, h = head0 + item % heads;
        const uint32_t p0[4] = {x0.x, x0.y, x0.z, x0.w}, p1[4] = {x1.x, x1.y, x1.z, x1.w};
        if (item + kRows < items) load(item + kRows);
        float u[8], v[8];
        unpack8<BF16>(p0, u);
        unpack8<BF16>(p1, v);
        const uint16_t *w = h < a.heads ? a.q_weight : a.k_weight;
        if (w != nullptr) {
            float sum = 0.0f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(u[i], u[i], fmaf(v[i], v[i], sum));
            const unsigned mask = kLanes == 32 ? kFullWarp : ((1u << kLanes) - 1u) << ((threadIdx.x & 31) / kLanes * kLanes);
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
            const float f = rsqrtf(sum * (1.0f / D) + a.eps);
            const uint4 w0 = *reinterpret_cast<const uint4 *>(w + at0), w1 = *reinterpret_cast<const uint4 *>(w + at1);
            const uint32_t q0[4] = {w0.x, w0.y, w0.z, w0.w}, q1[4] = {w1.x, w1.y, w1.z, w1.w};
            float g0[8], g1[8];
            unpack8<BF16>(q0, g0);
            unpack8<BF16>(q1, g1);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                u[i] *= f * g0[i];
                v[i] *= f * g1[i];
            }
        }
        // what is not turned stays as it is: a product with 0 would let an infinity through
        const float4 *cs = reinterpret_cast<const float4 *>(&angle[t][lane * 8]);
        auto rotate = [](float &a, float &b, float cos, float sin) {
            const float y = a * cos - b * sin;
            b = b * cos + a * sin;
            a = y;
        };
        if (PAIRS ? lane * 8 < half : lane < units) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const float4 c = cs[i];  // of pairs 2i and 2i + 1
                if constexpr (PAIRS) {
                    float *s = i < 2 ? u + 4 * i : v + 4 * (i - 2);
                    if (lane * 8 + 2 * i < half) rotate(s[0], s[1], c.x, c.y);
                    if (lane * 8 + 2 * i + 1 < half) rotate(s[2], s[3], c.z, c.w);
                } else {
                    rotate(u[2 * i], v[2 * i], c.x, c.y);
                    rotate(u[2 * i + 1], v[2 * i + 1], c.z, c.w);
                }
            }
        }
        uint32_t y0[4], y1[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            y0[i] = pack2<BF16>(u[2 * i], u[2 * i + 1]);
            y1[i] = pack2<BF16>(v[2 * i], v[2 * i + 1]);
        }
        const int64_t token = token0 + t, seq = token / a.n_tokens, i = token % a.n_tokens;
        uint16_t *out = h < a.heads ? a.Q_out + seq * a.q_out.seq + i * a.q_out.token + h * a.q_out.head
                                    : a.K_out + seq * a.k_out.seq + i * a.k_out.token + (h - a.heads) * a.k_out.head;
        *reinterpret_cast<uint4 *>(out + at0) = make_uint4(y0[0], y0[1], y0[2], y0[3]);
        *reinterpret_cast<uint4 *>(out + at1) = make_uint4(y1[0], y1[1], y1[2], y1[3]);
    }
}

// Any even head size up to 256, any alignment: a warp a head, a lane a value at a time.
template <bool BF16>
__global__ void __launch_bounds__(kRotaryThreads)
qk_rotary_any_kernel(const __grid_constant__ RotaryArgs a) {
    __shared__ float2 angle[kMostTokens][128];
    __shared__ float value[kRotaryThreads / 32][256];
    pdl_launch_dependents();
    pdl_wait();
    const int64_t token0 = int64_t(blockIdx.x) * a.tokens;
    const int tokens = static_cast<int>(min(int64_t(a.tokens), a.total - token0));
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, half = a.rotary / 2, D = a.head_dim;
    const int head0 = blockIdx.y * a.head_share, heads = min(a.head_share, a.heads + a.kv_heads - head0);
    for (int at = threadIdx.x; at < tokens * half; at += kRotaryThreads) {
        const int64_t token = token0 + at / half, seq = token / a.n_tokens;
        angle[at / half][at % half] = turn(a.start[seq] + token % a.n_tokens, a.freq[at % half]);
    }
    __syncthreads();
    for (int item = warp; item < tokens * heads; item += kRotaryThreads / 32) {
        const int t = item / heads, h = head0 + item % heads;
        const int64_t token = token0 + t, seq = token / a.n_tokens, i = token % a.n_tokens;
        const bool is_q = h < a.heads;
        const uint16_t *x = is_q ? a.Q + seq * a.q.seq + i * a.q.token + h * a.q.head
                                 : a.K + seq * a.k.seq + i * a.k.token + (h - a.heads) * a.k.head;
        uint16_t *out = is_q ? a.Q_out + seq * a.q_out.seq + i * a.q_out.token + h * a.q_out.head
                             : a.K_out + seq * a.k_out.seq + i * a.k_out.token + (h - a.heads) * a.k_out.head;
        const uint16_t *w = is_q ? a.q_weight : a.k_weight;
        float sum = 0.0f;
        for (int d = lane; d < D; d += 32) {
            const float v = widen<BF16>(x[d]);
            value[warp][d] = v;
            sum = fmaf(v, v, sum);
        }
        if (w != nullptr) {
#pragma unroll
            for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFullWarp, sum, o);
            const float f = rsqrtf(sum / D + a.eps);
            for (int d = lane; d < D; d += 32) value[warp][d] *= f * widen<BF16>(w[d]);
        }
        __syncwarp();
        for (int d = lane; d < D; d += 32) {
            float y = value[warp][d];
            if (d < a.rotary) {
                const bool second = a.pairs ? d & 1 : d >= half;
                const float2 cs = angle[t][a.pairs ? d >> 1 : second ? d - half : d];
                const float other = value[warp][a.pairs ? d ^ 1 : second ? d - half : d + half];
                y = second ? y * cs.x + other * cs.y : y * cs.x - other * cs.y;
            }
            out[d] = narrow<BF16>(y);
        }
        __syncwarp();
    }
}

static bool pieces16(const void *p, const sp_strides &s) {
    return aligned16(p) && s.seq % 8 == 0 && s.token % 8 == 0 && s.head % 8 == 0;
}

sp_status launch_qk_rotary(const QkRotary &r, cudaStream_t stream) {
    RotaryArgs a = {};
    a.Q = static_cast<const uint16_t *>(r.Q);
    a.K = static_cast<const uint16_t *>(r.K);
    a.Q_out = static_cast<uint16_t *>(r.Q_out);
    a.K_out = static_cast<uint16_t *>(r.K_out);
    a.q_weight = static_cast<const uint16_t *>(r.q_weight);
    a.k_weight = static_cast<const uint16_t *>(r.k_weight);
    a.q = r.q;
    a.k = r.k;
    a.q_out = r.q_out;
    a.k_out = r.k_out;
    a.start = r.start;
    a.freq = r.freq;
    a.n_tokens = r.n_tokens;
    a.total = r.n_seqs * r.n_tokens;
    a.heads = r.n_heads;
    a.kv_heads = r.n_kv_heads;
    a.head_dim = r.head_dim;
    a.rotary = r.rotary;
    a.eps = r.eps;
    a.pairs = r.pairs;
    const bool fast = (r.head_dim == 64 || r.head_dim == 128) && (r.pairs || r.rotary % 16 == 0) &&
                      pieces16(r.Q, r.q) && pieces16(r.K, r.k) && pieces16(r.Q_out, r.q_out) && pieces16(r.K_out, r.k_out) &&
                      aligned16(r.q_weight) && aligned16(r.k_weight);
    // Whole tokens, several to a block once the device is full of blocks; few tokens are shared out by
    // heads instead, each block working the angles out for itself.
    const int heads = a.heads + a.kv_heads, rows = fast ? kRotaryThreads / (r.head_dim / 16) : kRotaryThreads / 32;
    a.tokens = static_cast<int>(std::max(int64_t(1), std::min(int64_t(kMostTokens), a.total / (148 * 8))));
    a.head_share = heads;
    while (a.head_share > rows && a.total * ((heads + a.head_share - 1) / a.head_share) < 148) a.head_share = (a.head_share + 1) / 2;
    const int64_t blocks = (a.total + a.tokens - 1) / a.tokens;
    PdlConfig pdl(dim3(static_cast<unsigned>(blocks), (heads + a.head_share - 1) / a.head_share), dim3(kRotaryThreads), stream);
    const bool bf16 = r.dtype == SP_BF16;
    cudaError_t e;
#define SP_LAUNCH(D, P) \
    e = bf16 ? cudaLaunchKernelEx(&pdl.cfg, qk_rotary_kernel<true, D, P>, a) : cudaLaunchKernelEx(&pdl.cfg, qk_rotary_kernel<false, D, P>, a)
    if (!fast) e = bf16 ? cudaLaunchKernelEx(&pdl.cfg, qk_rotary_any_kernel<true>, a) : cudaLaunchKernelEx(&pdl.cfg, qk_rotary_any_kernel<false>, a);
    else if (r.head_dim == 64 && r.pairs) SP_LAUNCH(64, true);
    else if (r.head_dim == 64) SP_LAUNCH(64, false);
    else if (r.pairs) SP_LAUNCH(128, true);
    else SP_LAUNCH(128, false);
#undef SP_LAUNCH
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

}  // namespace sp
