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
// partners of one another (halves) or hold whole pairs, so that no value changes lanes but in the sum
// of squares.  Pairs of values share an instruction (one by one, with the lane's pieces side by side
// and 88 registers, the large case below took 150 us: two thirds of the issue slots beside 55 % of the
// memory rate).  Measured (calls replayed from a graph): 32768 tokens of 40 heads of 128, normed, bf16
// 112 us (6.0 TB/s, 0.92 of the copy rate); 4 x 2047 tokens of 32 heads of 64, a quarter turned, f16
// 11 us (6.1 TB/s); 8 tokens 2.5 us, which is the launch.  Halves of 12 (24 values turned) in pieces of
// four: 140 us for the large case.
#include <algorithm>
#include <type_traits>

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

// Where a token's heads begin.
struct Offsets {
    int64_t q, k, q_out, k_out;
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

// Heads of D values in pieces of P, aligned as such; PAIRS (8), or halves with rotary a multiple of 2 P.
template <bool BF16, int D, bool PAIRS, int P>
__global__ void __launch_bounds__(kRotaryThreads, 5)
qk_rotary_kernel(const __grid_constant__ RotaryArgs a) {
    static_assert(P == 8 || (P == 4 && !PAIRS), "pairs are turned in pieces of 8");
    using Piece = typename std::conditional<P == 8, uint4, uint2>::type;
    constexpr int kLanes = D / (2 * P), kRows = kRotaryThreads / kLanes, W = P / 2;
    __shared__ __align__(16) float cosine[kMostTokens][D / 2], sine[kMostTokens][D / 2];
    __shared__ __align__(16) float weight[2][D];
    __shared__ Offsets offset[kMostTokens];
    pdl_launch_dependents();
    pdl_wait();
    const int64_t token0 = int64_t(blockIdx.x) * a.tokens;
    const int tokens = static_cast<int>(min(int64_t(a.tokens), a.total - token0));
    const int lane = threadIdx.x % kLanes, row = threadIdx.x / kLanes;
    const int head0 = blockIdx.y * a.head_share, heads = min(a.head_share, a.heads + a.kv_heads - head0);
    // Where the lane's two pieces lie in a head: neighbouring lanes' pieces are neighbours (with both
    // pieces of a lane side by side, 32768 tokens of 40 heads took 150 us).
    const int half = a.rotary / 2, units = PAIRS ? 0 : half / P;
    const bool halves = !PAIRS && lane < units;
    const int at0 = PAIRS || halves ? lane * P : a.rotary + (lane - units) * P;
    const int at1 = PAIRS ? D / 2 + at0 : halves ? at0 + half : at0 + (kLanes - units) * P;
    // (all tokens together are fewer than 2^31)
    auto place = [&](int t, uint32_t &seq) {
        const uint32_t token = static_cast<uint32_t>(token0) + t, n = static_cast<uint32_t>(a.n_tokens);
        seq = token / n;
        return token - seq * n;
    };
    // a head of a token at a time; the first one's values are on their way before anything else
    int t = 0, h = row;
    auto settle = [&] {
        while (h >= heads) {
            h -= heads;
            ++t;
        }
    };
    Piece x0, x1;
    auto load = [&](int64_t q_at, int64_t k_at) {
        const int at = head0 + h;
        const uint16_t *p = at < a.heads ? a.Q + q_at + at * a.q.head : a.K + k_at + (at - a.heads) * a.k.head;
        x0 = __ldcs(reinterpret_cast<const Piece *>(p + at0));
        x1 = __ldcs(reinterpret_cast<const Piece *>(p + at1));
    };
    settle();
    if (t < tokens) {
        uint32_t seq;
        const int64_t i = place(t, seq);
        load(seq * a.q.seq + i * a.q.token, seq * a.k.seq + i * a.k.token);
    }
    for (int n = threadIdx.x; n < tokens; n += kRotaryThreads) {
        uint32_t seq;
        const int64_t i = place(n, seq);
        offset[n] = Offsets{seq * a.q.seq + i * a.q.token, seq * a.k.seq + i * a.k.token,
                            seq * a.q_out.seq + i * a.q_out.token, seq * a.k_out.seq + i * a.k_out.token};
    }
    for (int at = threadIdx.x; at < tokens * half; at += kRotaryThreads) {
        uint32_t seq;
        const int64_t i = place(at / half, seq);
        const float2 cs = turn(a.start[seq] + i, a.freq[at % half]);
        cosine[at / half][at % half] = cs.x;
        sine[at / half][at % half] = cs.y;
    }
    for (int d = threadIdx.x; d < D; d += kRotaryThreads) {
        if (a.q_weight != nullptr) weight[0][d] = widen<BF16>(a.q_weight[d]);
        if (a.k_weight != nullptr) weight[1][d] = widen<BF16>(a.k_weight[d]);
    }
    __syncthreads();
    while (t < tokens) {
        const int at = head0 + h;
        const bool is_q = at < a.heads;
        const Piece now0 = x0, now1 = x1;
        const uint32_t *p0 = reinterpret_cast<const uint32_t *>(&now0), *p1 = reinterpret_cast<const uint32_t *>(&now1);
        uint16_t *out = is_q ? a.Q_out + offset[t].q_out + at * a.q_out.head : a.K_out + offset[t].k_out + (at - a.heads) * a.k_out.head;
        const float *cos = cosine[t], *sin = sine[t];
        h += kRows;
        settle();
        if (t < tokens) load(offset[t].q, offset[t].k);
        float2 u[W], v[W];
#pragma unroll
        for (int i = 0; i < W; ++i) {
            u[i] = unpack2<BF16>(p0[i]);
            v[i] = unpack2<BF16>(p1[i]);
        }
        if ((is_q ? a.q_weight : a.k_weight) != nullptr) {
            float2 sums = mul2(u[0], u[0]);
#pragma unroll
            for (int i = 1; i < W; ++i) sums = fma2(u[i], u[i], sums);
#pragma unroll
            for (int i = 0; i < W; ++i) sums = fma2(v[i], v[i], sums);
            float sum = sums.x + sums.y;
            const unsigned mask = ((1u << kLanes) - 1u) << ((threadIdx.x & 31) / kLanes * kLanes);
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
            const float f = rsqrtf(sum * (1.0f / D) + a.eps);
            const float4 *w0 = reinterpret_cast<const float4 *>(&weight[is_q ? 0 : 1][at0]), *w1 = reinterpret_cast<const float4 *>(&weight[is_q ? 0 : 1][at1]);
            const float2 f2 = make_float2(f, f);
#pragma unroll
            for (int i = 0; i < W; i += 2) {
                const float4 g0 = w0[i / 2], g1 = w1[i / 2];
                u[i] = mul2(u[i], mul2(make_float2(g0.x, g0.y), f2));
                u[i + 1] = mul2(u[i + 1], mul2(make_float2(g0.z, g0.w), f2));
                v[i] = mul2(v[i], mul2(make_float2(g1.x, g1.y), f2));
                v[i + 1] = mul2(v[i + 1], mul2(make_float2(g1.z, g1.w), f2));
            }
        }
        // what is not turned stays as it is: a product with 0 would let an infinity through
        auto rotate2 = [](float2 &a, float2 &b, float2 c, float2 s) {  // two pairs
            const float2 y = fma2(a, c, mul2(b, make_float2(-s.x, -s.y)));
            b = fma2(b, c, mul2(a, s));
            a = y;
        };
        if constexpr (PAIRS) {
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                float2 *s = i < 2 ? u + 2 * i : v + 2 * (i - 2);
                const int pair = (i < 2 ? 0 : D / 4) + lane * 4 + (i & 1) * 2;
                if (pair < half) {
                    const float2 c = *reinterpret_cast<const float2 *>(cos + pair), sn = *reinterpret_cast<const float2 *>(sin + pair);
                    float2 first = make_float2(s[0].x, s[1].x), second = make_float2(s[0].y, s[1].y);
                    rotate2(first, second, c, sn);
                    s[0] = make_float2(first.x, second.x);
                    if (pair + 1 < half) s[1] = make_float2(first.y, second.y);
                }
            }
        } else if (lane < units) {
#pragma unroll
            for (int i = 0; i < W; ++i)
                rotate2(u[i], v[i], *reinterpret_cast<const float2 *>(cos + lane * P + 2 * i), *reinterpret_cast<const float2 *>(sin + lane * P + 2 * i));
        }
        Piece y0, y1;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            reinterpret_cast<uint32_t *>(&y0)[i] = pack2<BF16>(u[i].x, u[i].y);
            reinterpret_cast<uint32_t *>(&y1)[i] = pack2<BF16>(v[i].x, v[i].y);
        }
        __stcs(reinterpret_cast<Piece *>(out + at0), y0);
        __stcs(reinterpret_cast<Piece *>(out + at1), y1);
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

// Whether every head begins on a boundary of n values (2 n bytes).
static bool pieces(const void *p, const sp_strides &s, int n) {
    return reinterpret_cast<uintptr_t>(p) % (2 * n) == 0 && s.seq % n == 0 && s.token % n == 0 && s.head % n == 0;
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
    const bool whole = r.head_dim == 64 || r.head_dim == 128;
    auto in_pieces = [&](int n) {
        return whole && pieces(r.Q, r.q, n) && pieces(r.K, r.k, n) && pieces(r.Q_out, r.q_out, n) && pieces(r.K_out, r.k_out, n);
    };
    // Values a piece: 8 where the layout and the halves allow it, else 4; else one by one.
    const int piece = in_pieces(8) && (r.pairs || r.rotary % 16 == 0) ? 8 : in_pieces(4) && !r.pairs && r.rotary % 8 == 0 ? 4 : 0;
    // Whole tokens, several to a block once the device is full of blocks; few tokens are shared out by
    // heads instead, each block working the angles out for itself.
    const int heads = a.heads + a.kv_heads, rows = piece > 0 ? kRotaryThreads / (r.head_dim / (2 * piece)) : kRotaryThreads / 32;
    a.tokens = static_cast<int>(std::max(int64_t(1), std::min(int64_t(kMostTokens), a.total / (148 * 8))));
    a.head_share = heads;
    while (a.head_share > rows && a.total * ((heads + a.head_share - 1) / a.head_share) < 148) a.head_share = (a.head_share + 1) / 2;
    const int64_t blocks = (a.total + a.tokens - 1) / a.tokens;
    PdlConfig pdl(dim3(static_cast<unsigned>(blocks), (heads + a.head_share - 1) / a.head_share), dim3(kRotaryThreads), stream);
    const bool bf16 = r.dtype == SP_BF16;
    cudaError_t e;
#define SP_LAUNCH(D, PAIRS, P) \
    e = bf16 ? cudaLaunchKernelEx(&pdl.cfg, qk_rotary_kernel<true, D, PAIRS, P>, a) : cudaLaunchKernelEx(&pdl.cfg, qk_rotary_kernel<false, D, PAIRS, P>, a)
    if (piece == 0) e = bf16 ? cudaLaunchKernelEx(&pdl.cfg, qk_rotary_any_kernel<true>, a) : cudaLaunchKernelEx(&pdl.cfg, qk_rotary_any_kernel<false>, a);
    else if (r.head_dim == 64 && r.pairs) SP_LAUNCH(64, true, 8);
    else if (r.pairs) SP_LAUNCH(128, true, 8);
    else if (r.head_dim == 64 && piece == 8) SP_LAUNCH(64, false, 8);
    else if (r.head_dim == 64) SP_LAUNCH(64, false, 4);
    else if (piece == 8) SP_LAUNCH(128, false, 8);
    else SP_LAUNCH(128, false, 4);
#undef SP_LAUNCH
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

}  // namespace sp
