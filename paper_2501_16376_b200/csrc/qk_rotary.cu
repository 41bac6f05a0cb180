// Norms of queries and keys for each head and the rotation by position, in one pass.
//
// Mathematics: y = x * rsqrt(mean x^2 + eps) * w over a head's D values (where w is given), then the
// first `rotary` of them in pairs (a, b) -> (a cos - b sin, b cos + a sin), the angle being
// place * freq[pair].  Everything is binary32 between the 16-bit loads and the one rounding at the end.
// The angle's product and its reduction to a turn are binary64: at place 10^6 a binary32 product is
// off by up to 2^-5 radians, which an output in 16 bits shows.
//
// Bound by memory, 4 bytes a value read once and written once, and next to it by the issue slots, which count
// double in a long run: the power limit then takes the clock from 1965 to 1710 MHz.  All heads of a
// token turn by the same angles, so a block takes whole tokens and works their cosines out once into
// shared memory.  A head is D / 16 lanes of 16 values, whose two 16-byte pieces are the partners of one another
// (halves) or hold whole pairs, so that no value changes lanes but in the sum of squares; pairs of
// values share an instruction, and are laid side by side for that as they are widened.  Lanes keep
// their head from token to token, so that addresses, weights and masks cost next to nothing (heads
// and tokens as one list of items took 112 us for the first case below, and 128 in a long run).
// Weights stay in shared memory, in the order of the lanes: in registers they cost a block of the four (111 us).
// Measured (calls replayed from a graph, inputs beyond the L2 cache): 32768 tokens of 40 heads of 128, pairs, normed,
// bf16 107 us (6.3 TB/s, 0.96 of the copy rate), 111 in a long run; the same in halves 107 us; 4 x 2047 tokens of 16 and
// 16 heads of 64, a quarter turned, f16 13 us; 8 tokens 2.6 us, which is the launch.  Halves of 12 (24 values
// turned) in pieces of four: 131 us for the large case.
#include <algorithm>
#include <type_traits>

#include "sp_device.cuh"
#include "sp_internal.h"

namespace sp {

namespace {

constexpr int kRotaryThreads = 256;  // one by one
constexpr int kMostThreads = 320, kFewThreads = 160;  // in pieces; what a block has where a token takes fewer
constexpr int kMostTokens = 8;       // of a block

struct RotaryArgs {
    const uint16_t *Q, *K, *q_weight, *k_weight;
    uint16_t *Q_out, *K_out;
    sp_strides q, k, q_out, k_out;
    const int32_t *start;
    const float *freq;
    int64_t n_tokens, total;  // of a sequence, of all
    int heads, kv_heads, head_dim, rotary;
    int tokens, head_share;  // of a block
    int slots;               // its tokens that are taken at a time
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

// Whether binary32 holds a row's mean of squares with all its bits (always, of binary16); otherwise the row
// is taken times row_scale, and eps times its square.
template <bool BF16>
__device__ __forceinline__ bool plain_mean(float mean) { return !BF16 || (mean > 0x1p-100f && mean < 0x1p126f); }
__device__ __forceinline__ float row_scale(float mean) { return mean > 1.0f ? 0x1p-70f : 0x1p80f; }

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
// kLanes threads keep one head, and take every a.slots-th of the block's tokens.
template <bool BF16, int D, bool PAIRS, int P>
__global__ void __launch_bounds__(kMostThreads, 4)
qk_rotary_kernel(const __grid_constant__ RotaryArgs a) {
    static_assert(P == 8 || (P == 4 && !PAIRS), "pairs are turned in pieces of 8");
    using Piece = typename std::conditional<P == 8, uint4, uint2>::type;
    constexpr int kLanes = D / (2 * P), W = P / 2;
    __shared__ __align__(16) float angle[kMostTokens][2][D / 2];  // cosines, sines
    __shared__ float4 weight[2][2][W / 2][kLanes];  // of queries, keys; of u, v below; four values of a lane
    __shared__ Offsets offset[kMostTokens];
    pdl_launch_dependents();
    pdl_wait();
    const int64_t token0 = int64_t(blockIdx.x) * a.tokens;
    const int tokens = static_cast<int>(min(int64_t(a.tokens), a.total - token0));
    const int lane = threadIdx.x % kLanes, row = threadIdx.x / kLanes, slot = row / a.head_share;
    const int head = blockIdx.y * a.head_share + row - slot * a.head_share;
    const bool is_q = head < a.heads, here = slot < a.slots && head < a.heads + a.kv_heads;
    // Where a lane's two pieces lie in a head: neighbouring lanes' pieces are neighbours.
    const int half = a.rotary / 2, units = PAIRS ? 0 : half / P;
    const bool halves = !PAIRS && lane < units;
    auto piece0 = [&](int l) { return PAIRS || l < units ? l * P : a.rotary + (l - units) * P; };
    auto apart_of = [&](int l) { return PAIRS ? D / 2 : l < units ? half : (kLanes - units) * P; };
    const int at0 = piece0(lane), apart = apart_of(lane);
    // (all tokens together are fewer than 2^31)
    auto place = [&](int t, uint32_t &seq) {
        const uint32_t token = static_cast<uint32_t>(token0) + t, n = static_cast<uint32_t>(a.n_tokens);
        seq = token / n;
        return token - seq * n;
    };
    const uint16_t *in = at0 + (is_q ? a.Q + head * a.q.head : a.K + (head - a.heads) * a.k.head);
    Piece x0, x1;
    auto load = [&](int64_t at) {
        x0 = __ldcs(reinterpret_cast<const Piece *>(in + at));
        x1 = __ldcs(reinterpret_cast<const Piece *>(in + at + apart));
    };
    // the first token's values are on their way before anything else
    int t = here ? slot : tokens;
    if (t < tokens) {
        uint32_t seq;
        const int64_t i = place(t, seq);
        load(is_q ? seq * a.q.seq + i * a.q.token : seq * a.k.seq + i * a.k.token);
    }
#pragma unroll 1
    for (int n = threadIdx.x; n < tokens; n += blockDim.x) {
        uint32_t seq;
        const int64_t i = place(n, seq);
        offset[n] = Offsets{seq * a.q.seq + i * a.q.token, seq * a.k.seq + i * a.k.token,
                            seq * a.q_out.seq + i * a.q_out.token, seq * a.k_out.seq + i * a.k_out.token};
    }
    const uint16_t *w = is_q ? a.q_weight : a.k_weight;
    const bool normed = here && w != nullptr;
#pragma unroll 1
    for (int n = threadIdx.x; n < 2 * W * kLanes; n += blockDim.x) {
        const int l = n % kLanes, i = n / kLanes % (W / 2), second = n / kLanes / (W / 2) & 1, of = n / kLanes / W;
        const uint16_t *from = of == 0 ? a.q_weight : a.k_weight;
        if (from == nullptr) continue;
        from += piece0(l) + (PAIRS ? i * (D / 2) + second : second * apart_of(l) + 4 * i);
        constexpr int kNext = PAIRS ? 2 : 1;
        weight[of][second][i][l] = make_float4(widen<BF16>(from[0]), widen<BF16>(from[kNext]), widen<BF16>(from[2 * kNext]), widen<BF16>(from[3 * kNext]));
    }
    const float4 *wl = &weight[is_q ? 0 : 1][0][0][lane];
    // a warp 32 angles of a token; stored so that a lane's lie four at a time, its neighbours' beside them
#pragma unroll 1
    for (int n = threadIdx.x >> 5; n < tokens * (half > 32 ? 2 : 1); n += blockDim.x >> 5) {
        const int of = half > 32 ? n >> 1 : n, pair = (half > 32 ? (n & 1) * 32 : 0) + (threadIdx.x & 31);
        if (pair < half) {
            uint32_t seq;
            const int64_t i = place(of, seq);
            const float2 cs = turn(a.start[seq] + i, a.freq[pair]);
            const int at = PAIRS || P == 4 ? pair : (pair >> 2 & 1) * (D / 4) + (pair >> 3) * 4 + (pair & 3);
            angle[of][0][at] = cs.x;
            angle[of][1][at] = cs.y;
        }
    }
    __syncthreads();
    uint16_t *out = at0 + (is_q ? a.Q_out + head * a.q_out.head : a.K_out + (head - a.heads) * a.k_out.head);
    const int64_t *offsets = is_q ? &offset[0].q : &offset[0].k;  // and of the output two further on
    while (t < tokens) {
        const uint32_t *p0 = reinterpret_cast<const uint32_t *>(&x0), *p1 = reinterpret_cast<const uint32_t *>(&x1);
        float2 u[W], v[W];  // partners: the halves' values, or the pairs' even and odd ones
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (PAIRS) {
                const uint32_t *p = i < 2 ? p0 + 2 * i : p1 + 2 * (i - 2);
                const float2 first = unpack2<BF16>(p[0]), second = unpack2<BF16>(p[1]);
                u[i] = make_float2(first.x, second.x);
                v[i] = make_float2(first.y, second.y);
            } else {
                u[i] = unpack2<BF16>(p0[i]);
                v[i] = unpack2<BF16>(p1[i]);
            }
        }
        if (t + a.slots < tokens) load(offsets[4 * (t + a.slots)]);
        if (normed) {
            float2 sums = mul2(u[0], u[0]);
#pragma unroll
            for (int i = 1; i < W; ++i) sums = fma2(u[i], u[i], sums);
#pragma unroll
            for (int i = 0; i < W; ++i) sums = fma2(v[i], v[i], sums);
            float sum = sums.x + sums.y;
            const unsigned mask = ((1u << kLanes) - 1u) << ((threadIdx.x & 31) / kLanes * kLanes);
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
            const float mean = sum * (1.0f / D) + a.eps;
            float f = rsqrtf(mean);
            if (!plain_mean<BF16>(mean)) {
                const float by = row_scale(mean);
                sum = 0.0f;
#pragma unroll
                for (int i = 0; i < W; ++i) {
                    u[i] = mul2(u[i], make_float2(by, by));
                    v[i] = mul2(v[i], make_float2(by, by));
                    sum = fmaf(u[i].x, u[i].x, fmaf(u[i].y, u[i].y, fmaf(v[i].x, v[i].x, fmaf(v[i].y, v[i].y, sum))));
                }
#pragma unroll
                for (int o = kLanes / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(mask, sum, o);
                f = rsqrtf(sum * (1.0f / D) + a.eps * by * by);
            }
            const float2 f2 = make_float2(f, f);
#pragma unroll
            for (int i = 0; i < W; i += 2) {
                const float4 gu = wl[i / 2 * kLanes], gv = wl[(W / 2 + i / 2) * kLanes];
                u[i] = mul2(mul2(u[i], f2), make_float2(gu.x, gu.y));
                u[i + 1] = mul2(mul2(u[i + 1], f2), make_float2(gu.z, gu.w));
                v[i] = mul2(mul2(v[i], f2), make_float2(gv.x, gv.y));
                v[i + 1] = mul2(mul2(v[i + 1], f2), make_float2(gv.z, gv.w));
            }
        }
        // what is not turned stays as it is: a product with 0 would let an infinity through
        if (PAIRS ? half > 0 : halves) {
            const float4 *cs = reinterpret_cast<const float4 *>(angle[t][0]) + lane;
#pragma unroll
            for (int i = 0; i < W; i += 2) {
                const float4 c = cs[i / 2 * (D / 16)], s = cs[D / 8 + i / 2 * (D / 16)];
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                    const float2 ck = k == 0 ? make_float2(c.x, c.y) : make_float2(c.z, c.w), sk = k == 0 ? make_float2(s.x, s.y) : make_float2(s.z, s.w);
                    float2 &x = u[i + k], &y = v[i + k];
                    const float2 turned = fma2(x, ck, mul2(y, make_float2(-sk.x, -sk.y))), other = fma2(y, ck, mul2(x, sk));
                    if (!PAIRS || half == D / 2) {
                        x = turned;
                        y = other;
                    } else {
                        const int pair = (i < 2 ? 0 : D / 4) + lane * 4 + 2 * k;
                        if (pair < half) x.x = turned.x, y.x = other.x;
                        if (pair + 1 < half) x.y = turned.y, y.y = other.y;
                    }
                }
            }
        }
        Piece y0, y1;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            if constexpr (PAIRS) {
                uint32_t *y = reinterpret_cast<uint32_t *>(i < 2 ? &y0 : &y1) + 2 * (i & 1);
                y[0] = pack2<BF16>(u[i].x, v[i].x);
                y[1] = pack2<BF16>(u[i].y, v[i].y);
            } else {
                reinterpret_cast<uint32_t *>(&y0)[i] = pack2<BF16>(u[i].x, u[i].y);
                reinterpret_cast<uint32_t *>(&y1)[i] = pack2<BF16>(v[i].x, v[i].y);
            }
        }
        uint16_t *to = out + offsets[4 * t + 2];
        t += a.slots;
        __stcs(reinterpret_cast<Piece *>(to), y0);
        __stcs(reinterpret_cast<Piece *>(to + apart), y1);
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
            const float mean = sum / D + a.eps;
            float f = rsqrtf(mean);
            if (!plain_mean<BF16>(mean)) {
                const float by = row_scale(mean);
                sum = 0.0f;
                for (int d = lane; d < D; d += 32) {
                    const float v = value[warp][d] *= by;
                    sum = fmaf(v, v, sum);
                }
#pragma unroll
                for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(kFullWarp, sum, o);
                f = rsqrtf(sum / D + a.eps * by * by);
            }
            for (int d = lane; d < D; d += 32) value[warp][d] = value[warp][d] * f * widen<BF16>(w[d]);
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
    // A block has all of a token's heads where it has threads for them, and several tokens once the device
    // (1280 threads an SM) is full three times over; few tokens are shared out by heads instead, each block
    // working the angles out for itself.
    const int heads = a.heads + a.kv_heads, lanes = piece > 0 ? r.head_dim / (2 * piece) : 32;
    const int least = piece > 0 ? 64 / lanes : kRotaryThreads / 32;
    a.head_share = piece > 0 ? (heads + (heads * lanes - 1) / kMostThreads) / ((heads * lanes - 1) / kMostThreads + 1) : heads;
    while (a.head_share > least && a.total * ((heads + a.head_share - 1) / a.head_share) < 148) a.head_share = (a.head_share + 1) / 2;
    const int parts = (heads + a.head_share - 1) / a.head_share;
    const int full = 3 * 148 * std::max(1, 1280 / std::max(kFewThreads, a.head_share * lanes));
    a.tokens = static_cast<int>(std::min(int64_t(kMostTokens), (a.total * parts + full - 1) / full));
    a.slots = std::max(1, std::min(a.tokens, kFewThreads / (a.head_share * lanes)));
    const int64_t blocks = (a.total + a.tokens - 1) / a.tokens;
    const int threads = piece > 0 ? (a.slots * a.head_share * lanes + 31) / 32 * 32 : kRotaryThreads;
    PdlConfig pdl(dim3(static_cast<unsigned>(blocks), (heads + a.head_share - 1) / a.head_share), dim3(threads), stream);
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
