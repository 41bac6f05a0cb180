// Entry points for serving a pruned model (4-bit weights, 8-bit key/value cache): argument
// validation on the host and dispatch; nothing here synchronises unless the header says so.
#include <algorithm>
#include <cmath>

#include "sp_api.h"
#include "sp_tma.cuh"

namespace sp {

static WaitReader g_wait_readers[16];
static int g_wait_reader_count = 0;

void register_wait_reader(WaitReader reader) {
    if (g_wait_reader_count < 16) g_wait_readers[g_wait_reader_count++] = reader;
}

// The driver's tensor-map encoder, looked up once (the library does not link the driver).
static PFN_cuTensorMapEncodeTiled_v12000 tensor_map_encoder() {
    static const PFN_cuTensorMapEncodeTiled_v12000 fn = [] {
        void *p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            p = nullptr;
        return reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
    }();
    return fn;
}

static cudaError_t encode_tiles(CUtensorMap *map, CUtensorMapDataType type, int element_bytes, const void *base,
                                int64_t rows, int64_t row_elements, int64_t pitch_bytes, int box_rows,
                                int box_bytes = 128) {
    const auto encode = tensor_map_encoder();
    if (encode == nullptr) return cudaErrorNotSupported;
    const cuuint64_t dims[2] = {static_cast<cuuint64_t>(row_elements), static_cast<cuuint64_t>(rows)};
    const cuuint64_t strides[1] = {static_cast<cuuint64_t>(pitch_bytes)};
    const cuuint32_t box[2] = {static_cast<cuuint32_t>(box_bytes / element_bytes), static_cast<cuuint32_t>(box_rows)};
    const cuuint32_t step[2] = {1, 1};
    const CUresult r = encode(map, type, 2, const_cast<void *>(base), dims, strides, box, step,
                              CU_TENSOR_MAP_INTERLEAVE_NONE,
                              box_bytes == 128  ? CU_TENSOR_MAP_SWIZZLE_128B
                              : box_bytes == 64 ? CU_TENSOR_MAP_SWIZZLE_64B
                                                : CU_TENSOR_MAP_SWIZZLE_NONE,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE);
    return r == CUDA_SUCCESS ? cudaSuccess : cudaErrorInvalidValue;
}
cudaError_t encode_byte_tiles(CUtensorMap *map, const void *base, int64_t rows, int64_t row_bytes, int64_t pitch,
                              int box_rows) {
    return encode_tiles(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, base, rows, row_bytes, pitch, box_rows);
}

cudaError_t encode_byte_rows(CUtensorMap *map, const void *base, int64_t rows, int row_bytes, int box_rows) {
    return encode_tiles(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 1, base, rows, row_bytes, row_bytes, box_rows, row_bytes);
}
cudaError_t encode_scale_tiles(CUtensorMap *map, const void *base, int64_t rows, int box_rows) {
    return encode_tiles(map, CU_TENSOR_MAP_DATA_TYPE_UINT32, 4, base, rows, 128, 512, box_rows, 512);
}
cudaError_t encode_half_tiles(CUtensorMap *map, const void *base, int64_t rows, int64_t cols, int64_t ld, int box_rows) {
    return encode_tiles(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, 2, base, rows, cols, ld * 2, box_rows);
}

constexpr int64_t kMaxMx4Side = int64_t(1) << 30;  // rows, columns and tokens of a 4-bit product

// Whether a product takes the kernels that tile over tokens: when they are more than the columns of
// one mma of the streaming kernel.  bf16, 4096 columns: 8 tokens there against 9 in tiles take 6.9 and
// 9.1 us for 4096 rows, 14.4 and 18.0 for 14336.  With 4-bit activations they take 7.2 and 9.0, but
// 15.5 and 12.8: the rule does not tell the two modes apart, and large matrices lose by it there.
// (With two such columns, at 16 tokens, the streaming kernel took 9.3 against 9.9 and 22.8 against
// 18.6, and is not kept for the small difference.)
static bool takes_tiles(int64_t n_tokens) { return n_tokens > kMx4StreamTokens; }

static sp_status check_codes(const void *codes, int64_t ldc, const void *scales, int64_t n_cols) {
    if (codes == nullptr || scales == nullptr) return SP_ERR_INVALID_ARG;
    if (!aligned16(codes) || !aligned16(scales)) return SP_ERR_INVALID_ARG;
    if (ldc % 16 != 0 || ldc < (n_cols + 31) / 32 * 16) return SP_ERR_SHAPE;
    return SP_OK;
}

constexpr int64_t kMaxCacheTokens = int64_t(1) << 30;  // of a sequence

static sp_status check_cache(const sp_cache *c) {
    if (c == nullptr) return SP_ERR_INVALID_ARG;
    if (c->n_blocks < 0 || c->n_seqs < 0 || c->table_cols < 0 || c->n_kv_heads < 1) return SP_ERR_INVALID_ARG;
    if (c->head_dim != 64 && c->head_dim != 128) return SP_ERR_SHAPE;
    if (c->block_tokens != 16 && c->block_tokens != 32 && c->block_tokens != 64) return SP_ERR_SHAPE;
    if (c->ld_table < c->table_cols || c->n_kv_heads > 65535 || c->n_seqs > 32767) return SP_ERR_SHAPE;
    if (c->table_cols > kMaxCacheTokens / c->block_tokens) return SP_ERR_SHAPE;
    if (c->n_seqs > 0 && c->table_cols > 0 && c->table == nullptr) return SP_ERR_INVALID_ARG;
    if (c->n_blocks > 0 && (c->k == nullptr || c->v == nullptr || c->k_scale == nullptr || c->v_scale == nullptr))
        return SP_ERR_INVALID_ARG;
    if (!aligned16(c->k) || !aligned16(c->v)) return SP_ERR_INVALID_ARG;
    return SP_OK;
}

}  // namespace sp

using namespace sp;

extern "C" {

int64_t sp_mx4_scale_bytes(int64_t n_rows, int64_t n_cols) {
    if (n_rows <= 0 || n_cols <= 0 || n_rows > kMaxMx4Side || n_cols > kMaxMx4Side) return 0;
    return (n_rows + 127) / 128 * ((n_cols + 127) / 128) * 512;
}

sp_status sp_mx4_quantize(const void *W, sp_dtype dtype, int64_t n_rows, int64_t n_cols, int64_t ldw,
                          const uint32_t *mask, uint8_t *codes, int64_t ldc, uint8_t *scales, sp_stream stream) {
    SP_CALL_RANGE();
    if (!valid_dtype(dtype)) return SP_ERR_DTYPE;
    if (n_rows < 0 || n_cols < 0) return SP_ERR_INVALID_ARG;
    if (n_rows > kMaxMx4Side || n_cols > kMaxMx4Side || ldw < n_cols) return SP_ERR_SHAPE;
    if (n_rows == 0 || n_cols == 0) return SP_OK;
    if (W == nullptr) return SP_ERR_INVALID_ARG;
    sp_status st = check_codes(codes, ldc, scales, n_cols);
    if (st != SP_OK) return st;
    return launch_mx4_quantize(W, dtype, n_rows, n_cols, ldw, mask, codes, ldc, scales, static_cast<cudaStream_t>(stream));
}

sp_status sp_mx4_dequantize(const uint8_t *codes, int64_t ldc, const uint8_t *scales, int64_t n_rows, int64_t n_cols,
                            sp_dtype dtype, void *W_out, int64_t ldo, sp_stream stream) {
    SP_CALL_RANGE();
    if (!valid_dtype(dtype)) return SP_ERR_DTYPE;
    if (n_rows < 0 || n_cols < 0) return SP_ERR_INVALID_ARG;
    if (n_rows > kMaxMx4Side || n_cols > kMaxMx4Side || ldo < n_cols) return SP_ERR_SHAPE;
    if (n_rows == 0 || n_cols == 0) return SP_OK;
    if (W_out == nullptr) return SP_ERR_INVALID_ARG;
    sp_status st = check_codes(codes, ldc, scales, n_cols);
    if (st != SP_OK) return st;
    return launch_mx4_dequantize(codes, ldc, scales, n_rows, n_cols, dtype, W_out, ldo, static_cast<cudaStream_t>(stream));
}

sp_status sp_mx4_linear_workspace(int64_t n_tokens, int64_t n_rows, int64_t n_cols, int mode, int64_t *bytes) {
    if (bytes == nullptr || n_tokens < 0 || n_rows < 0 || n_cols < 0) return SP_ERR_INVALID_ARG;
    if (mode != SP_MX4_A16 && mode != SP_MX4_A4) return SP_ERR_INVALID_ARG;
    if (n_tokens > kMaxMx4Side || n_rows > kMaxMx4Side || n_cols > kMaxMx4Side) return SP_ERR_SHAPE;
    *bytes = 0;
    if (n_rows > 0 && n_cols > 0 && takes_tiles(n_tokens))
        *bytes = mode == SP_MX4_A4 ? mx4_gemm_workspace(n_tokens, n_cols) : mx4_gemm16_workspace(n_tokens, n_cols);
    return SP_OK;
}

sp_status sp_mx4_linear(const void *X, sp_dtype dtype, int64_t n_tokens, int64_t ldx, const uint8_t *codes, int64_t ldc,
                        const uint8_t *scales, int64_t n_rows, int64_t n_cols, int mode, void *Y, int64_t ldy,
                        void *workspace, int64_t workspace_bytes, sp_stream stream) {
    SP_CALL_RANGE();
    if (!valid_dtype(dtype)) return SP_ERR_DTYPE;
    int64_t need = 0;
    sp_status st = sp_mx4_linear_workspace(n_tokens, n_rows, n_cols, mode, &need);
    if (st != SP_OK) return st;
    if (n_cols < 1 || ldx < n_cols || ldy < n_rows) return SP_ERR_SHAPE;
    if (n_tokens == 0 || n_rows == 0) return SP_OK;
    if (X == nullptr || Y == nullptr) return SP_ERR_INVALID_ARG;
    st = check_codes(codes, ldc, scales, n_cols);
    if (st != SP_OK) return st;
    if (mode == SP_MX4_A16 && mx4_gemm16_reads(X, ldx)) need = 0;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))) return SP_ERR_INVALID_ARG;
    const Mx4Product p{X, n_tokens, ldx, codes, ldc, scales, n_rows, n_cols, Y, ldy, dtype, mode == SP_MX4_A4};
    if (takes_tiles(n_tokens))
        return p.quantize_x ? launch_mx4_gemm(p, workspace, static_cast<cudaStream_t>(stream))
                            : launch_mx4_gemm16(p, workspace, static_cast<cudaStream_t>(stream));
    return launch_mx4_stream(p, static_cast<cudaStream_t>(stream));
}

sp_status sp_cache_append(const sp_cache *cache, const void *K, const sp_strides *k_strides, const void *V,
                          const sp_strides *v_strides, sp_dtype dtype, int64_t n_new, const int32_t *start,
                          const int32_t *count, sp_stream stream) {
    SP_CALL_RANGE();
    sp_status st = check_cache(cache);
    if (st != SP_OK) return st;
    if (!valid_dtype(dtype)) return SP_ERR_DTYPE;
    if (n_new < 0 || k_strides == nullptr || v_strides == nullptr) return SP_ERR_INVALID_ARG;
    if (n_new > kMaxCacheTokens) return SP_ERR_SHAPE;
    if (n_new == 0 || cache->n_seqs == 0 || cache->table_cols == 0) return SP_OK;
    if (K == nullptr || V == nullptr || start == nullptr) return SP_ERR_INVALID_ARG;
    return launch_cache_append(*cache, K, *k_strides, V, *v_strides, dtype, n_new, start, count,
                               static_cast<cudaStream_t>(stream));
}

sp_status sp_cache_attention_workspace(const sp_cache *cache, int64_t n_q, int n_heads, int64_t max_len, int want_acc,
                                       int64_t *bytes) {
    sp_status st = check_cache(cache);
    if (st != SP_OK) return st;
    if (bytes == nullptr || n_q < 0 || n_heads < 1 || max_len < 0) return SP_ERR_INVALID_ARG;
    if (n_heads % cache->n_kv_heads != 0 || max_len > kMaxCacheTokens) return SP_ERR_SHAPE;
    // rows share blocks of at most 16; their least launch has a block for each
    const int64_t group = n_heads / cache->n_kv_heads;
    if (n_q > 8192 / group || cache->n_kv_heads * ((n_q * group + 7) / 8) > 65535) return SP_ERR_SHAPE;
    *bytes = cache_attention_workspace(*cache, n_q, n_heads, max_len, want_acc != 0);
    return SP_OK;
}

sp_status sp_cache_attention(const sp_cache *cache, const void *Q, const sp_strides *q_strides, sp_dtype dtype,
                             int64_t n_q, int n_heads, const int32_t *lens, int64_t max_len, float scale, void *O,
                             const sp_strides *o_strides, float *lse, const float *acc_in, float *acc_out,
                             int64_t ld_acc, void *workspace, int64_t workspace_bytes, sp_stream stream) {
    SP_CALL_RANGE();
    int64_t need = 0;
    sp_status st = sp_cache_attention_workspace(cache, n_q, n_heads, max_len, acc_out != nullptr, &need);
    if (st != SP_OK) return st;
    if (!valid_dtype(dtype)) return SP_ERR_DTYPE;
    if (q_strides == nullptr || o_strides == nullptr || !std::isfinite(scale)) return SP_ERR_INVALID_ARG;
    if (acc_out != nullptr && ld_acc < max_len) return SP_ERR_SHAPE;
    if (cache->n_seqs == 0 || (n_q == 0 && acc_out == nullptr)) return SP_OK;
    if ((n_q > 0 && (Q == nullptr || O == nullptr)) || lens == nullptr) return SP_ERR_INVALID_ARG;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))) return SP_ERR_INVALID_ARG;
    return launch_cache_attention(*cache, Q, *q_strides, dtype, n_q, n_heads, lens, max_len, scale, O, *o_strides, lse,
                                  acc_in, acc_out, ld_acc, workspace, static_cast<cudaStream_t>(stream));
}

sp_status sp_cache_evict(const sp_cache *src, const int32_t *lens, int64_t max_len, const float *acc, int64_t ld_acc,
                         int64_t budget, int64_t recent, const sp_cache *dst, int32_t *kept_out, float *acc_out,
                         int64_t ld_acc_out, int32_t *lens_out, sp_stream stream) {
    SP_CALL_RANGE();
    sp_status st = check_cache(src);
    if (st == SP_OK) st = check_cache(dst);
    if (st != SP_OK) return st;
    if (max_len < 0 || budget < 0 || recent < 0) return SP_ERR_INVALID_ARG;
    if (src->n_kv_heads != dst->n_kv_heads || src->head_dim != dst->head_dim || src->block_tokens != dst->block_tokens ||
        src->n_seqs != dst->n_seqs)
        return SP_ERR_SHAPE;
    if (max_len > kMaxCacheTokens || budget > kMaxCacheTokens || ld_acc < max_len) return SP_ERR_SHAPE;
    if (dst->table_cols < (budget + dst->block_tokens - 1) / dst->block_tokens) return SP_ERR_SHAPE;
    if (acc_out != nullptr && ld_acc_out < budget) return SP_ERR_SHAPE;
    if (src->n_seqs == 0) return SP_OK;
    if (lens == nullptr || (acc == nullptr && max_len > 0) || (kept_out == nullptr && budget > 0)) return SP_ERR_INVALID_ARG;
    return launch_cache_evict(*src, lens, max_len, acc, ld_acc, budget, recent, *dst, kept_out, acc_out, ld_acc_out,
                              lens_out, static_cast<cudaStream_t>(stream));
}

sp_status sp_qk_norm_rotary(const void *Q, const sp_strides *q_strides, int n_heads, const void *K,
                            const sp_strides *k_strides, int n_kv_heads, sp_dtype dtype, int64_t n_seqs, int64_t n_tokens,
                            int head_dim, const void *q_weight, const void *k_weight, float eps, const int32_t *start,
                            const float *freq, int rotary, int pairs, void *Q_out, const sp_strides *q_out_strides,
                            void *K_out, const sp_strides *k_out_strides, sp_stream stream) {
    SP_CALL_RANGE();
    if (!valid_dtype(dtype)) return SP_ERR_DTYPE;
    if (n_heads < 0 || n_kv_heads < 0 || n_seqs < 0 || n_tokens < 0) return SP_ERR_INVALID_ARG;
    if (head_dim < 2 || head_dim > 256 || head_dim % 2 != 0 || rotary < 0 || rotary > head_dim || rotary % 2 != 0)
        return SP_ERR_SHAPE;
    if (n_heads > 65535 - n_kv_heads || (n_seqs > 0 && n_tokens > 0x7fffffff / n_seqs)) return SP_ERR_SHAPE;
    if (!std::isfinite(eps) || eps < 0.0f) return SP_ERR_INVALID_ARG;
    if (n_heads + n_kv_heads == 0 || n_seqs == 0 || n_tokens == 0) return SP_OK;
    if (n_heads > 0 && (Q == nullptr || Q_out == nullptr || q_strides == nullptr || q_out_strides == nullptr)) return SP_ERR_INVALID_ARG;
    if (n_kv_heads > 0 && (K == nullptr || K_out == nullptr || k_strides == nullptr || k_out_strides == nullptr)) return SP_ERR_INVALID_ARG;
    if (rotary > 0 && (start == nullptr || freq == nullptr)) return SP_ERR_INVALID_ARG;
    const sp_strides none = {};
    const QkRotary r{Q, K, q_weight, k_weight, Q_out, K_out, n_heads > 0 ? *q_strides : none, n_kv_heads > 0 ? *k_strides : none,
                     n_heads > 0 ? *q_out_strides : none, n_kv_heads > 0 ? *k_out_strides : none, dtype, n_seqs, n_tokens,
                     n_heads, n_kv_heads, head_dim, rotary, start, freq, eps, pairs != 0};
    return launch_qk_rotary(r, static_cast<cudaStream_t>(stream));
}

static sp_status check_pages(const sp_cache *c) {
    sp_status st = check_cache(c);
    if (st == SP_OK && c->n_blocks > (1 << 30)) st = SP_ERR_SHAPE;
    return st;
}

sp_status sp_cache_fork_workspace(const sp_cache *cache, int64_t n, int64_t *bytes) {
    sp_status st = check_pages(cache);
    if (st != SP_OK) return st;
    if (bytes == nullptr || n < 0) return SP_ERR_INVALID_ARG;
    if (n > (1 << 24)) return SP_ERR_SHAPE;
    *bytes = cache_fork_workspace(*cache, n);
    return SP_OK;
}

sp_status sp_cache_fork(const sp_cache *cache, int32_t *refs, const int32_t *dst, const int32_t *src, int64_t n,
                        void *workspace, int64_t workspace_bytes, sp_stream stream) {
    SP_CALL_RANGE();
    int64_t need = 0;
    sp_status st = sp_cache_fork_workspace(cache, n, &need);
    if (st != SP_OK) return st;
    if (n == 0 || cache->n_seqs == 0 || cache->table_cols == 0) return SP_OK;
    if (dst == nullptr || (refs == nullptr && cache->n_blocks > 0)) return SP_ERR_INVALID_ARG;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))) return SP_ERR_INVALID_ARG;
    return launch_cache_fork(*cache, refs, dst, src, n, workspace, static_cast<cudaStream_t>(stream));
}

sp_status sp_cache_reserve_workspace(const sp_cache *cache, int64_t n_new, int64_t *bytes) {
    sp_status st = check_pages(cache);
    if (st != SP_OK) return st;
    if (bytes == nullptr || n_new < 0) return SP_ERR_INVALID_ARG;
    if (n_new > kMaxCacheTokens) return SP_ERR_SHAPE;
    const int64_t touched = std::min(cache->table_cols, n_new / cache->block_tokens + 2);
    if (cache->n_seqs > 0 && touched > (int64_t(1) << 30) / cache->n_seqs) return SP_ERR_SHAPE;
    *bytes = cache_reserve_workspace(*cache, n_new);
    return SP_OK;
}

sp_status sp_cache_reserve(const sp_cache *cache, int32_t *refs, const int32_t *start, const int32_t *count, int64_t n_new,
                           int32_t *status, void *workspace, int64_t workspace_bytes, sp_stream stream) {
    SP_CALL_RANGE();
    int64_t need = 0;
    sp_status st = sp_cache_reserve_workspace(cache, n_new, &need);
    if (st != SP_OK) return st;
    if (status == nullptr || (refs == nullptr && cache->n_blocks > 0) || (start == nullptr && cache->n_seqs > 0)) return SP_ERR_INVALID_ARG;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))) return SP_ERR_INVALID_ARG;
    return launch_cache_reserve(*cache, refs, start, count, n_new, status, workspace, static_cast<cudaStream_t>(stream));
}

sp_status sp_cache_compact_workspace(const sp_cache *cache, int64_t *bytes) {
    sp_status st = check_pages(cache);
    if (st != SP_OK) return st;
    if (bytes == nullptr) return SP_ERR_INVALID_ARG;
    *bytes = cache_compact_workspace(*cache);
    return SP_OK;
}

sp_status sp_cache_compact(const sp_cache *cache, const int32_t *refs, int32_t *table_out, int64_t ld_table_out,
                           int32_t *refs_out, int32_t *live, void *workspace, int64_t workspace_bytes, sp_stream stream) {
    SP_CALL_RANGE();
    int64_t need = 0;
    sp_status st = sp_cache_compact_workspace(cache, &need);
    if (st != SP_OK) return st;
    if (ld_table_out < cache->table_cols) return SP_ERR_SHAPE;
    if (table_out == cache->table && table_out != nullptr && ld_table_out != cache->ld_table) return SP_ERR_SHAPE;
    if (live == nullptr || (cache->n_blocks > 0 && (refs == nullptr || refs_out == nullptr))) return SP_ERR_INVALID_ARG;
    if (cache->n_seqs > 0 && cache->table_cols > 0 && table_out == nullptr) return SP_ERR_INVALID_ARG;
    if (workspace == nullptr || workspace_bytes < need || !aligned16(workspace)) return SP_ERR_INVALID_ARG;
    return launch_cache_compact(*cache, refs, table_out, ld_table_out, refs_out, live, workspace,
                                static_cast<cudaStream_t>(stream));
}

sp_status sp_cache_attention_shared_workspace(const sp_cache *cache, int64_t n_q, int n_heads, int64_t max_len,
                                              int64_t n_groups, int64_t max_prefix, int64_t max_group, int64_t *bytes) {
    int64_t alone = 0;
    sp_status st = sp_cache_attention_workspace(cache, n_q, n_heads, max_len, 0, &alone);
    if (st != SP_OK) return st;
    if (bytes == nullptr || n_groups < 0 || max_prefix < 0 || max_group < 0) return SP_ERR_INVALID_ARG;
    if (n_groups > 32767 || max_prefix > kMaxCacheTokens || max_group > 32767) return SP_ERR_SHAPE;
    SharedAttention s = {};
    s.n_q = n_q;
    s.n_heads = n_heads;
    s.max_len = max_len;
    s.n_groups = n_groups;
    s.max_prefix = max_prefix;
    s.max_group = max_group;
    if (!cache_shared_fits(*cache, s)) return SP_ERR_SHAPE;
    *bytes = cache_shared_workspace(*cache, s);
    return SP_OK;
}

sp_status sp_cache_attention_shared(const sp_cache *cache, const void *Q, const sp_strides *q_strides, sp_dtype dtype,
                                    int64_t n_q, int n_heads, const int32_t *lens, int64_t max_len,
                                    const int32_t *group_start, int64_t n_groups, const int32_t *prefix,
                                    int64_t max_prefix, int64_t max_group, float scale, void *O,
                                    const sp_strides *o_strides, float *lse, void *workspace, int64_t workspace_bytes,
                                    sp_stream stream) {
    SP_CALL_RANGE();
    int64_t need = 0;
    sp_status st = sp_cache_attention_shared_workspace(cache, n_q, n_heads, max_len, n_groups, max_prefix, max_group, &need);
    if (st != SP_OK) return st;
    if (!valid_dtype(dtype)) return SP_ERR_DTYPE;
    if (q_strides == nullptr || o_strides == nullptr || !std::isfinite(scale)) return SP_ERR_INVALID_ARG;
    if (cache->n_blocks > 0x7fffffff / (int64_t(cache->n_kv_heads) * cache->block_tokens)) return SP_ERR_SHAPE;
    if (cache->n_seqs == 0 || n_q == 0) return SP_OK;
    if (Q == nullptr || O == nullptr || lens == nullptr) return SP_ERR_INVALID_ARG;
    if (n_groups > 0 && (group_start == nullptr || prefix == nullptr)) return SP_ERR_INVALID_ARG;
    if (need > 0 && (workspace == nullptr || workspace_bytes < need || !aligned16(workspace))) return SP_ERR_INVALID_ARG;
    const SharedAttention s{Q, *q_strides, *o_strides, dtype, n_q, max_len, n_groups, max_prefix, max_group, n_heads,
                            lens, group_start, prefix, scale, O, lse};
    return launch_cache_shared(*cache, s, workspace, static_cast<cudaStream_t>(stream));
}

sp_status sp_wait_status(int *expired, int clear) {
    SP_CALL_RANGE();
    if (expired == nullptr) return SP_ERR_INVALID_ARG;
    *expired = 0;
    cudaError_t e = cudaDeviceSynchronize();
    if (e != cudaSuccess) return cuda_fail(e);
    for (int i = 0; i < g_wait_reader_count; ++i) {
        unsigned int n = 0;
        e = g_wait_readers[i](&n, clear != 0);
        if (e != cudaSuccess) return cuda_fail(e);
        *expired += static_cast<int>(n);
    }
    return SP_OK;
}

}  // extern "C"
