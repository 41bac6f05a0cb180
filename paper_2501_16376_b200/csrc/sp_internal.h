// Internal declarations shared by the translation units of the library.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

#include "sp_debug.cuh"
#include "swiftprune.h"

namespace sp {

constexpr int kStripChannels = 256;  // channels covered by one warp-wide 16-byte load
constexpr int kMaxSlabs = 128;       // token slabs that own a row of partial sums
constexpr int kTile = 256;           // weights per warp tile (32 lanes x 8)
constexpr int64_t kMaxDin = 1 << 20;

// Status word written by the finalisation kernel.
constexpr int kFlagDegenerate = 1;

constexpr int64_t kEwmaMaxLaunchRows = int64_t(1) << 30;  // rows one EWMA launch can cover
constexpr int kEwmaMaxJobs = 16;                           // weight matrices, likewise

// Scalars produced by finalisation; lives in device memory inside the context.
struct DeviceScalars {
    double S;             // sum_q colsq[q]
    float S32;            // (float)S
    float hazard_w2;      // a weight with w^2 >= this could change S in "S - w^2" (binary32)
    int flags;            // kFlag*
    unsigned int ticket;  // arrival counter of the finalisation kernel (returns to 0)
    unsigned long long search_counters[SP_NUM_COUNTERS];  // scratch of sp_search_la
    // state of sp_search_la's bisection when it runs on the device
    float search_la, search_lo, search_hi, search_best_la;
    double search_best_gap, search_best_frac;
};

// Powers of a = 1-alpha and b = 1-beta that the scan kernel needs (a lane owns P consecutive
// weights), computed on the host in fp64 and rounded once.
struct ScanConstants {
    float alpha, beta, la;
    float a, b;            // 1-alpha, 1-beta (rounded in fp32 like the definition)
    float a_lane[32];      // a^(P*lane)
    float b_lane[32];
    float a_step[5];       // a^(P*2^k)
    float b_step[5];
};

struct HostPipe;  // staging slots and streams of the host-buffer entry points (host_pipe.cu)

}  // namespace sp

struct sp_ctx {
    int device;
    int sm_count;
    int64_t d_in;
    int64_t n_pad;             // d_in rounded up to a multiple of kStripChannels
    int strips;                // n_pad / kStripChannels
    int64_t n_tokens;          // host-side count
    int slabs_valid;           // slab rows of `partial` that hold data
    bool dirty;                // batches arrived since the last finalisation
    int calib_blocks_per_sm;   // measured occupancy of the accumulation kernel
    double *partial;           // [kMaxSlabs][n_pad] fp64 partial column sums
    double *colsq;             // [n_pad]
    double *strip_sum;         // [strips]
    float *factor;             // [n_pad + 256] c_q, zero in the padding
    float *factor_pairs;       // the same values in the layout of the EWMA pair kernel (calib.cu)
    sp::DeviceScalars *scalars;
    sp::HostPipe *host_pipe;   // created by the first host-buffer call
};

namespace sp {

// Thread-local CUDA error text and the global launch counter (api.cu).
sp_status cuda_fail(cudaError_t e);
void count_launch(int n = 1);
inline sp_status check_launch() {
    cudaError_t e = cudaGetLastError();
    if (e != cudaSuccess) return cuda_fail(e);
    count_launch();
    return SP_OK;
}

// Readers of the bounded waits that ran out, one for each translation unit that has such waits
// (sp_tma.cuh); sp_wait_status collects them.
typedef cudaError_t (*WaitReader)(unsigned int *out, bool clear);
void register_wait_reader(WaitReader reader);  // api_serve.cu

// calib.cu
int calib_query_blocks_per_sm();
sp_status launch_calib_accumulate(sp_ctx *ctx, const void *X, sp_dtype dtype, int64_t n_tokens,
                                  int64_t ldx, cudaStream_t stream, bool x_complete = false);
sp_status launch_finalize(sp_ctx *ctx, cudaStream_t stream);
sp_status launch_finalize_pending(sp_ctx *const *ctxs, int count, cudaStream_t stream);
// One batch for each of several contexts (all different) in one launch; every item must satisfy
// calib_multi_applies (16-byte access).
struct CalibItem {
    const void *X;
    int64_t n_tokens, ldx;
};
bool calib_multi_applies(const sp_ctx *ctx, const void *X, int64_t ldx, int64_t n_tokens);
sp_status launch_calib_accumulate_multi(sp_ctx *const *ctxs, const CalibItem *items, int count,
                                        sp_dtype dtype, cudaStream_t stream, bool x_complete);
int64_t calib_static_max_d_in();
sp_status launch_calib_stats_static(int device, const void *X, sp_dtype dtype, int64_t n_tokens,
                                    int64_t d_in, int64_t ldx, double *colsq_out,
                                    float *factor_out, double *S_out, cudaStream_t stream);

// elementwise.cu
sp_status launch_score(const sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows,
                       int64_t ldw, float *scores, cudaStream_t stream);
sp_status launch_apply_mask(const void *W, sp_dtype dtype, int64_t n_rows, int64_t n_cols,
                            int64_t ldw, const uint32_t *mask, void *W_out, int64_t ldo,
                            cudaStream_t stream);

// select_nm_compressed.cu
sp_status launch_select_24_compressed(const sp_ctx *ctx, const void *W, sp_dtype dtype,
                                      int64_t n_rows, int64_t ldw, void *values, int64_t ldv,
                                      uint32_t *meta, cudaStream_t stream);

// One weight matrix of a selection launch that covers several.
struct EwmaLaunchJob {
    const void *W;
    void *W_out;     // nullable
    uint32_t *mask;  // nullable
    int64_t n_rows, ldw, ldo;
    const sp_ctx *ctx = nullptr;  // statistics to prune it with; null: those of the call's context
};

// select_nm.cu: N:M selection of up to kEwmaMaxJobs matrices (each with the statistics of its
// own context, or of `ctx`), in as few launches as their layouts and requested outputs allow
sp_status launch_select_nm(const sp_ctx *ctx, const EwmaLaunchJob *jobs, int n_jobs, sp_dtype dtype,
                           int N, int M, cudaStream_t stream);
inline sp_status launch_select_nm(const sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows,
                                  int64_t ldw, int N, int M, uint32_t *mask, void *W_out,
                                  int64_t ldo, cudaStream_t stream) {
    const EwmaLaunchJob job{W, W_out, mask, n_rows, ldw, ldo};
    return launch_select_nm(ctx, &job, 1, dtype, N, M, stream);
}

// select_ewma.cu
// Algorithm 1 on several matrices of one dtype (each with the statistics of its own context, or
// of `ctx`), in as few launches as their layouts allow.
sp_status launch_select_ewma(const sp_ctx *ctx, const EwmaLaunchJob *jobs, int n_jobs,
                             sp_dtype dtype, const sp_ewma_params &p, unsigned long long *counters,
                             cudaStream_t stream, bool la_from_device = false);
inline sp_status launch_select_ewma(const sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows,
                                    int64_t ldw, const sp_ewma_params &p, uint32_t *mask,
                                    void *W_out, int64_t ldo, unsigned long long *counters,
                                    cudaStream_t stream, bool la_from_device = false) {
    const EwmaLaunchJob job{W, W_out, mask, n_rows, ldw, ldo};
    return launch_select_ewma(ctx, &job, 1, dtype, p, counters, stream, la_from_device);
}
// True when launch_select_ewma would take the kernel that can read la from DeviceScalars.
bool ewma_pair_path_applies(const void *W, int64_t ldw, int64_t n);
sp_status launch_search_la_device(sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows,
                                  int64_t ldw, float target, float alpha, float beta,
                                  int iterations, float *la_out, double *achieved_out,
                                  cudaStream_t stream);

// select_ewma_sweep.cu
sp_status launch_ewma_sweep(const sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows,
                            int64_t ldw, const sp_ewma_params &p, uint32_t *mask, void *W_out,
                            int64_t ldo, unsigned long long *counters, cudaStream_t stream);

// select_ewma_tiled.cu
sp_status launch_ewma_literal_tiled(const sp_ctx *ctx, const void *W, sp_dtype dtype,
                                    int64_t n_rows, int64_t ldw, const sp_ewma_params &p,
                                    uint32_t *mask, void *W_out, int64_t ldo,
                                    unsigned long long *counters, cudaStream_t stream);

// host_pipe.cu
void host_pipe_destroy(HostPipe *hp);
sp_status host_calib_accumulate(sp_ctx *ctx, const void *X_host, sp_dtype dtype, int64_t n_tokens,
                                int64_t ldx, cudaStream_t stream);
sp_status host_select(sp_ctx *ctx, int kind, const void *W_host, sp_dtype dtype, int64_t n_rows,
                      int64_t ldw, int N, int M, const sp_ewma_params *params,
                      uint32_t *mask_host, void *W_out_host, int64_t ldo, cudaStream_t stream);

// Launch configuration with programmatic dependent launch allowed: the kernel may be scheduled
// while the previous kernel of the stream drains; every kernel launched this way executes
// griddepcontrol.wait before it touches memory an earlier kernel may still be writing.
struct PdlConfig {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[1];
    PdlConfig(dim3 grid, dim3 block, cudaStream_t stream) : cfg{}, attr{} {
        cfg.gridDim = grid;
        cfg.blockDim = block;
        cfg.dynamicSmemBytes = 0;
        cfg.stream = stream;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
};

// The same for clusters of `blocks` neighbours along x.
struct ClusterPdlConfig {
    cudaLaunchConfig_t cfg;
    cudaLaunchAttribute attr[2];
    ClusterPdlConfig(int blocks, dim3 grid, dim3 block, cudaStream_t stream) : cfg{}, attr{} {
        cfg.gridDim = grid;
        cfg.blockDim = block;
        cfg.stream = stream;
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        attr[1].id = cudaLaunchAttributeClusterDimension;
        attr[1].val.clusterDim.x = static_cast<unsigned>(blocks);
        attr[1].val.clusterDim.y = 1;
        attr[1].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = blocks > 1 ? 2 : 1;
    }
};

// Allows a kernel all the dynamic shared memory of an SM, once for each device.
class DynamicSmem {
   public:
    cudaError_t allow(const void *kernel) {
        int device = 0;
        cudaError_t e = cudaGetDevice(&device);
        if (e != cudaSuccess) return e;
        const uint64_t bit = uint64_t(1) << (device & 63);
        if (done_.load(std::memory_order_acquire) & bit) return cudaSuccess;
        cudaFuncAttributes attr;
        e = cudaFuncGetAttributes(&attr, kernel);
        if (e != cudaSuccess) return e;
        e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 kMaxBlockSmem - static_cast<int>(attr.sharedSizeBytes));
        if (e == cudaSuccess) done_.fetch_or(bit, std::memory_order_release);
        return e;
    }
    static constexpr int kMaxBlockSmem = 227 * 1024;

   private:
    std::atomic<uint64_t> done_{0};
};

sp_status launch_ewma_trace(const sp_ctx *ctx, const void *W, sp_dtype dtype, int64_t n_rows,
                            int64_t ldw, const sp_ewma_params &p, float *est_out, float *dev_out,
                            float *score_out, cudaStream_t stream);

// mx4_quantize.cu
sp_status launch_mx4_quantize(const void *W, sp_dtype dtype, int64_t n_rows, int64_t n_cols,
                              int64_t ldw, const uint32_t *mask, uint8_t *codes, int64_t ldc,
                              uint8_t *scales, cudaStream_t stream);
sp_status launch_mx4_dequantize(const uint8_t *codes, int64_t ldc, const uint8_t *scales,
                                int64_t n_rows, int64_t n_cols, sp_dtype dtype, void *W,
                                int64_t ldw, cudaStream_t stream);

// A product with a microscaled 4-bit matrix: Y [n_tokens, n_rows] = X [n_tokens, n_cols] W^T.
struct Mx4Product {
    const void *X;
    int64_t n_tokens, ldx;
    const uint8_t *codes;
    int64_t ldc;
    const uint8_t *scales;
    int64_t n_rows, n_cols;
    void *Y;
    int64_t ldy;
    sp_dtype dtype;
    bool quantize_x;  // SP_MX4_A4
};
// mx4_stream.cu: up to 8 tokens, the weights stream by once
constexpr int kMx4StreamTokens = 8;
sp_status launch_mx4_stream(const Mx4Product &p, cudaStream_t stream);
// mx4_gemm.cu: both operands in 4 bits (quantises X into the workspace first)
int64_t mx4_gemm_workspace(int64_t n_tokens, int64_t n_cols);
sp_status launch_mx4_gemm(const Mx4Product &p, void *workspace, cudaStream_t stream);
// mx4_gemm16.cu: 16-bit activations (the workspace takes rows that TMA cannot read)
int64_t mx4_gemm16_workspace(int64_t n_tokens, int64_t n_cols);
bool mx4_gemm16_reads(const void *X, int64_t ldx);  // whether TMA reads the rows as they are
sp_status launch_mx4_gemm16(const Mx4Product &p, void *workspace, cudaStream_t stream);

// cache_append.cu, cache_attention.cu, cache_evict.cu: the 8-bit key/value cache
sp_status launch_cache_append(const sp_cache &cache, const void *K, const sp_strides &ks, const void *V,
                              const sp_strides &vs, sp_dtype dtype, int64_t n_new, const int32_t *start,
                              const int32_t *count, cudaStream_t stream);
int64_t cache_attention_workspace(const sp_cache &c, int64_t n_q, int n_heads, int64_t max_len, bool want_acc);
sp_status launch_cache_attention(const sp_cache &c, const void *Q, const sp_strides &q, sp_dtype dtype, int64_t n_q,
                                 int n_heads, const int32_t *lens, int64_t max_len, float scale, void *O,
                                 const sp_strides &o, float *lse, const float *acc_in, float *acc_out, int64_t ld_acc,
                                 void *workspace, cudaStream_t stream);
sp_status launch_cache_evict(const sp_cache &src, const int32_t *lens, int64_t max_len, const float *acc, int64_t ld_acc,
                             int64_t budget, int64_t recent, const sp_cache &dst, int32_t *kept, float *acc_out,
                             int64_t ld_acc_out, int32_t *lens_out, cudaStream_t stream);

// qk_rotary.cu: norms of queries and keys and the rotation by position
struct QkRotary {
    const void *Q, *K, *q_weight, *k_weight;
    void *Q_out, *K_out;
    sp_strides q, k, q_out, k_out;
    sp_dtype dtype;
    int64_t n_seqs, n_tokens;
    int n_heads, n_kv_heads, head_dim, rotary;
    const int32_t *start;
    const float *freq;
    float eps;
    bool pairs;
};
sp_status launch_qk_rotary(const QkRotary &r, cudaStream_t stream);

// cache_pages.cu: shared blocks of the 8-bit cache
int64_t cache_fork_workspace(const sp_cache &c, int64_t n);
sp_status launch_cache_fork(const sp_cache &c, int32_t *refs, const int32_t *dst, const int32_t *src,
                            int64_t n, void *workspace, cudaStream_t stream);
int64_t cache_reserve_workspace(const sp_cache &c, int64_t n_new);
sp_status launch_cache_reserve(const sp_cache &c, int32_t *refs, const int32_t *start,
                               const int32_t *count, int64_t n_new, int32_t *status, void *workspace, cudaStream_t stream);
int64_t cache_compact_workspace(const sp_cache &c);
sp_status launch_cache_compact(const sp_cache &c, const int32_t *refs, int32_t *table_out, int64_t ld_table_out,
                               int32_t *refs_out, int32_t *live, void *workspace, cudaStream_t stream);

// cache_shared.cu: attention over a prefix that a group of sequences shares
struct SharedAttention {
    const void *Q;
    sp_strides q, o;
    sp_dtype dtype;
    int64_t n_q, max_len, n_groups, max_prefix, max_group;
    int n_heads;
    const int32_t *lens, *group_start, *prefix;
    float scale;
    void *O;
    float *lse;
};
bool cache_shared_fits(const sp_cache &c, const SharedAttention &s);  // whether the queries' rows fit in a launch
int64_t cache_shared_workspace(const sp_cache &c, const SharedAttention &s);
sp_status launch_cache_shared(const sp_cache &c, const SharedAttention &s, void *workspace, cudaStream_t stream);

inline bool aligned16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace sp
