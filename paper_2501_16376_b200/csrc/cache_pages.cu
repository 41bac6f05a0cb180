// Blocks of the 8-bit cache that several sequences share: rows of the table become copies of other
// rows (fork, free), the places of new tokens become writable (reserve), live blocks move to the
// front of the pool (compact).  refs[x] counts the table entries that name block x.
//
// Everything is whole numbers and copies, and comes out the same whatever the order of the atomics:
// counts are sums, and where requests compete the lowest one is taken.  The bookkeeping is a few
// thousand words: bound by the latency of its steps, so fork is one kernel and reserve and compact
// are one block for the bookkeeping (a scan needs no other launch then) and one kernel over the
// device for the copies, which are bound by memory (block bytes read once and written once).
// Measured (replayed from a graph): fork and reserve of 64 answers of 4 prompts 12 us, of 128 with 120
// copied blocks of 0.5 MB 21.7 us (5.8 TB/s of copies); compact of 300 blocks 5.6 us, of 8192 with 1900
// moved blocks of 64 KB 46 us, of which the copies are 37 (6.6 TB/s, the copy rate).
#include <algorithm>

#include "cache_common.cuh"
#include "sp_internal.h"

namespace sp {

namespace {

constexpr int kForkThreads = 1024, kForkWarps = kForkThreads / 32;
constexpr int kBookThreads = 1024, kBookWarps = kBookThreads / 32;
constexpr int kCopyThreads = 256, kCopyEach = 4;  // 16-byte pieces a thread has in flight

struct ForkArgs {
    int32_t *table, *refs;
    const int32_t *dst, *src;
    int32_t *staged;  // [blocks of the grid][n][32] where they do not fit in shared memory
    int64_t ld_table;
    int n, n_seqs, cols, n_blocks;
};

__device__ __forceinline__ bool names(int id, int n_blocks) { return static_cast<uint32_t>(id) < static_cast<uint32_t>(n_blocks); }

}  // namespace

// A block has 32 columns of the table, which no other block touches: it reads the source rows, waits
// for itself, and writes.  Of several entries for one row the last counts.
__global__ void __launch_bounds__(kForkThreads)
cache_fork_kernel(const ForkArgs a) {
    extern __shared__ int32_t fork_smem[];
    int32_t *winner = fork_smem;  // of a row: the last entry that names it
    int32_t *staged = a.staged != nullptr ? a.staged + int64_t(blockIdx.x) * a.n * 32 : fork_smem + a.n_seqs;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, col = blockIdx.x * 32 + lane;
    const bool here = col < a.cols;
    pdl_launch_dependents();
    pdl_wait();
    for (int i = threadIdx.x; i < a.n; i += kForkThreads)
        if (names(a.dst[i], a.n_seqs)) winner[a.dst[i]] = -1;
    __syncthreads();
    for (int i = threadIdx.x; i < a.n; i += kForkThreads)
        if (names(a.dst[i], a.n_seqs)) atomicMax(&winner[a.dst[i]], i);
    __syncthreads();
#pragma unroll 4
    for (int i = warp; i < a.n; i += kForkWarps) {
        const int d = a.dst[i], s = a.src != nullptr ? a.src[i] : -1;
        if (!here || !names(d, a.n_seqs) || winner[d] != i) continue;
        const int now = names(s, a.n_seqs) ? a.table[s * a.ld_table + col] : -1, was = a.table[d * a.ld_table + col];
        staged[int64_t(i) * 32 + lane] = now;
        if (was == now) continue;
        if (names(was, a.n_blocks)) atomicSub(&a.refs[was], 1);
        if (names(now, a.n_blocks)) atomicAdd(&a.refs[now], 1);
    }
    __syncthreads();
#pragma unroll 4
    for (int i = warp; i < a.n; i += kForkWarps) {
        const int d = a.dst[i];
        if (here && names(d, a.n_seqs) && winner[d] == i) a.table[d * a.ld_table + col] = staged[int64_t(i) * 32 + lane];
    }
}

// ------------------------------------------------------------------ scans of one block

// Exclusive sum over the block's threads, in their order, and the total.
__device__ __forceinline__ int block_scan(int v, int *warp_sums, int &total) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int sum = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(kFullWarp, sum, o);
        if (lane >= o) sum += up;
    }
    __syncthreads();  // the sums of the scan before have been read
    if (lane == 31) warp_sums[warp] = sum;
    __syncthreads();
    const int w = warp_sums[lane];
    int all = w;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const int up = __shfl_up_sync(kFullWarp, all, o);
        if (lane >= o) all += up;
    }
    total = __shfl_sync(kFullWarp, all, 31);
    return sum - v + __shfl_sync(kFullWarp, all - w, warp);
}

// Live blocks among those of a warp's stretch: the pool is cut into one stretch of whole 32 for every warp.
struct Stretch {
    int begin, end;
    __device__ __forceinline__ Stretch(int n_blocks) {
        const int each = (n_blocks + kBookWarps * 32 - 1) / (kBookWarps * 32) * 32;
        begin = min(n_blocks, static_cast<int>(threadIdx.x >> 5) * each);
        end = min(n_blocks, begin + each);
    }
};
// `flags` keeps what a lane saw in its first 32 looks (pools up to 32768 blocks), for is_live.
__device__ __forceinline__ int count_live(const int32_t *refs, const Stretch &s, uint32_t &flags) {
    const int lane = threadIdx.x & 31;
    int live = 0;
    flags = 0u;
#pragma unroll 8
    for (int i = s.begin, look = 0; i < s.end; i += 32, ++look) {
        const uint32_t one = i + lane < s.end && refs[i + lane] > 0;
        live += one;
        if (look < 32) flags |= one << look;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) live += __shfl_xor_sync(kFullWarp, live, o);
    return live;
}
__device__ __forceinline__ bool is_live(const int32_t *refs, const Stretch &s, uint32_t flags, int i) {
    const int look = (i - s.begin) >> 5, at = i + (threadIdx.x & 31);
    return look < 32 ? (flags >> look) & 1u : at < s.end && refs[at] > 0;
}

// ------------------------------------------------------------------ reserve

namespace {
struct ReserveArgs {
    sp_cache cache;
    int32_t *table, *refs;
    const int32_t *start, *count;
    int32_t *status;
    int32_t *asked, *first;  // [n_blocks]: requests for a shared block, and the lowest of them
    int32_t *rank, *free;    // [requests]: place of a request among those that need a block; free blocks
    int2 *copies;            // [n_seqs]: (from, to), from < 0 where nothing is copied
    int64_t n_new;
    int per;                 // requests of a sequence
    int requests, block_shift;
};

struct Request {
    int row;
    int64_t entry;        // of the table
    int id;               // the block named there, or < 0
    bool asked, partial;  // whether it is asked for; whether tokens before the new ones lie in it
};
__device__ __forceinline__ Request request(const ReserveArgs &a, int r) {
    const sp_cache &c = a.cache;
    Request q = {};
    q.id = -1;
    if (r >= a.requests) return q;
    q.row = r / a.per;
    const int start = a.start[q.row];
    const int64_t n = a.count != nullptr ? min(int64_t(a.count[q.row]), a.n_new) : a.n_new;
    const int64_t place = (start >> a.block_shift) + (r - q.row * a.per), first = place << a.block_shift;
    if (start < 0 || n <= 0 || first >= start + n || place >= c.table_cols) return q;
    q.asked = true;
    q.partial = first < start;
    q.entry = q.row * c.ld_table + place;
    const int id = a.table[q.entry];
    q.id = names(id, static_cast<int>(c.n_blocks)) ? id : -1;
    return q;
}
}  // namespace

// Requests in the order of sequences and places; free blocks in ascending order.  A shared block that
// all who share it ask for stays with the first of them.
__global__ void __launch_bounds__(kBookThreads)
cache_reserve_kernel(const __grid_constant__ ReserveArgs a) {
    __shared__ int warp_sums[kBookWarps], live_before[kBookWarps + 1];
    const sp_cache &c = a.cache;
    const int n_blocks = static_cast<int>(c.n_blocks), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_launch_dependents();
    pdl_wait();
    for (int r = threadIdx.x; r < a.requests; r += kBookThreads) {
        const Request q = request(a, r);
        if (q.id >= 0) {
            a.asked[q.id] = 0;
            a.first[q.id] = 0x7fffffff;
        }
        if (r % a.per == 0) a.copies[r / a.per] = make_int2(-1, -1);
    }
    const Stretch mine(n_blocks);
    uint32_t flags;
    const int live = count_live(a.refs, mine, flags);
    if (lane == 0) live_before[warp] = live;
    __syncthreads();
    for (int r = threadIdx.x; r < a.requests; r += kBookThreads) {
        const Request q = request(a, r);
        if (q.id >= 0) {
            atomicAdd(&a.asked[q.id], 1);
            atomicMin(&a.first[q.id], r);
        }
    }
    if (warp == 0) {  // live blocks before each warp's stretch
        const int v = live_before[lane];
        int sum = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(kFullWarp, sum, o);
            if (lane >= o) sum += up;
        }
        live_before[lane] = sum - v;
        if (lane == 31) live_before[32] = sum;
    }
    __syncthreads();
    const int n_free = n_blocks - live_before[kBookWarps];
    int need = 0;
    for (int r0 = 0; r0 < a.requests; r0 += kBookThreads) {
        const int r = r0 + static_cast<int>(threadIdx.x);
        const Request q = request(a, r);
        bool wants = q.asked;
        if (q.id >= 0) {
            const int refs = a.refs[q.id];
            if (refs <= 1 || (a.asked[q.id] >= refs && a.first[q.id] == r)) wants = false;
        }
        int total;
        const int at = block_scan(wants, warp_sums, total);
        if (r < a.requests) a.rank[r] = wants ? need + at : -1;
        need += total;
    }
    const bool served = need <= n_free;
    if (threadIdx.x == 0) {
        a.status[0] = served ? 0 : need - n_free;
        a.status[1] = served ? n_free - need : n_free;
    }
    if (!served || need == 0) return;
    // the free blocks that are handed out
    int before = mine.begin - live_before[warp];
    for (int i = mine.begin; i < mine.end && before < need; i += 32) {
        const bool is_free = i + lane < mine.end && !is_live(a.refs, mine, flags, i);
        const unsigned vote = __ballot_sync(kFullWarp, is_free);
        const int at = before + __popc(vote & ((1u << lane) - 1u));
        if (is_free && at < need) a.free[at] = i + lane;
        before += __popc(vote);
    }
    __syncthreads();
    for (int r = threadIdx.x; r < a.requests; r += kBookThreads) {
        const int at = a.rank[r];
        if (at < 0) continue;
        const Request q = request(a, r);
        const int id = a.free[at];
        a.table[q.entry] = id;
        a.refs[id] = 1;
        if (q.id >= 0) {
            atomicSub(&a.refs[q.id], 1);
            if (q.partial) a.copies[q.row] = make_int2(q.id, id);
        }
    }
}

// ------------------------------------------------------------------ copies

// One block of the cache, K and V, all heads, and their scales; piece `part` of `parts`.
__device__ __forceinline__ void copy_block(const sp_cache &c, int64_t from, int64_t to, int64_t part) {
    const int64_t each = int64_t(c.n_kv_heads) * c.block_tokens * c.head_dim / 16;  // pieces of K, and of V
    const uint4 *k_from = static_cast<const uint4 *>(c.k) + from * each, *v_from = static_cast<const uint4 *>(c.v) + from * each;
    uint4 *k_to = static_cast<uint4 *>(c.k) + to * each, *v_to = static_cast<uint4 *>(c.v) + to * each;
    const int64_t at = part * (kCopyThreads * kCopyEach) + threadIdx.x;
    uint4 k[kCopyEach], v[kCopyEach];
#pragma unroll
    for (int i = 0; i < kCopyEach; ++i)
        if (at + i * kCopyThreads < each) {
            k[i] = __ldcs(k_from + at + i * kCopyThreads);
            v[i] = __ldcs(v_from + at + i * kCopyThreads);
        }
#pragma unroll
    for (int i = 0; i < kCopyEach; ++i)
        if (at + i * kCopyThreads < each) {
            __stcs(k_to + at + i * kCopyThreads, k[i]);
            __stcs(v_to + at + i * kCopyThreads, v[i]);
        }
    if (part == 0)
        for (int h = threadIdx.x; h < c.n_kv_heads; h += kCopyThreads) {
            c.k_scale[to * c.n_kv_heads + h] = c.k_scale[from * c.n_kv_heads + h];
            c.v_scale[to * c.n_kv_heads + h] = c.v_scale[from * c.n_kv_heads + h];
        }
}
static int64_t copy_parts(const sp_cache &c) {
    const int64_t each = int64_t(c.n_kv_heads) * c.block_tokens * c.head_dim / 16;
    return (each + kCopyThreads * kCopyEach - 1) / (kCopyThreads * kCopyEach);
}

// Block x: a piece of the copy of sequence x / parts.
__global__ void __launch_bounds__(kCopyThreads)
cache_reserve_copy_kernel(const __grid_constant__ sp_cache c, const int2 *copies, int parts) {
    pdl_launch_dependents();
    pdl_wait();
    for (int64_t x = blockIdx.x; x < c.n_seqs * parts; x += gridDim.x) {
        const int2 copy = copies[x / parts];
        if (copy.x >= 0) copy_block(c, copy.x, copy.y, x % parts);
    }
}

// ------------------------------------------------------------------ compact

namespace {
struct CompactArgs {
    sp_cache cache;
    const int32_t *refs;
    int32_t *table_out, *refs_out, *live;
    int64_t ld_table_out;
    int32_t *moves;   // how many
    int32_t *remap;   // [n_blocks]: a block's new number, -1 for free ones
    int32_t *holes, *movers;  // [n_blocks / 2 + 1]
};
}  // namespace

// The k-th live block past the first n_live numbers moves to the k-th free number among them.
__global__ void __launch_bounds__(kBookThreads)
cache_compact_kernel(const __grid_constant__ CompactArgs a) {
    __shared__ int live_before[kBookWarps + 1], low_live;
    const int n_blocks = static_cast<int>(a.cache.n_blocks), lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_launch_dependents();
    pdl_wait();
    const Stretch mine(n_blocks);
    uint32_t flags;
    const int live = count_live(a.refs, mine, flags);
    if (lane == 0) live_before[warp] = live;
    if (threadIdx.x == 0) low_live = 0;
    __syncthreads();
    if (warp == 0) {
        const int v = live_before[lane];
        int sum = v;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const int up = __shfl_up_sync(kFullWarp, sum, o);
            if (lane >= o) sum += up;
        }
        live_before[lane] = sum - v;
        if (lane == 31) live_before[32] = sum;
    }
    __syncthreads();
    const int n_live = live_before[kBookWarps];
    // live blocks among the first n_live numbers: each warp's share of them
    {
        int low = 0;
        for (int i = mine.begin; i < min(mine.end, n_live); i += 32) low += i + lane < n_live && is_live(a.refs, mine, flags, i);
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) low += __shfl_xor_sync(kFullWarp, low, o);
        if (lane == 0 && low != 0) atomicAdd(&low_live, low);
    }
    __syncthreads();
    const int stay = low_live, moves = n_live - stay;
    if (threadIdx.x == 0) {
        *a.live = n_live;
        *a.moves = moves;
    }
    int before = live_before[warp];
    for (int i = mine.begin; i < mine.end; i += 32) {
        const int id = i + lane;
        const bool in = id < mine.end, alive = is_live(a.refs, mine, flags, i);
        const unsigned vote = __ballot_sync(kFullWarp, alive);
        const int at = before + __popc(vote & ((1u << lane) - 1u));  // live blocks before this one
        if (in) {
            if (alive && id >= n_live) a.movers[at - stay] = id;
            else a.remap[id] = alive ? id : -1;
            if (!alive && id < n_live) a.holes[id - at] = id;
        }
        before += __popc(vote);
    }
    __syncthreads();
    if (a.refs_out != a.refs)
        for (int i = threadIdx.x; i < n_blocks; i += kBookThreads) {
            const int n = a.refs[i];
            a.refs_out[i] = i < n_live && n > 0 ? n : 0;
        }
    else  // what is no live block's count becomes 0
        for (int i = threadIdx.x; i < n_live; i += kBookThreads)
            if (a.refs[i] < 0) a.refs_out[i] = 0;
    __syncthreads();
    for (int k = threadIdx.x; k < moves; k += kBookThreads) {
        const int from = a.movers[k], to = a.holes[k];
        a.remap[from] = to;
        a.refs_out[to] = a.refs[from];
    }
    if (a.refs_out == a.refs) {
        __syncthreads();
        for (int i = n_live + threadIdx.x; i < n_blocks; i += kBookThreads) a.refs_out[i] = 0;
    }
}

__global__ void __launch_bounds__(kCopyThreads)
cache_compact_copy_kernel(const __grid_constant__ CompactArgs a, int parts) {
    const sp_cache &c = a.cache;
    pdl_launch_dependents();
    pdl_wait();
    const int64_t entries = c.n_seqs * c.table_cols;
    for (int64_t i = int64_t(blockIdx.x) * kCopyThreads + threadIdx.x; i < entries; i += int64_t(gridDim.x) * kCopyThreads) {
        const int64_t row = i / c.table_cols, col = i % c.table_cols;
        const int id = c.table[row * c.ld_table + col];
        a.table_out[row * a.ld_table_out + col] = names(id, static_cast<int>(c.n_blocks)) ? a.remap[id] : id;
    }
    const int64_t pieces = int64_t(*a.moves) * parts;
    for (int64_t x = blockIdx.x; x < pieces; x += gridDim.x) copy_block(c, a.movers[x / parts], a.holes[x / parts], x % parts);
}

// ------------------------------------------------------------------ launches

constexpr int kMostForkSmem = 200 * 1024;
static bool fork_fits(const sp_cache &c, int64_t n) { return (c.n_seqs + n * 32) * 4 <= kMostForkSmem; }

int64_t cache_fork_workspace(const sp_cache &c, int64_t n) {
    return fork_fits(c, n) ? 0 : (c.table_cols + 31) / 32 * n * 128;
}

sp_status launch_cache_fork(const sp_cache &c, int32_t *refs, const int32_t *dst, const int32_t *src,
                            int64_t n, void *workspace, cudaStream_t stream) {
    ForkArgs a = {};
    a.table = const_cast<int32_t *>(c.table);
    a.refs = refs;
    a.dst = dst;
    a.src = src;
    a.ld_table = c.ld_table;
    a.n = static_cast<int>(n);
    a.n_seqs = static_cast<int>(c.n_seqs);
    a.cols = static_cast<int>(c.table_cols);
    a.n_blocks = static_cast<int>(c.n_blocks);
    a.staged = fork_fits(c, n) ? nullptr : static_cast<int32_t *>(workspace);
    PdlConfig pdl(dim3(static_cast<unsigned>((c.table_cols + 31) / 32)), dim3(kForkThreads), stream);
    pdl.cfg.dynamicSmemBytes = (c.n_seqs + (a.staged == nullptr ? n * 32 : 0)) * 4;
    static DynamicSmem limit;
    cudaError_t e = pdl.cfg.dynamicSmemBytes > 48 * 1024 ? limit.allow(reinterpret_cast<const void *>(cache_fork_kernel)) : cudaSuccess;
    if (e == cudaSuccess) e = cudaLaunchKernelEx(&pdl.cfg, cache_fork_kernel, a);
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

static int64_t requests_of_a_sequence(const sp_cache &c, int64_t n_new) {
    return std::min(c.table_cols, (n_new + c.block_tokens - 2) / c.block_tokens + 1);
}

int64_t cache_reserve_workspace(const sp_cache &c, int64_t n_new) {
    return 8 * c.n_seqs + 8 * c.n_blocks + 8 * c.n_seqs * requests_of_a_sequence(c, n_new);
}

sp_status launch_cache_reserve(const sp_cache &c, int32_t *refs, const int32_t *start,
                               const int32_t *count, int64_t n_new, int32_t *status, void *workspace, cudaStream_t stream) {
    ReserveArgs a = {};
    a.cache = c;
    a.table = const_cast<int32_t *>(c.table);
    a.refs = refs;
    a.start = start;
    a.count = count;
    a.status = status;
    a.n_new = n_new;
    a.per = static_cast<int>(requests_of_a_sequence(c, n_new));
    a.requests = static_cast<int>(c.n_seqs * a.per);
    a.block_shift = c.block_tokens == 16 ? 4 : c.block_tokens == 32 ? 5 : 6;
    a.copies = static_cast<int2 *>(workspace);
    a.asked = reinterpret_cast<int32_t *>(a.copies + c.n_seqs);
    a.first = a.asked + c.n_blocks;
    a.rank = a.first + c.n_blocks;
    a.free = a.rank + a.requests;
    PdlConfig pdl(dim3(1), dim3(kBookThreads), stream);
    cudaError_t e = cudaLaunchKernelEx(&pdl.cfg, cache_reserve_kernel, a);
    if (e != cudaSuccess) return cuda_fail(e);
    sp_status st = check_launch();
    if (st != SP_OK || a.requests == 0 || c.n_blocks == 0) return st;
    const int64_t parts = copy_parts(c);
    PdlConfig second(dim3(static_cast<unsigned>(std::min(c.n_seqs * parts, int64_t(148 * 8)))), dim3(kCopyThreads), stream);
    e = cudaLaunchKernelEx(&second.cfg, cache_reserve_copy_kernel, c, static_cast<const int2 *>(a.copies), static_cast<int>(parts));
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

int64_t cache_compact_workspace(const sp_cache &c) { return 4 * (2 * c.n_blocks + 4); }

sp_status launch_cache_compact(const sp_cache &c, const int32_t *refs, int32_t *table_out, int64_t ld_table_out,
                               int32_t *refs_out, int32_t *live, void *workspace, cudaStream_t stream) {
    CompactArgs a = {};
    a.cache = c;
    a.refs = refs;
    a.table_out = table_out;
    a.ld_table_out = ld_table_out;
    a.refs_out = refs_out;
    a.live = live;
    a.moves = static_cast<int32_t *>(workspace);
    a.remap = a.moves + 1;
    a.holes = a.remap + c.n_blocks;
    a.movers = a.holes + c.n_blocks / 2 + 1;
    PdlConfig pdl(dim3(1), dim3(kBookThreads), stream);
    cudaError_t e = cudaLaunchKernelEx(&pdl.cfg, cache_compact_kernel, a);
    if (e != cudaSuccess) return cuda_fail(e);
    sp_status st = check_launch();
    if (st != SP_OK) return st;
    const int64_t parts = copy_parts(c), most = std::max(c.n_blocks / 2 * parts, (c.n_seqs * c.table_cols + kCopyThreads - 1) / kCopyThreads);
    PdlConfig second(dim3(static_cast<unsigned>(std::max(int64_t(1), std::min(most, int64_t(148 * 8))))), dim3(kCopyThreads), stream);
    e = cudaLaunchKernelEx(&second.cfg, cache_compact_copy_kernel, a, static_cast<int>(parts));
    if (e != cudaSuccess) return cuda_fail(e);
    return check_launch();
}

}  // namespace sp
