// Block tables and slot maps of a paged cache, from request lengths alone.
//
// Request r holds old[r] tokens and gets new[r] more. With B tokens to a block it needs the
// blocks ceil(old / B) .. ceil((old + new) / B) - 1 on top of those it has; they are taken from
// the free list in request order, so request r's begin at the exclusive prefix sum of the
// counts before it. New row i (the rows of all requests in order) is token
// old[r] + i - start[r] of its request, in slot block * B + token % B.
//
// Every thread block computes both prefix sums itself, into shared memory, and then fills its
// share of the table and of the slot map: a row's block is either one that the table held
// before (which no thread writes) or comes straight from the free list, so no thread block
// waits for another and one launch is enough. Bound by latency: the lengths' load, the scan,
// one binary search and one dependent load, for some four rows a thread at most of the sizes below. Measured: 16
// requests of one new token 2.2 us, 509 requests with 24 prompt chunks among them 3.8 us, 64 prompts of 325,598 rows
// 5.3 us. (A thread's four rows side by side: no faster.)
#include "cm_qcache_kernels.h"

namespace cm {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / 32;

__device__ __forceinline__ int64_t clamp_len(int32_t x) { return x > 0 ? x : 0; }

struct Request {
    int64_t old_len, new_len;   // as far as the table reaches
    int64_t first, need;        // first fresh block and their number
    int64_t kv;
};

__device__ __forceinline__ Request request(const QcacheTablesParams &p, int r) {
    Request q;
    const int64_t cap = p.table_width << p.log2_block;
    q.old_len = clamp_len(p.old_lens[r]);
    q.new_len = clamp_len(p.new_lens[r]);
    q.kv = min(q.old_len + q.new_len, cap);
    const int64_t mask = ((int64_t)1 << p.log2_block) - 1;
    q.first = min((q.old_len + mask) >> p.log2_block, p.table_width);
    q.need = max(((q.kv + mask) >> p.log2_block) - q.first, (int64_t)0);
    return q;
}

// Index of the last entry of starts[0 .. n) that is <= x (starts ascends, starts[0] = 0).
__device__ __forceinline__ int owner(const int32_t *starts, int n, int32_t x) {
    int lo = 0, hi = n;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (starts[mid] <= x) lo = mid; else hi = mid;
    }
    return lo;
}

__global__ void __launch_bounds__(kThreads) tables_kernel(const QcacheTablesParams p) {
    after_kernels_before();
    extern __shared__ int32_t prefix[];   // row starts, then block starts, of the requests
    int32_t *row_start = prefix, *block_start = prefix + p.requests;
    __shared__ int64_t warp_rows[kWarps], warp_blocks[kWarps];
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    int64_t rows = 0, blocks = 0;         // before the requests of this step
    for (int r0 = 0; r0 < p.requests; r0 += kThreads) {
        const int r = r0 + tid;
        Request q{0, 0, 0, 0, 0};
        if (r < p.requests) q = request(p, r);
        int64_t a = q.new_len, b = q.need;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int64_t x = __shfl_up_sync(~0u, a, d), y = __shfl_up_sync(~0u, b, d);
            if (lane >= d) { a += x; b += y; }
        }
        if (lane == 31) { warp_rows[warp] = a; warp_blocks[warp] = b; }
        __syncthreads();
        int64_t before_a = rows, before_b = blocks;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) { before_a += warp_rows[w]; before_b += warp_blocks[w]; }
            rows += warp_rows[w];
            blocks += warp_blocks[w];
        }
        if (r < p.requests) {
            // rows and blocks past the last that are written need no exact place
            row_start[r] = (int32_t)min(before_a + a - q.new_len, (int64_t)INT32_MAX);
            block_start[r] = (int32_t)min(before_b + b - q.need, (int64_t)INT32_MAX);
            if (blockIdx.x == 0) {
                const int64_t start = min(before_a + a - q.new_len, p.max_rows), end = min(before_a + a, p.max_rows);
                p.row_starts[r] = (int32_t)start;
                p.kv_lens[r] = (int32_t)q.kv;
                // the lengths of a request that was cut short do not say which tokens its rows are
                if (p.context_out) {
                    const bool cut = end - start < q.new_len || q.kv < q.old_len + q.new_len;
                    p.context_out[r] = cut ? (int32_t)q.old_len : -1;
                }
            }
        }
        __syncthreads();
    }
    if (blockIdx.x == 0 && tid == 0) {
        p.row_starts[p.requests] = (int32_t)min(rows, p.max_rows);
        p.counts[0] = blocks;
        p.counts[1] = rows;
    }
    const int64_t step = (int64_t)gridDim.x * kThreads, at = (int64_t)blockIdx.x * kThreads + tid;
    const int64_t fresh = min(blocks, (int64_t)INT32_MAX);
    for (int64_t e = at; e < fresh; e += step) {
        const int r = owner(block_start, p.requests, (int32_t)e);
        const Request q = request(p, r);
        const int64_t j = e - block_start[r];
        if (j < q.need)
            p.block_table[r * p.table_width + q.first + j] = e < p.num_free ? p.free_blocks[e] : -1;
    }
    for (int64_t i = at; i < p.max_rows; i += step) {
        int64_t slot = -1;
        if (i < rows) {
            const int r = owner(row_start, p.requests, (int32_t)i);
            const Request q = request(p, r);
            const int64_t pos = q.old_len + i - row_start[r], j = pos >> p.log2_block;
            if (j < p.table_width) {
                const int64_t e = block_start[r] + j - q.first;
                int32_t block = -1;
                if (j < q.first) block = p.block_table[r * p.table_width + j];
                else if (e < p.num_free) block = p.free_blocks[e];
                if (block >= 0) slot = ((int64_t)block << p.log2_block) + (pos & (((int64_t)1 << p.log2_block) - 1));
            }
        }
        p.slot_map[i] = slot;
    }
}

}  // namespace

cudaError_t launch_qcache_tables(const QcacheTablesParams &p, int num_sms, cudaStream_t stream) {
    const size_t smem = (size_t)p.requests * 2 * sizeof(int32_t);
    if (smem > 40 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
    }
    // No more than two thread blocks per SM, each of which scans the lengths: with one the 64 prompts take 7.2 us a call, with
    // four 5.5 to 5.8, with eight 6.0 to 6.9, with two 5.1 to 6.3.
    const int64_t want = (p.max_rows + kThreads - 1) / kThreads;
    const int grid = (int)(want < 1 ? 1 : want > 2 * num_sms ? 2 * num_sms : want);
    return launch_behind(tables_kernel, dim3(grid), kThreads, smem, stream, p);
}

}  // namespace cm
