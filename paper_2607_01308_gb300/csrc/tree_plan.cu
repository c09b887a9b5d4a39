// Ancestor masks and positions of drafted tokens, from their parents.
//
// Row i of a request was drafted behind row a(i) < i of it, or behind the context alone:
//   mask(i) = {i} u mask(a(i)),   position(i) = context + depth(i),   depth(i) = depth(a(i)) + 1
// A thread walks from its row to the root through the parents in shared memory. Parents come before their
// rows, so the words of a mask are met from the last to the first and each is held in a register until the
// walk leaves it. Bound by latency: lengths, parents, and a shared-memory read for each level (64 trees of 26 rows
// 2.1 us, 509 of up to 200 rows 4.0 us).
#include "cm_tree_kernels.h"

namespace cm {
namespace {

constexpr int kThreads = 256;
constexpr int kRowsPerBlock = 2048;           // of one request, where they are not a tree

__device__ __forceinline__ int32_t position(int64_t context, int64_t depth) { return (int32_t)min(context + depth, (int64_t)INT32_MAX); }

__global__ void __launch_bounds__(kThreads) plan_kernel(const __grid_constant__ TreePlanParams p) {
    __shared__ int16_t parent[kTreeMaxNodes];
    after_kernels_before();
    const int r = blockIdx.x, limit = 32 * p.words;
    const RequestRows q = request_rows(p.row_starts, r, p.total_rows);
    const int64_t context = max(p.context_lens[r], 0);
    if (p.parents && blockIdx.y == 0) {
        for (int i = threadIdx.x; i < min(q.n, limit); i += kThreads) {
            const int a = p.parents[q.first + i];
            parent[i] = (int16_t)(a >= 0 && a < i ? a : -1);
        }
        __syncthreads();
    }
    for (int64_t at = blockIdx.y * kThreads + threadIdx.x; at < q.n; at += gridDim.y * kThreads) {
        const int i = (int)at;
        const int64_t row = q.first + at;
        uint32_t *mask = p.mask ? p.mask + row * p.words : nullptr;
        if (p.parents && i < limit) {
            if (blockIdx.y != 0) continue;    // the first block has their parents
            int depth = 0, word = i >> 5;
            uint32_t bits = 1u << (i & 31);
            if (mask)
                for (int w = p.words - 1; w > word; --w) mask[w] = 0;
            for (int a = parent[i]; a >= 0; a = parent[a], ++depth) {
                if (a >> 5 != word) {
                    if (mask) {
                        mask[word] = bits;
                        for (int w = word - 1; w > a >> 5; --w) mask[w] = 0;
                    }
                    word = a >> 5;
                    bits = 0;
                }
                bits |= 1u << (a & 31);
            }
            if (mask) {
                mask[word] = bits;
                for (int w = word - 1; w >= 0; --w) mask[w] = 0;
            }
            if (p.positions) p.positions[row] = position(context, depth);
        } else {
            // rows one behind another, or behind the tree's last: those see the context alone
            if (mask)
                for (int w = 0; w < p.words; ++w)
                    mask[w] = p.parents || i >= limit ? 0u : i >= 32 * w + 31 ? ~0u : i < 32 * w ? 0u : (2u << (i & 31)) - 1;
            if (p.positions) p.positions[row] = position(context, p.parents ? 0 : i);
        }
    }
}

}  // namespace

cudaError_t launch_tree_plan(const TreePlanParams &p, cudaStream_t stream) {
    // more blocks for a request where the rows are too many for trees
    const int64_t per = ((int64_t)p.total_rows + p.requests - 1) / p.requests;
    const int64_t blocks = (per + kRowsPerBlock - 1) / kRowsPerBlock;
    const dim3 grid(p.requests, (unsigned)(blocks < 1 ? 1 : blocks > 256 ? 256 : blocks));
    return launch_behind(plan_kernel, grid, kThreads, 0, stream, p);
}

}  // namespace cm
