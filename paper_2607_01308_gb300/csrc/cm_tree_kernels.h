// Internal interface between the host side of the operators around a tree of drafted tokens (cm_tree.cpp)
// and their kernels: masks and positions (tree_plan.cu), norm and rotation of q and k (rotate.cu), the check of
// drafted tokens (tree_verify.cu) and the move of accepted rows (qcache_keep.cu). Not part of the public ABI.
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

#include "cm_qcache_kernels.h"

namespace cm {

constexpr int kTreeMaxNodes = 256;            // rows of a request that can be a tree: 8 words of a mask
constexpr int kTreeMaxWords = kTreeMaxNodes / 32;

// ---------------------------------------------------------------- masks and positions
struct TreePlanParams {
    const int32_t *row_starts, *context_lens;
    const int32_t *parents;                   // null: each row's is the one before it
    uint32_t *mask;                           // [total_rows][words], may be null
    int32_t *positions;                       // [total_rows], may be null
    int32_t requests, total_rows, words;
};
cudaError_t launch_tree_plan(const TreePlanParams &p, cudaStream_t stream);

// ---------------------------------------------------------------- norm and rotation
struct RotateParams {
    const uint16_t *in[2];                    // q, k
    uint16_t *out[2];
    const uint16_t *weight[2];                // null: no norm
    int64_t in_row[2], in_head[2], out_row[2], out_head[2];   // strides, elements
    const int32_t *positions;
    const uint64_t *turns;                    // [head_dim / 2]: turns per position, as fractions of 2^64
    int64_t rows;
    int32_t heads[2];
    int32_t head_dim;
    float eps;
};
cudaError_t launch_rotate(const RotateParams &p, int num_sms, cudaStream_t stream);

// ---------------------------------------------------------------- check of drafted tokens
struct TreeVerifyParams {
    const int32_t *row_starts, *parents, *tokens;
    const void *target, *draft;               // [total_rows][vocab], draft may be null
    int64_t target_stride, draft_stride;      // elements
    const float *accept, *sample;             // [total_rows], [requests]
    int32_t *path, *kept, *next_token;
    int32_t requests, total_rows, vocab, max_nodes, type;
};
cudaError_t launch_tree_verify(const TreeVerifyParams &p, cudaStream_t stream);

// ---------------------------------------------------------------- accepted rows to the front
struct QcacheKeepParams {
    uint8_t *codes[2];                        // K, V
    float *scales[2];
    int64_t stride_block, stride_layer, stride_head, stride_token;
    int64_t scale_stride_block, scale_stride_layer, scale_stride_head;
    int64_t num_blocks;
    const int32_t *block_table;
    int64_t table_width;
    const int32_t *row_starts, *kv_lens, *context_lens;
    const int32_t *path, *kept;
    int32_t *lens_out, *freed;
    int64_t *freed_count;
    int64_t max_freed;
    int32_t requests, total_rows;
    int32_t layers, heads, head_dim, log2_block, format;
    int32_t chunks;                           // thread blocks of a request
};
cudaError_t launch_qcache_keep(QcacheKeepParams p, int num_sms, cudaStream_t stream);

#ifdef __CUDACC__
// The rows of request r, within the buffers whatever row_starts says.
struct RequestRows {
    int first, n;
};
__device__ __forceinline__ RequestRows request_rows(const int32_t *row_starts, int r, int total_rows) {
    const int first = min(max(row_starts[r], 0), total_rows);
    return {first, min(max(row_starts[r + 1], first), total_rows) - first};
}
#endif

}  // namespace cm
