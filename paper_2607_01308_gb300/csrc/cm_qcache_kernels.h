// Internal interface between the host side of the 8-bit cache operators (cm_qcache.cpp) and
// their kernels: block tables and slot maps (qcache_tables.cu), the cache write
// (qcache_append.cu) and attention (qcache_attention.cu, qcache_prefill.cu). Not part of the public ABI.
#pragma once

#include <cstddef>
#include <cstdint>

#include <cuda_runtime.h>

#include "cm.h"

namespace cm {

// ---------------------------------------------------------------- block tables
constexpr int kQcacheMaxRequests = 16384;   // per call: two words of shared memory each

struct QcacheTablesParams {
    const int32_t *old_lens, *new_lens;   // [requests]
    const int32_t *free_blocks;           // [num_free]
    int32_t *block_table;                 // [requests][table_width]
    int32_t *row_starts, *kv_lens;
    int32_t *context_out;                 // may be null
    int64_t *slot_map;                    // [max_rows]
    int64_t *counts;                      // [2]: blocks needed, rows
    int64_t num_free, table_width, max_rows;
    int32_t requests;
    int32_t log2_block;
};
cudaError_t launch_qcache_tables(const QcacheTablesParams &p, int num_sms, cudaStream_t stream);

// ---------------------------------------------------------------- cache write
struct QcacheAppendParams {
    uint8_t *codes[2];            // K, V: layer 0 of the call
    float *scales[2];
    const uint16_t *rows[2];      // bf16 rows: layer 0, head 0, row 0
    const int64_t *slots;         // [num_rows]
    int64_t num_rows, num_slots;  // slots of the pool (blocks * block size)
    int64_t stride_block, stride_layer, stride_head, stride_token;       // codes, bytes
    int64_t scale_stride_block, scale_stride_layer, scale_stride_head;   // elements
    int64_t row_stride_layer, row_stride_head, row_stride_row;           // bf16 elements
    int32_t layers, heads, head_dim, log2_block;
    int32_t format;
    int32_t window;               // rows per thread block (the leaders among them are its work)
};
cudaError_t launch_qcache_append(QcacheAppendParams p, int num_sms, cudaStream_t stream);

// ---------------------------------------------------------------- attention
// A range of kv tiles that is cut: the row tile and kv head that it belongs to, and the last thread
// block that has a part of it.
struct QcacheSplit {
    int32_t request, head, row_tile, row0, rows, last_block;
};

struct QcacheAttentionParams {
    const uint8_t *k, *v;         // codes of the layer
    const float *k_scale, *v_scale;
    int64_t stride_block, stride_head, stride_token;
    int64_t scale_stride_block, scale_stride_head;
    int64_t num_blocks;
    const int32_t *block_table;
    int64_t table_width;
    const int32_t *row_starts, *kv_lens;
    const int32_t *context_lens;  // [requests]
    const uint16_t *q;
    uint16_t *out;
    float *lse;                   // may be null
    int64_t q_stride_row, q_stride_head, out_stride_row, out_stride_head;
    float *part_o;                // workspace: partial outputs, then their (maximum, sum) pairs
    float *part_ml;
    unsigned int *arrived;        // decode: parts of a range that have come
    QcacheSplit *splits;          // prefill: the range that each thread block begins and does not end
    unsigned int *error;          // the context's word: bit 0 set when a bounded wait ran out
    float scale_log2;             // softmax scale * log2(e)
    int32_t requests, heads, group, head_dim, log2_block;
    int32_t total_rows, causal, format;
    int32_t no_context;           // -1: context_lens is another array of that size, and no request was cut short; else 0
    int32_t withhold;             // prefill, failure injection: an arrival that does not come, in thread block 0
};

constexpr int kQcacheWithholdQueries = 1;   // of the query rows
constexpr int kQcacheWithholdEntries = 2;   // of every tile's blocks and scales, which are not looked up either

// The workspace holds, for every thread block of a launch, two partial results and an arrival
// counter or a QcacheSplit.
constexpr int kQcacheDecodeBlocksPerSm = 4;
constexpr int kQcacheMaxAttentionRequests = 4096;   // a word of shared memory each
size_t qcache_workspace_bytes(int head_dim, int num_sms);
void qcache_workspace_split(QcacheAttentionParams &p, void *workspace, int num_sms);
// `rows_per_request`: the largest number of query rows of one request that is expected.
cudaError_t launch_qcache_attention(const QcacheAttentionParams &p, int rows_per_request, int num_sms, int device,
                                    cudaStream_t stream);
// The kernel for more rows per request, and the part rows of one of its thread blocks.
cudaError_t launch_qcache_prefill(const QcacheAttentionParams &p, int num_sms, int device, cudaStream_t stream);
size_t qcache_prefill_part_rows(int head_dim);

#ifdef __CUDACC__
// Launches a kernel that may be set up while the one before it in the stream ends. Its threads call
// after_kernels_before() before they read or write global memory; nothing else is relaxed. (The
// kernels read with plain loads throughout: what a kernel before still writes while this one is set up is not
// read-only for its life, as the non-coherent loads ask.)
template <class... Params, class... Args>
cudaError_t launch_behind(void (*kernel)(Params...), dim3 grid, unsigned int threads, size_t shared, cudaStream_t stream, const Args &...args) {
    cudaLaunchAttribute early;
    early.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    early.val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = grid;
    config.blockDim = dim3(threads);
    config.dynamicSmemBytes = shared;
    config.stream = stream;
    config.attrs = &early;
    config.numAttrs = 1;
    return cudaLaunchKernelEx(&config, kernel, args...);
}

// Waits until the kernels before this one have ended and their writes are seen. The next kernel is set up
// when this one's blocks have ended: letting it in from the start held up short kernels (one token over
// 1,041 cached: 8.4 us against 9.3).
__device__ __forceinline__ void after_kernels_before() {
    asm volatile("griddepcontrol.wait;" ::: "memory");
}
#endif

}  // namespace cm
