// Host side of the 8-bit paged cache (cm_qcache_* of include/cm.h): every argument that the host
// can see is checked before anything is launched. Nothing is allocated or kept, so the calls take
// no lock.
#include "cm.h"
#include "cm_testing.h"

#include <cmath>

#include "cm_host_checks.h"
#include "cm_tree_kernels.h"

namespace {

using namespace cm::checks;

// What a call asks for besides causal or whole attention.
struct Extras {
    int32_t withhold;             // 0, or what the many-rows kernel is to wait for in vain (failure injection; that kernel
                                  // then runs whatever the rows)
    bool trees;                   // rows see their context and the rows that tree_mask names
    const uint32_t *tree_mask;
    int32_t tree_words;
};

cm_status attend(cm_context *ctx, const cm_qcache *cache, int32_t layer, const cm_qcache_batch *batch,
                 const cm_qcache_query *query, void *workspace, int64_t workspace_bytes, cm_stream_t stream,
                 const Extras &extras) {
    TraceRange trace(extras.trees ? "cm_qcache_attend_tree" : "cm_qcache_attend");
    return guarded([&]() -> cm_status {
        if (!ctx) return fail(CM_ERR_INVALID_ARG, "context is NULL");
        cm_status st = check_cache(cache);
        if (st != CM_OK) return st;
        st = check_batch(batch, cm::kQcacheMaxAttentionRequests);
        if (st != CM_OK) return st;
        if (!query) return fail(CM_ERR_INVALID_ARG, "query descriptor is NULL");
        if (cache->head_dim < 32 || cache->head_dim > 256)
            return fail(CM_ERR_UNSUPPORTED, "attention needs head_dim 32, 64, 128 or 256");
        if (layer < 0 || layer >= cache->num_layers) return fail(CM_ERR_INVALID_ARG, "layer outside the cache");
        if (batch->block_size != cache->block_size)
            return fail(CM_ERR_SHAPE_MISMATCH, "the batch's block_size is not the cache's");
        if (query->flags & ~CM_QCACHE_CONTEXT_LENS) return fail(CM_ERR_INVALID_ARG, "unknown query flags");
        const int32_t *context_lens = query->flags & CM_QCACHE_CONTEXT_LENS ? query->context_lens : nullptr;
        if (!aligned(context_lens, 4)) return fail(CM_ERR_ALIGNMENT, "context_lens must be 4-byte aligned");
        if (query->num_q_heads < 1 || query->num_q_heads % cache->num_kv_heads)
            return fail(CM_ERR_SHAPE_MISMATCH, "num_q_heads is not a multiple of the cache's kv heads");
        const int32_t group = query->num_q_heads / cache->num_kv_heads;
        if (group > 128) return fail(CM_ERR_UNSUPPORTED, "more than 128 query heads to a kv head");
        if (query->total_rows < 0 || query->max_rows_per_request < 0)
            return fail(CM_ERR_INVALID_ARG, "total_rows < 0 or max_rows_per_request < 0");
        const float scale_log2 = query->softmax_scale * 1.44269504088896340736f;
        if (!std::isfinite(scale_log2)) return fail(CM_ERR_INVALID_ARG, "softmax_scale (times log2 e) is not finite");
        if (extras.trees && (extras.tree_words < 1 || extras.tree_words > cm::kTreeMaxWords))
            return fail(CM_ERR_INVALID_ARG, "a mask has 1 to 8 words a row");
        if (query->total_rows == 0 || batch->num_requests == 0) return CM_OK;
        if (extras.trees && !extras.tree_mask) return fail(CM_ERR_INVALID_ARG, "mask is NULL");
        if (!aligned(extras.tree_mask, 4)) return fail(CM_ERR_ALIGNMENT, "mask must be 4-byte aligned");
        if (!query->q || !query->out || !workspace) return fail(CM_ERR_INVALID_ARG, "q, out or workspace is NULL");
        if (!aligned(query->q, 16) || !aligned(query->out, 16) || !aligned(query->lse, 4) || !aligned(workspace, 16))
            return fail(CM_ERR_ALIGNMENT, "q, out and workspace must be 16-byte aligned");
        for (int64_t s : {query->q_stride_row, query->q_stride_head, query->out_stride_row, query->out_stride_head}) {
            if (s < 0) return fail(CM_ERR_INVALID_ARG, "row strides must not be negative");
            if (s % 8) return fail(CM_ERR_ALIGNMENT, "row strides must be multiples of 8 elements");
        }
        if ((query->total_rows > 1 && query->out_stride_row < cache->head_dim) ||
            (query->num_q_heads > 1 && query->out_stride_head < cache->head_dim))
            return fail(CM_ERR_INVALID_ARG, "rows of out lie on one another");
        const int num_sms = cm::context_num_sms(ctx);
        if (workspace_bytes < 0 || (uint64_t)workspace_bytes < cm::qcache_workspace_bytes(cache->head_dim, num_sms))
            return fail(CM_ERR_CAPACITY, "workspace is smaller than cm_qcache_workspace says");
        const double tiles = (double)batch->table_width * batch->block_size / 64 + 9;   // and their setup
        const double row_tiles = (double)query->total_rows * group / 8 + batch->num_requests;
        if (tiles * row_tiles >= 2147483648.0)
            return fail(CM_ERR_UNSUPPORTED, "too much work for one call: split the rows");
        cm::QcacheAttentionParams p{};
        p.k = static_cast<const uint8_t *>(cache->k_codes) + layer * cache->stride_layer;
        p.v = static_cast<const uint8_t *>(cache->v_codes) + layer * cache->stride_layer;
        p.k_scale = cache->k_scales + layer * cache->scale_stride_layer;
        p.v_scale = cache->v_scales + layer * cache->scale_stride_layer;
        p.stride_block = cache->stride_block;
        p.stride_head = cache->stride_head;
        p.stride_token = cache->stride_token;
        p.scale_stride_block = cache->scale_stride_block;
        p.scale_stride_head = cache->scale_stride_head;
        p.num_blocks = cache->num_blocks;
        p.block_table = batch->block_table;
        p.table_width = batch->table_width;
        p.row_starts = batch->row_starts;
        p.kv_lens = batch->kv_lens;
        p.context_lens = context_lens ? context_lens : batch->kv_lens;
        p.no_context = context_lens ? 0 : -1;
        p.q = static_cast<const uint16_t *>(query->q);
        p.out = static_cast<uint16_t *>(query->out);
        p.lse = query->lse;
        p.q_stride_row = query->q_stride_row;
        p.q_stride_head = query->q_stride_head;
        p.out_stride_row = query->out_stride_row;
        p.out_stride_head = query->out_stride_head;
        p.scale_log2 = scale_log2;
        p.requests = batch->num_requests;
        p.heads = cache->num_kv_heads;
        p.group = group;
        p.head_dim = cache->head_dim;
        p.log2_block = log2_of(cache->block_size);
        p.total_rows = query->total_rows;
        p.causal = query->causal != 0 && !extras.trees;
        p.tree = extras.tree_mask;
        p.tree_words = extras.tree_words;
        p.format = cache->format;
        p.error = cm::context_error_word(ctx);
        p.withhold = extras.withhold;
        cm::qcache_workspace_split(p, workspace, num_sms);
        const int64_t rows = (int64_t)(query->max_rows_per_request ? query->max_rows_per_request : query->total_rows) * group;
        return on_device(ctx, "attention launch", [&] {
            const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
            if (extras.withhold)   // a tree's kernel goes by the rows, the others' is the one of long prompts
                return cm::launch_qcache_prefill(p, (int)(extras.trees && rows < INT32_MAX ? rows : INT32_MAX), num_sms,
                                                 cm::context_device(ctx), s);
            return cm::launch_qcache_attention(p, (int)(rows < INT32_MAX ? rows : INT32_MAX), num_sms,
                                               cm::context_device(ctx), s);
        });
    });
}

}  // namespace

extern "C" {

cm_status cm_qcache_schedule(cm_context *ctx, const cm_qcache_batch *batch, const int32_t *context_lens,
                             const int32_t *new_lens, const int32_t *free_blocks, int64_t num_free,
                             int64_t *slot_map, int64_t max_rows, int64_t *counts, cm_stream_t stream) {
    return cm_qcache_schedule_cut(ctx, batch, context_lens, new_lens, free_blocks, num_free, slot_map, max_rows,
                                  counts, nullptr, stream);
}

cm_status cm_qcache_schedule_cut(cm_context *ctx, const cm_qcache_batch *batch, const int32_t *context_lens,
                                 const int32_t *new_lens, const int32_t *free_blocks, int64_t num_free,
                                 int64_t *slot_map, int64_t max_rows, int64_t *counts, int32_t *context_out,
                                 cm_stream_t stream) {
    TraceRange trace("cm_qcache_schedule");
    return guarded([&]() -> cm_status {
        if (!ctx) return fail(CM_ERR_INVALID_ARG, "context is NULL");
        cm_status st = check_batch(batch, cm::kQcacheMaxRequests);
        if (st != CM_OK) return st;
        if (num_free < 0 || max_rows < 0 || max_rows > INT32_MAX)
            return fail(CM_ERR_INVALID_ARG, "num_free < 0, or max_rows not in [0, 2^31 - 1]");
        if ((batch->num_requests > 0 && (!context_lens || !new_lens)) || (num_free > 0 && !free_blocks) ||
            (max_rows > 0 && !slot_map) || !counts)
            return fail(CM_ERR_INVALID_ARG, "a length, free-list, slot or count pointer is NULL");
        if (!aligned(context_lens, 4) || !aligned(new_lens, 4) || !aligned(free_blocks, 4) ||
            !aligned(context_out, 4) || !aligned(slot_map, 8) || !aligned(counts, 8))
            return fail(CM_ERR_ALIGNMENT, "int32 arrays must be 4-byte, int64 arrays 8-byte aligned");
        if (batch->num_requests > 0 && (context_lens == batch->kv_lens || new_lens == batch->kv_lens))
            return fail(CM_ERR_INVALID_ARG, "kv_lens must not be one of the length inputs");
        if (context_out && batch->num_requests > 0 &&
            (context_out == context_lens || context_out == new_lens || context_out == batch->kv_lens || context_out == batch->row_starts))
            return fail(CM_ERR_INVALID_ARG, "context_out must not be another of the length arrays");
        cm::QcacheTablesParams p{};
        p.old_lens = context_lens;
        p.new_lens = new_lens;
        p.free_blocks = free_blocks;
        p.block_table = batch->block_table;
        p.row_starts = batch->row_starts;
        p.kv_lens = batch->kv_lens;
        p.context_out = context_out;
        p.slot_map = slot_map;
        p.counts = counts;
        p.num_free = num_free;
        p.table_width = batch->table_width;
        p.max_rows = max_rows;
        p.requests = batch->num_requests;
        p.log2_block = log2_of(batch->block_size);
        return on_device(ctx, "block table launch", [&] {
            return cm::launch_qcache_tables(p, cm::context_num_sms(ctx), reinterpret_cast<cudaStream_t>(stream));
        });
    });
}

cm_status cm_qcache_append(cm_context *ctx, const cm_qcache *cache, int32_t layer, int32_t num_layers,
                           const void *k, const void *v, int64_t stride_layer, int64_t stride_head,
                           int64_t stride_row, const int64_t *slot_map, int64_t num_rows,
                           cm_stream_t stream) {
    TraceRange trace("cm_qcache_append");
    return guarded([&]() -> cm_status {
        if (!ctx) return fail(CM_ERR_INVALID_ARG, "context is NULL");
        cm_status st = check_cache(cache);
        if (st != CM_OK) return st;
        if (layer < 0 || num_layers < 1 || num_layers > cache->num_layers - layer)
            return fail(CM_ERR_INVALID_ARG, "layers outside the cache");
        if (num_rows < 0 || num_rows > INT32_MAX)
            return fail(CM_ERR_INVALID_ARG, "num_rows must be in [0, 2^31 - 1]");
        if (num_rows == 0) return CM_OK;
        if (!k || !v || !slot_map) return fail(CM_ERR_INVALID_ARG, "k, v or slot_map is NULL");
        if (!aligned(k, 16) || !aligned(v, 16) || !aligned(slot_map, 8))
            return fail(CM_ERR_ALIGNMENT, "k and v must be 16-byte, slot_map 8-byte aligned");
        for (int64_t s : {stride_layer, stride_head, stride_row}) {
            if (s < 0) return fail(CM_ERR_INVALID_ARG, "row strides must not be negative");
            if (s % 8) return fail(CM_ERR_ALIGNMENT, "row strides must be multiples of 8 elements");
        }
        cm::QcacheAppendParams p{};
        p.codes[0] = static_cast<uint8_t *>(cache->k_codes) + layer * cache->stride_layer;
        p.codes[1] = static_cast<uint8_t *>(cache->v_codes) + layer * cache->stride_layer;
        p.scales[0] = cache->k_scales + layer * cache->scale_stride_layer;
        p.scales[1] = cache->v_scales + layer * cache->scale_stride_layer;
        p.rows[0] = static_cast<const uint16_t *>(k);
        p.rows[1] = static_cast<const uint16_t *>(v);
        p.slots = slot_map;
        p.num_rows = num_rows;
        p.num_slots = cache->num_blocks * cache->block_size;
        p.stride_block = cache->stride_block;
        p.stride_layer = cache->stride_layer;
        p.stride_head = cache->stride_head;
        p.stride_token = cache->stride_token;
        p.scale_stride_block = cache->scale_stride_block;
        p.scale_stride_layer = cache->scale_stride_layer;
        p.scale_stride_head = cache->scale_stride_head;
        p.row_stride_layer = stride_layer;
        p.row_stride_head = stride_head;
        p.row_stride_row = stride_row;
        p.layers = num_layers;
        p.heads = cache->num_kv_heads;
        p.head_dim = cache->head_dim;
        p.log2_block = log2_of(cache->block_size);
        p.format = cache->format;
        return on_device(ctx, "cache write launch", [&] {
            return cm::launch_qcache_append(p, cm::context_num_sms(ctx), reinterpret_cast<cudaStream_t>(stream));
        });
    });
}

cm_status cm_qcache_attend(cm_context *ctx, const cm_qcache *cache, int32_t layer,
                           const cm_qcache_batch *batch, const cm_qcache_query *query, void *workspace,
                           int64_t workspace_bytes, cm_stream_t stream) {
    return attend(ctx, cache, layer, batch, query, workspace, workspace_bytes, stream, Extras{});
}

cm_status cm_qcache_attend_tree(cm_context *ctx, const cm_qcache *cache, int32_t layer,
                                const cm_qcache_batch *batch, const cm_qcache_query *query, const uint32_t *mask,
                                int32_t words, void *workspace, int64_t workspace_bytes, cm_stream_t stream) {
    return attend(ctx, cache, layer, batch, query, workspace, workspace_bytes, stream, Extras{0, true, mask, words});
}

cm_status cm_testing_qcache_attend_withheld(cm_context *ctx, const cm_qcache *cache, int32_t layer,
                                            const cm_qcache_batch *batch, const cm_qcache_query *query,
                                            void *workspace, int64_t workspace_bytes, int32_t what,
                                            cm_stream_t stream) {
    if (what != cm::kQcacheWithholdQueries && what != cm::kQcacheWithholdEntries)
        return fail(CM_ERR_INVALID_ARG, "nothing that can be withheld");
    return attend(ctx, cache, layer, batch, query, workspace, workspace_bytes, stream, Extras{what, false, nullptr, 0});
}

cm_status cm_testing_qcache_attend_tree_withheld(cm_context *ctx, const cm_qcache *cache, int32_t layer,
                                                 const cm_qcache_batch *batch, const cm_qcache_query *query,
                                                 const uint32_t *mask, int32_t words, void *workspace, int64_t workspace_bytes,
                                                 int32_t what, cm_stream_t stream) {
    if (what != cm::kQcacheWithholdQueries && what != cm::kQcacheWithholdEntries)
        return fail(CM_ERR_INVALID_ARG, "nothing that can be withheld");
    return attend(ctx, cache, layer, batch, query, workspace, workspace_bytes, stream, Extras{what, true, mask, words});
}

cm_status cm_qcache_workspace(cm_context *ctx, int32_t head_dim, int64_t *out_bytes) {
    return guarded([&]() -> cm_status {
        if (!ctx) return fail(CM_ERR_INVALID_ARG, "context is NULL");
        if (!out_bytes) return fail(CM_ERR_INVALID_ARG, "out_bytes is NULL");
        if (!is_pow2(head_dim) || head_dim < 32 || head_dim > 256)
            return fail(CM_ERR_UNSUPPORTED, "attention needs head_dim 32, 64, 128 or 256");
        *out_bytes = (int64_t)cm::qcache_workspace_bytes(head_dim, cm::context_num_sms(ctx));
        return CM_OK;
    });
}

}  // extern "C"
