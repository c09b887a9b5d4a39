// Host side of the operators around a tree of drafted tokens (cm_qcache_tree, cm_qk_rotate, cm_tree_verify and
// cm_qcache_keep of include/cm.h): every argument that the host can see is checked before anything is launched. Nothing
// is allocated or kept, so the calls take no lock.
#include "cm.h"

#include <cmath>

#include "cm_host_checks.h"
#include "cm_tree_kernels.h"

namespace {

using namespace cm::checks;

// Byte ranges [a, a + n) and [b, b + m) share a byte.
bool overlap(const void *a, int64_t n, const void *b, int64_t m) {
    const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
    return a && b && n > 0 && m > 0 && x < y + (uintptr_t)m && y < x + (uintptr_t)n;
}

// Whether the wider of two strides (d at least, of several each) steps over all that the other reaches: rows of d elements do not meet then.
bool apart(int64_t stride_a, int64_t n_a, int64_t stride_b, int64_t n_b, int64_t d) {
    const bool a_first = stride_a < stride_b;
    const int64_t inner = a_first ? stride_a : stride_b, outer = a_first ? stride_b : stride_a, n = a_first ? n_a : n_b;
    return inner <= (outer - d) / (n - 1);
}

}  // namespace

extern "C" {

cm_status cm_qcache_tree(cm_context *ctx, const cm_qcache_batch *batch, const int32_t *context_lens, const int32_t *parents,
                         int32_t total_rows, int32_t words, uint32_t *mask, int32_t *positions, cm_stream_t stream) {
    TraceRange trace("cm_qcache_tree");
    return guarded([&]() -> cm_status {
        if (!ctx) return fail(CM_ERR_INVALID_ARG, "context is NULL");
        if (!batch) return fail(CM_ERR_INVALID_ARG, "batch descriptor is NULL");
        if (batch->num_requests < 0) return fail(CM_ERR_INVALID_ARG, "num_requests < 0");
        if (batch->num_requests > cm::kQcacheMaxRequests) return fail(CM_ERR_UNSUPPORTED, "too many requests for one call");
        if (total_rows < 0) return fail(CM_ERR_INVALID_ARG, "total_rows < 0");
        if (words < 1 || words > cm::kTreeMaxWords) return fail(CM_ERR_INVALID_ARG, "a mask has 1 to 8 words a row");
        if (batch->num_requests == 0 || total_rows == 0) return CM_OK;
        if (!batch->row_starts || !context_lens) return fail(CM_ERR_INVALID_ARG, "row_starts or context_lens is NULL");
        if (!aligned(batch->row_starts, 4) || !aligned(context_lens, 4) || !aligned(parents, 4) || !aligned(mask, 4) || !aligned(positions, 4))
            return fail(CM_ERR_ALIGNMENT, "arrays must be 4-byte aligned");
        const int64_t row_bytes = (int64_t)total_rows * 4;
        if (overlap(mask, row_bytes * words, parents, row_bytes) || overlap(positions, row_bytes, parents, row_bytes) ||
            overlap(mask, row_bytes * words, positions, row_bytes))
            return fail(CM_ERR_INVALID_ARG, "parents, mask and positions must not overlap");
        cm::TreePlanParams p{};
        p.row_starts = batch->row_starts;
        p.context_lens = context_lens;
        p.parents = parents;
        p.mask = mask;
        p.positions = positions;
        p.requests = batch->num_requests;
        p.total_rows = total_rows;
        p.words = words;
        return on_device(ctx, "tree launch", [&] { return cm::launch_tree_plan(p, reinterpret_cast<cudaStream_t>(stream)); });
    });
}

cm_status cm_qk_rotate(cm_context *ctx, const cm_qk_rows *rows, cm_stream_t stream) {
    TraceRange trace("cm_qk_rotate");
    return guarded([&]() -> cm_status {
        if (!ctx) return fail(CM_ERR_INVALID_ARG, "context is NULL");
        if (!rows) return fail(CM_ERR_INVALID_ARG, "rows descriptor is NULL");
        if (rows->reserved != 0) return fail(CM_ERR_INVALID_ARG, "reserved must be 0");
        if (!is_pow2(rows->head_dim) || rows->head_dim < 16 || rows->head_dim > 512)
            return fail(CM_ERR_INVALID_ARG, "head_dim must be a power of two in [16, 512]");
        if (rows->num_rows < 0 || rows->num_rows > INT32_MAX) return fail(CM_ERR_INVALID_ARG, "num_rows must be in [0, 2^31 - 1]");
        if (rows->num_q_heads < 0 || rows->num_q_heads > 65535 || rows->num_kv_heads < 0 || rows->num_kv_heads > 65535)
            return fail(CM_ERR_INVALID_ARG, "heads must be in [0, 65535]");
        if (!(rows->eps >= 0.f) || !std::isfinite(rows->eps)) return fail(CM_ERR_INVALID_ARG, "eps must be finite and not negative");
        if (rows->num_rows == 0 || rows->num_q_heads + rows->num_kv_heads == 0) return CM_OK;
        if ((rows->num_q_heads && (!rows->q || !rows->q_out)) || (rows->num_kv_heads && (!rows->k || !rows->k_out)) || !rows->positions)
            return fail(CM_ERR_INVALID_ARG, "q, k, an output or positions is NULL");
        for (const void *x : {rows->q, rows->k, (const void *)rows->q_out, (const void *)rows->k_out, rows->q_weight, rows->k_weight})
            if (!aligned(x, 16)) return fail(CM_ERR_ALIGNMENT, "rows and weights must be 16-byte aligned");
        if (!aligned(rows->positions, 4)) return fail(CM_ERR_ALIGNMENT, "positions must be 4-byte aligned");
        for (int64_t s : {rows->q_stride_row, rows->q_stride_head, rows->k_stride_row, rows->k_stride_head, rows->q_out_stride_row,
                          rows->q_out_stride_head, rows->k_out_stride_row, rows->k_out_stride_head}) {
            if (s < 0) return fail(CM_ERR_INVALID_ARG, "strides must not be negative");
            if (s % 8) return fail(CM_ERR_ALIGNMENT, "strides must be multiples of 8 elements");
        }
        const int64_t heads[2] = {rows->num_q_heads, rows->num_kv_heads};
        const int64_t out_row[2] = {rows->q_out_stride_row, rows->k_out_stride_row}, out_head[2] = {rows->q_out_stride_head, rows->k_out_stride_head};
        const int64_t in_row[2] = {rows->q_stride_row, rows->k_stride_row}, in_head[2] = {rows->q_stride_head, rows->k_stride_head};
        const void *in[2] = {rows->q, rows->k}, *out[2] = {rows->q_out, rows->k_out};
        for (int i = 0; i < 2; ++i) {
            const int64_t n_row = heads[i] ? rows->num_rows : 0, n_head = heads[i];
            const bool some_rows = n_row > 1, some_heads = n_head > 1;
            if ((some_rows && out_row[i] < rows->head_dim) || (some_heads && out_head[i] < rows->head_dim) ||
                (some_rows && some_heads && !apart(out_row[i], n_row, out_head[i], n_head, rows->head_dim)))
                return fail(CM_ERR_INVALID_ARG, "rows of an output lie on one another");
            if (in[i] == out[i] && ((some_rows && in_row[i] != out_row[i]) || (some_heads && in_head[i] != out_head[i])))
                return fail(CM_ERR_INVALID_ARG, "in place, the strides must be alike");
        }
        cm::RotateParams p{};
        p.in[0] = static_cast<const uint16_t *>(rows->q);
        p.in[1] = static_cast<const uint16_t *>(rows->k);
        p.out[0] = static_cast<uint16_t *>(rows->q_out);
        p.out[1] = static_cast<uint16_t *>(rows->k_out);
        p.weight[0] = static_cast<const uint16_t *>(rows->q_weight);
        p.weight[1] = static_cast<const uint16_t *>(rows->k_weight);
        p.in_row[0] = rows->q_stride_row;
        p.in_row[1] = rows->k_stride_row;
        p.in_head[0] = rows->q_stride_head;
        p.in_head[1] = rows->k_stride_head;
        for (int i = 0; i < 2; ++i) {
            p.out_row[i] = out_row[i];
            p.out_head[i] = out_head[i];
            p.heads[i] = (int32_t)heads[i];
        }
        p.positions = rows->positions;
        p.turns = cm::context_turns(ctx, rows->head_dim);
        p.rows = rows->num_rows;
        p.head_dim = rows->head_dim;
        p.eps = rows->eps;
        return on_device(ctx, "rotation launch", [&] {
            return cm::launch_rotate(p, cm::context_num_sms(ctx), reinterpret_cast<cudaStream_t>(stream));
        });
    });
}

cm_status cm_tree_verify(cm_context *ctx, const cm_tree_drafts *drafts, cm_stream_t stream) {
    TraceRange trace("cm_tree_verify");
    return guarded([&]() -> cm_status {
        if (!ctx) return fail(CM_ERR_INVALID_ARG, "context is NULL");
        if (!drafts) return fail(CM_ERR_INVALID_ARG, "drafts descriptor is NULL");
        if (drafts->type != CM_PROB_F32 && drafts->type != CM_PROB_BF16) return fail(CM_ERR_INVALID_ARG, "unknown probability type");
        if (drafts->num_requests < 0 || drafts->total_rows < 0) return fail(CM_ERR_INVALID_ARG, "num_requests < 0 or total_rows < 0");
        if (drafts->num_requests > cm::kQcacheMaxRequests) return fail(CM_ERR_UNSUPPORTED, "too many requests for one call");
        if (drafts->vocab < 1 || drafts->vocab > 1 << 20) return fail(CM_ERR_UNSUPPORTED, "vocab must be in [1, 2^20]");
        if (drafts->max_nodes < 1 || drafts->max_nodes > cm::kTreeMaxNodes)
            return fail(CM_ERR_INVALID_ARG, "max_nodes must be in [1, 256]");
        if (drafts->num_requests == 0) return CM_OK;
        if (!drafts->row_starts || !drafts->kept || !drafts->next_token || !drafts->sample ||
            (drafts->total_rows > 0 && (!drafts->parents || !drafts->tokens || !drafts->target || !drafts->accept || !drafts->path)))
            return fail(CM_ERR_INVALID_ARG, "a pointer other than draft is NULL");
        for (const void *x : {(const void *)drafts->row_starts, (const void *)drafts->parents, (const void *)drafts->tokens,
                              (const void *)drafts->accept, (const void *)drafts->sample, (const void *)drafts->path,
                              (const void *)drafts->kept, (const void *)drafts->next_token})
            if (!aligned(x, 4)) return fail(CM_ERR_ALIGNMENT, "int32 and fp32 arrays must be 4-byte aligned");
        const uintptr_t size = drafts->type == CM_PROB_F32 ? 4 : 2;
        if (!aligned(drafts->target, size) || !aligned(drafts->draft, size))
            return fail(CM_ERR_ALIGNMENT, "probabilities must be aligned to their size");
        if (drafts->target_stride < 0 || drafts->draft_stride < 0) return fail(CM_ERR_INVALID_ARG, "strides must not be negative");
        cm::TreeVerifyParams p{};
        p.row_starts = drafts->row_starts;
        p.parents = drafts->parents;
        p.tokens = drafts->tokens;
        p.target = drafts->target;
        p.draft = drafts->draft;
        p.target_stride = drafts->target_stride;
        p.draft_stride = drafts->draft_stride;
        p.accept = drafts->accept;
        p.sample = drafts->sample;
        p.path = drafts->path;
        p.kept = drafts->kept;
        p.next_token = drafts->next_token;
        p.requests = drafts->num_requests;
        p.total_rows = drafts->total_rows;
        p.vocab = drafts->vocab;
        p.max_nodes = drafts->max_nodes;
        p.type = drafts->type;
        return on_device(ctx, "verification launch", [&] { return cm::launch_tree_verify(p, reinterpret_cast<cudaStream_t>(stream)); });
    });
}

cm_status cm_qcache_keep(cm_context *ctx, const cm_qcache *cache, const cm_qcache_batch *batch, const int32_t *context_lens,
                         const int32_t *path, const int32_t *kept, int32_t total_rows, int32_t *lens_out, int32_t *freed,
                         int64_t max_freed, int64_t *freed_count, cm_stream_t stream) {
    TraceRange trace("cm_qcache_keep");
    return guarded([&]() -> cm_status {
        if (!ctx) return fail(CM_ERR_INVALID_ARG, "context is NULL");
        cm_status st = check_cache(cache);
        if (st != CM_OK) return st;
        st = check_batch(batch, cm::kQcacheMaxRequests);
        if (st != CM_OK) return st;
        if (batch->block_size != cache->block_size)
            return fail(CM_ERR_SHAPE_MISMATCH, "the batch's block_size is not the cache's");
        if (total_rows < 0 || max_freed < 0 || max_freed > INT32_MAX)
            return fail(CM_ERR_INVALID_ARG, "total_rows < 0, or max_freed not in [0, 2^31 - 1]");
        if (!freed_count || (max_freed > 0 && !freed) ||
            (batch->num_requests > 0 && (!context_lens || !kept || !lens_out || (total_rows > 0 && !path))))
            return fail(CM_ERR_INVALID_ARG, "a length, path, block list or count pointer is NULL");
        if (!aligned(context_lens, 4) || !aligned(path, 4) || !aligned(kept, 4) || !aligned(lens_out, 4) || !aligned(freed, 4) ||
            !aligned(freed_count, 8))
            return fail(CM_ERR_ALIGNMENT, "int32 arrays must be 4-byte, the count 8-byte aligned");
        const int64_t request_bytes = (int64_t)batch->num_requests * 4;
        for (const void *x : {(const void *)context_lens, (const void *)kept, (const void *)batch->kv_lens, (const void *)batch->row_starts})
            if (overlap(lens_out, request_bytes, x, request_bytes))
                return fail(CM_ERR_INVALID_ARG, "lens_out must not be one of the arrays that are read");
        cm::QcacheKeepParams p{};
        p.codes[0] = static_cast<uint8_t *>(cache->k_codes);
        p.codes[1] = static_cast<uint8_t *>(cache->v_codes);
        p.scales[0] = cache->k_scales;
        p.scales[1] = cache->v_scales;
        p.stride_block = cache->stride_block;
        p.stride_layer = cache->stride_layer;
        p.stride_head = cache->stride_head;
        p.stride_token = cache->stride_token;
        p.scale_stride_block = cache->scale_stride_block;
        p.scale_stride_layer = cache->scale_stride_layer;
        p.scale_stride_head = cache->scale_stride_head;
        p.num_blocks = cache->num_blocks;
        p.block_table = batch->block_table;
        p.table_width = batch->table_width;
        p.row_starts = batch->row_starts;
        p.kv_lens = batch->kv_lens;
        p.context_lens = context_lens;
        p.path = path;
        p.kept = kept;
        p.lens_out = lens_out;
        p.freed = freed;
        p.freed_count = freed_count;
        p.max_freed = max_freed;
        p.requests = batch->num_requests;
        p.total_rows = total_rows;
        p.layers = cache->num_layers;
        p.heads = cache->num_kv_heads;
        p.head_dim = cache->head_dim;
        p.log2_block = log2_of(cache->block_size);
        p.format = cache->format;
        return on_device(ctx, "cache move launch", [&] {
            return cm::launch_qcache_keep(p, cm::context_num_sms(ctx), reinterpret_cast<cudaStream_t>(stream));
        });
    });
}

}  // extern "C"
