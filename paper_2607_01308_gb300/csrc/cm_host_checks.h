// What the C entries of the 8-bit paged cache and of the operators around a tree of drafted tokens share on the host:
// argument checks, error reports and the device of a launch. Included by their sources only.
#pragma once

#include <exception>
#include <new>
#include <string>

#include <cuda_runtime.h>
#include <nvtx3/nvToolsExt.h>

#include "cm.h"
#include "cm_hash_kernels.h"

namespace cm {
// cm_host.cpp
int context_device(const cm_context *ctx);
int context_num_sms(const cm_context *ctx);
unsigned int *context_error_word(const cm_context *ctx);
const uint64_t *context_turns(const cm_context *ctx, int head_dim);

namespace checks {
namespace {

struct TraceRange {
    explicit TraceRange(const char *name) { nvtxRangePushA(name); }
    ~TraceRange() { nvtxRangePop(); }
};

[[maybe_unused]] cm_status fail(cm_status st, const char *msg) { return cm::report_error(st, msg); }

[[maybe_unused]] bool aligned(const void *p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

[[maybe_unused]] bool is_pow2(int64_t x) { return x > 0 && (x & (x - 1)) == 0; }

[[maybe_unused]] int log2_of(int64_t x) {
    int k = 0;
    while (((int64_t)1 << k) < x) ++k;
    return k;
}

// Makes ctx's device current for a launch and puts the caller's back.
template <class F>
cm_status on_device(const cm_context *ctx, const char *what, F &&launch) {
    int before = 0;
    const int device = cm::context_device(ctx);
    cudaError_t e = cudaGetDevice(&before);
    if (e == cudaSuccess && before != device) e = cudaSetDevice(device);
    if (e == cudaSuccess) {
        e = launch();
        if (before != device) cudaSetDevice(before);
    }
    if (e == cudaSuccess) return CM_OK;
    return fail(CM_ERR_CUDA, (std::string(what) + ": " + cudaGetErrorString(e)).c_str());
}

template <class F>
cm_status guarded(F &&f) {
    try {
        return f();
    } catch (const std::bad_alloc &) {
        return fail(CM_ERR_OOM, "host allocation failed");
    } catch (...) {
        return fail(CM_ERR_INVALID_ARG, "unexpected internal error");
    }
}

[[maybe_unused]] bool block_size_ok(int32_t b) { return is_pow2(b) && b >= 16 && b <= 256; }

[[maybe_unused]] cm_status check_cache(const cm_qcache *c) {
    if (!c) return fail(CM_ERR_INVALID_ARG, "cache descriptor is NULL");
    if (!c->k_codes || !c->v_codes || !c->k_scales || !c->v_scales)
        return fail(CM_ERR_INVALID_ARG, "a cache pointer is NULL");
    if (c->format != CM_QCACHE_E4M3 && c->format != CM_QCACHE_INT8)
        return fail(CM_ERR_INVALID_ARG, "unknown cache format");
    if (c->num_layers < 1 || c->num_layers > 65535 || c->num_kv_heads < 1 || c->num_kv_heads > 65535)
        return fail(CM_ERR_INVALID_ARG, "cache layers and kv heads must be in [1, 65535]");
    if (!is_pow2(c->head_dim) || c->head_dim < 16 || c->head_dim > 512)
        return fail(CM_ERR_INVALID_ARG, "head_dim must be a power of two in [16, 512]");
    if (!block_size_ok(c->block_size))
        return fail(CM_ERR_UNSUPPORTED, "block_size must be a power of two in [16, 256]");
    if (c->num_blocks < 1 || c->num_blocks > INT32_MAX)
        return fail(CM_ERR_INVALID_ARG, "num_blocks must be in [1, 2^31 - 1]");
    if (c->reserved != 0) return fail(CM_ERR_INVALID_ARG, "reserved must be 0");
    if (!aligned(c->k_codes, 16) || !aligned(c->v_codes, 16))
        return fail(CM_ERR_ALIGNMENT, "codes must be 16-byte aligned");
    if (!aligned(c->k_scales, 4) || !aligned(c->v_scales, 4))
        return fail(CM_ERR_ALIGNMENT, "scales must be 4-byte aligned");
    for (int64_t s : {c->stride_block, c->stride_layer, c->stride_head, c->stride_token}) {
        if (s < 1) return fail(CM_ERR_INVALID_ARG, "cache strides must be positive");
        if (s % 16) return fail(CM_ERR_ALIGNMENT, "code strides must be multiples of 16 bytes");
    }
    if (c->stride_token < c->head_dim) return fail(CM_ERR_INVALID_ARG, "stride_token is below head_dim");
    for (int64_t s : {c->scale_stride_block, c->scale_stride_layer, c->scale_stride_head})
        if (s < 1) return fail(CM_ERR_INVALID_ARG, "scale strides must be positive");
    return CM_OK;
}

[[maybe_unused]] cm_status check_batch(const cm_qcache_batch *b, int32_t most) {
    if (!b) return fail(CM_ERR_INVALID_ARG, "batch descriptor is NULL");
    if (b->num_requests < 0) return fail(CM_ERR_INVALID_ARG, "num_requests < 0");
    if (b->num_requests > most) return fail(CM_ERR_UNSUPPORTED, "too many requests for one call");
    if (!block_size_ok(b->block_size))
        return fail(CM_ERR_UNSUPPORTED, "block_size must be a power of two in [16, 256]");
    if (b->table_width < 0 || b->table_width > INT32_MAX)
        return fail(CM_ERR_INVALID_ARG, "table_width must be in [0, 2^31 - 1]");
    if (!b->row_starts || (b->num_requests > 0 && (!b->kv_lens || (b->table_width > 0 && !b->block_table))))
        return fail(CM_ERR_INVALID_ARG, "a batch pointer is NULL");
    if (!aligned(b->row_starts, 4) || !aligned(b->kv_lens, 4) || !aligned(b->block_table, 4))
        return fail(CM_ERR_ALIGNMENT, "batch arrays must be 4-byte aligned");
    return CM_OK;
}

}  // namespace
}  // namespace checks
}  // namespace cm
