// The rows of an accepted path to the front of their request's new tokens, in every layer of an 8-bit paged
// cache, and the blocks behind them.
//
// Request r holds c tokens in front of its new rows; path_i, ascending, is the i-th accepted one: token c + path_i becomes
// token c + i. Rows in front of the first with path_i > i stay as they are. For each block that takes others, of
// each layer and head, and for K and V on their own:
//   scale' = max(the block's scale if tokens in front of the moved ones stay in it, the scales of the blocks they come from)
//   code'  = code * (scale of its block / scale') to nearest even; as it is where the ratio is 1
// so a value that moves is rounded once more at most, and not at all if the scales are alike.
//
// path_i >= i, so what a block takes comes from itself or from later blocks, and a warp that goes through one
// (layer, head, K or V) of a request block by block, and reads some rows (kHeld * 512 / head_dim of them) before it writes
// them, never reads what it has written. A thread block looks up where a request's rows lie once, for several layers and
// heads. One more thread block adds up the lengths and lists the blocks given back. Bound by the chain of dependent reads:
// lengths, path and table, then for each pair of heads that a warp takes codes and scales, and, where a scale grows, the tokens that
// stay, some rows after another. 64 requests, 36 layers of 8 heads of 128, two to three such rounds to a warp, about two rows moved in
// each: 10.0 us again and again on one cache, whose scales have grown then; 13 where codes and scales are not in L2, 33 there where some
// 4,100 scales grow. Four heads to a warp 9.9 instead of 10.0, but 4.4 instead of 3.5 for 6 requests of 4 layers; one head 10.9.
#include "cm_tree_kernels.h"

#include "cm_qcache_codes.h"

namespace cm {
namespace {

constexpr int kThreads = 256, kWarps = kThreads / 32;
constexpr int kPairs = 2;                     // (layer, head) that a warp moves at a time, K and V of each
constexpr int kHeld = 1;                      // vectors of a lane of each that are read before they are written
constexpr int kBlocksPerSm = 3;

// What entry i of a request's path names: places of the row's present and new slot, negative if there are none.
struct Place {
    int block, at;                            // the token's block and its place in it
};

struct Request {
    int first, n;                             // rows
    int64_t context, kv;
};

__device__ __forceinline__ Request request(const QcacheKeepParams &p, int r) {
    const RequestRows q = request_rows(p.row_starts, r, p.total_rows);
    const int64_t cap = min(p.table_width << p.log2_block, (int64_t)INT32_MAX);
    return {q.first, q.n, max(p.context_lens[r], 0), min((int64_t)max(p.kv_lens[r], 0), cap)};
}

__device__ __forceinline__ Place place(const QcacheKeepParams &p, int r, const Request &q, int64_t token) {
    if (token >= q.kv) return {-1, 0};
    const int b = p.block_table[r * p.table_width + (token >> p.log2_block)];
    return {b >= 0 && b < p.num_blocks ? b : -1, (int)(token & ((1 << p.log2_block) - 1))};
}

// Whether path entry `now` (after `before`) is one more accepted row that the cache holds.
__device__ __forceinline__ bool follows(const Request &q, int before, int now) { return now > before && now < q.n; }

template <int FORMAT>
__device__ __forceinline__ uint4 rescale(const uint4 &x, float ratio) {
    if (ratio == 1.f) return x;
    return make_uint4(shrink<FORMAT>(x.x, ratio), shrink<FORMAT>(x.y, ratio), shrink<FORMAT>(x.z, ratio), shrink<FORMAT>(x.w, ratio));
}

// K and V of up to kPairs (layer, head) of a request by a warp: their rows lie alike, so that they are read together.
template <int FORMAT>
__device__ __forceinline__ void move_rows(const QcacheKeepParams &p, int pair0, const Place *from, const Place *to, int begin, int end) {
    constexpr int kTasks = 2 * kPairs;
    const int lane = threadIdx.x % 32;
    const int log2_vecs = 31 - __clz(p.head_dim) - 4, row = lane >> log2_vecs, rows = 32 >> log2_vecs;
    uint8_t *codes[kTasks];
    float *scales[kTasks];
    const int tasks = 2 * min(kPairs, p.layers * p.heads - pair0);
#pragma unroll
    for (int u = 0; u < kTasks; ++u) {
        const int pair = pair0 + (u < tasks ? u / 2 : 0);
        const int64_t layer = pair / p.heads, head = pair - layer * p.heads;
        codes[u] = p.codes[u % 2] + layer * p.stride_layer + head * p.stride_head + (lane & ((1 << log2_vecs) - 1)) * 16;
        scales[u] = p.scales[u % 2] + layer * p.scale_stride_layer + head * p.scale_stride_head;
    }
    auto code_at = [&](int u, int64_t offset) { return reinterpret_cast<uint4 *>(codes[u] + offset); };
    auto place_at = [&](const Place &x, int more) { return x.block * p.stride_block + (x.at + more) * p.stride_token; };
    for (int i0 = begin; i0 < end;) {
        const Place first = to[i0];
        const int i1 = min(end, i0 + (1 << p.log2_block) - first.at);
        const int64_t scale_at = first.block * p.scale_stride_block;
        // the first rows are on their way while the scales are looked at
        uint4 x[kTasks][kHeld];
        float s[kTasks][kHeld], old[kTasks], now[kTasks];
        auto load = [&](int base) {
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                const int i = base + j * rows + row;
                if (i < i1) {
                    const Place f = from[i];
                    const int64_t at = place_at(f, 0), scale = f.block * p.scale_stride_block;
#pragma unroll
                    for (int u = 0; u < kTasks; ++u)
                        if (u < tasks) {
                            x[u][j] = *code_at(u, at);
                            s[u][j] = scales[u][scale];
                        }
                }
            }
        };
        load(i0);
#pragma unroll
        for (int u = 0; u < kTasks; ++u) now[u] = old[u] = first.at && u < tasks ? scales[u][scale_at] : 0.f;
        for (int i = i0 + lane; i < i1; i += 32) {
            const int64_t scale = from[i].block * p.scale_stride_block;
#pragma unroll
            for (int u = 0; u < kTasks; ++u)
                if (u < tasks) now[u] = fmaxf(now[u], scales[u][scale]);
        }
#pragma unroll
        for (int u = 0; u < kTasks; ++u)
#pragma unroll
            for (int d = 16; d; d /= 2) now[u] = fmaxf(now[u], __shfl_xor_sync(~0u, now[u], d));
        for (int base = i0; base < i1; base += kHeld * rows) {
            if (base != i0) load(base);
            __syncwarp();                     // all of them are read before one is written over
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                const int i = base + j * rows + row;
                if (i < i1) {
                    const int64_t at = place_at(first, i - i0);
#pragma unroll
                    for (int u = 0; u < kTasks; ++u)
                        if (u < tasks) *code_at(u, at) = rescale<FORMAT>(x[u][j], s[u][j] == now[u] ? 1.f : __fdiv_rn(s[u][j], now[u]));
                }
            }
        }
#pragma unroll
        for (int u = 0; u < kTasks; ++u)
            if (first.at && now[u] > old[u]) {          // the tokens that stay in the block (old: 0 beyond the tasks, and now too)
                const float ratio = __fdiv_rn(old[u], now[u]);
#pragma unroll 2
                for (int t = row; t < first.at; t += rows) {
                    uint4 *at = code_at(u, first.block * p.stride_block + t * p.stride_token);
                    *at = rescale<FORMAT>(*at, ratio);
                }
            }
        __syncwarp();                         // every lane has read the scales
#pragma unroll
        for (int u = 0; u < kTasks; ++u)
            if (u < tasks && lane == u) scales[u][scale_at] = now[u];
        __syncwarp();
        i0 = i1;
    }
}

// The last thread block: new lengths, and the blocks of the pool that no token is left in, in the requests' order. (A table has entries
// that name none where the free list was too short; on a free list they would be handed out in place of blocks that are there.)
__device__ __forceinline__ void count_blocks(const QcacheKeepParams &p) {
    __shared__ int64_t warp_sum[kWarps];
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    int64_t total = 0;
    for (int r0 = 0; r0 < p.requests; r0 += kThreads) {
        const int r = r0 + tid;
        int64_t n = 0, given = 0;              // table entries behind the last that is needed; those that name a block
        const int32_t *entries = nullptr;
        auto named = [&](int32_t b) { return b >= 0 && b < p.num_blocks; };
        if (r < p.requests) {
            const Request q = request(p, r);
            const int most = min(min(max(p.kept[r], 0), q.n), kTreeMaxNodes);
            int kept = 0, before = -1;
            for (; kept < most; ++kept) {
                const int now = p.path[q.first + kept];
                if (!follows(q, before, now) || place(p, r, q, q.context + now).block < 0 || place(p, r, q, q.context + kept).block < 0) break;
                before = now;
            }
            const int64_t length = q.context + kept, mask = ((int64_t)1 << p.log2_block) - 1;
            p.lens_out[r] = (int32_t)min(length, (int64_t)INT32_MAX);
            const int64_t begin = (length + mask) >> p.log2_block;
            n = max(((q.kv + mask) >> p.log2_block) - begin, (int64_t)0);
            entries = p.block_table + r * p.table_width + begin;
            for (int64_t j = 0; j < n; ++j) given += named(entries[j]);
        }
        int64_t upto = given;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const int64_t x = __shfl_up_sync(~0u, upto, d);
            if (lane >= d) upto += x;
        }
        if (lane == 31) warp_sum[warp] = upto;
        __syncthreads();
        int64_t at = total + upto - given;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            if (w < warp) at += warp_sum[w];
            total += warp_sum[w];
        }
        for (int64_t j = 0; j < n && at < p.max_freed; ++j) {
            const int32_t b = entries[j];
            if (named(b)) p.freed[at++] = b;
        }
        __syncthreads();
    }
    for (int64_t j = total + tid; j < p.max_freed; j += kThreads) p.freed[j] = -1;
    if (tid == 0) *p.freed_count = total;
}

template <int FORMAT>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) keep_kernel(const __grid_constant__ QcacheKeepParams p) {
    __shared__ Place from[kTreeMaxNodes], to[kTreeMaxNodes];
    __shared__ int first_moved, first_wrong;
    after_kernels_before();
    const int r = blockIdx.x / p.chunks, chunk = blockIdx.x % p.chunks;
    if (r == p.requests) {
        count_blocks(p);
        return;
    }
    if (threadIdx.x == 0) first_moved = first_wrong = kTreeMaxNodes;
    __syncthreads();
    const Request q = request(p, r);
    const int most = min(min(max(p.kept[r], 0), q.n), kTreeMaxNodes);
    for (int i = threadIdx.x; i < most; i += kThreads) {
        const int now = p.path[q.first + i], before = i ? p.path[q.first + i - 1] : -1;
        Place f{-1, 0}, t{-1, 0};
        if (follows(q, before, now)) {
            f = place(p, r, q, q.context + now);
            t = place(p, r, q, q.context + i);
        }
        from[i] = f;
        to[i] = t;
        if (f.block < 0 || t.block < 0) atomicMin(&first_wrong, i);
        if (now != i) atomicMin(&first_moved, i);
    }
    __syncthreads();
    const int begin = first_moved, end = min(most, first_wrong);
    if (begin >= end) return;
    for (int pair = (chunk * kWarps + threadIdx.x / 32) * kPairs; pair < p.layers * p.heads; pair += p.chunks * kWarps * kPairs)
        move_rows<FORMAT>(p, pair, from, to, begin, end);
}

}  // namespace

cudaError_t launch_qcache_keep(QcacheKeepParams p, int num_sms, cudaStream_t stream) {
    // thread blocks of a request: no more than its (layer, head) can use, nor, together, than run at a time
    const int64_t most = ((int64_t)p.layers * p.heads + kWarps * kPairs - 1) / (kWarps * kPairs);
    const int64_t fair = p.requests ? ((int64_t)kBlocksPerSm * num_sms + p.requests - 1) / p.requests : 1;
    p.chunks = (int)(most < fair ? most : fair);
    const dim3 grid((unsigned)(p.requests * p.chunks + 1));
    return p.format == CM_QCACHE_E4M3 ? launch_behind(keep_kernel<CM_QCACHE_E4M3>, grid, kThreads, 0, stream, p)
                                      : launch_behind(keep_kernel<CM_QCACHE_INT8>, grid, kThreads, 0, stream, p);
}

}  // namespace cm
