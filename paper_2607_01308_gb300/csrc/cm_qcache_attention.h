// Device helpers that the attention kernels over the 8-bit cache share: the even cut of the
// work, the block table and the joining of partial results. Included by their sources only.
#pragma once

#include <cmath>

#include "cm_qcache_kernels.h"

namespace cm {
namespace {

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

__device__ __forceinline__ float pow2f(int k) { return __int_as_float((k + 127) << 23); }   // k in [-126, 127]

__device__ __forceinline__ uint32_t pack_half(float lo, float hi) {
    uint32_t w;
    asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}

// Request r's share of the work: `rows` query rows (query tokens x heads of a group) in tiles
// of ROWS, each over the kv tokens in tiles of TILE. Lengths are clamped to what the buffers
// hold, so that a wrong one reads nothing outside. Query token i is token first + i of its request.
struct RequestShape {
    int row0, first, kv;
    int rows, row_tiles, tiles;
};

template <int ROWS, int TILE>
__device__ __forceinline__ RequestShape request_shape(const QcacheAttentionParams &p, int r) {
    RequestShape s;
    const int64_t cap = min(p.table_width << p.log2_block, (int64_t)INT32_MAX - 1024);
    s.row0 = min(max(p.row_starts[r], 0), p.total_rows);
    const int q_len = min(max(p.row_starts[r + 1], s.row0), p.total_rows) - s.row0;
    const int kv = (int)min((int64_t)max(p.kv_lens[r], 0), cap);
    // A request that was cut short: the two lengths do not say which tokens its rows are. Its context length is loaded with
    // the others and selected by (without context_lens it is a length, made negative), except with two query tiles, where a
    // test keeps the issuing loop shorter: 8 prompts of 700 tokens, 8 kv heads x 4 of 128, 80 us against 84; the other
    // way round 29 requests of 3 rows take 19.7 us instead of 19.2, prompts of head_dim 256 49.3 instead of 48.2.
    s.kv = kv;
    s.first = kv - q_len;
    if constexpr (ROWS == 256) {
        const int context = p.no_context ? -1 : p.context_lens[r];
        if (context >= 0) {
            s.kv = (int)min((uint32_t)kv, (uint32_t)context + (uint32_t)q_len);
            s.first = min(context, s.kv);
        }
    } else {
        const int context = p.context_lens[r] | p.no_context;
        s.kv = context < 0 ? kv : (int)min((uint32_t)kv, (uint32_t)context + (uint32_t)q_len);
        s.first = context < 0 ? kv - q_len : min(context, s.kv);
    }
    s.rows = q_len * p.group;
    s.row_tiles = (s.rows + ROWS - 1) / ROWS;
    s.tiles = max(1, (s.kv + TILE - 1) / TILE);   // one without tokens too: its rows are written
    return s;
}

// Sums of units in 32 bits. The host refuses calls whose requests could come to 2^31 units together, so only
// row starts that do not ascend (rows that several requests claim) reach that: the sum stays there, and such a call
// does nothing, where one that wrapped around would send blocks to places outside the requests.
constexpr uint32_t kTooMany = 0x7fffffffu;
__device__ __forceinline__ uint32_t add_units(uint32_t a, uint32_t b) { return min(a + b, kTooMany); }

// A unit of work is a kv tile of one row tile and kv head. What beginning and ending a (row tile, head)
// costs besides its tiles (the query rows, the first copies, the parts' meeting) counts as SETUP units in
// front of them, or short requests would come to the same few thread blocks.

// The requests' units for one kv head as exclusive prefix sums in prefix[0 .. requests]; returns their
// total. Every thread of the block takes part.
template <int THREADS, int ROWS, int TILE, int SETUP>
__device__ __forceinline__ uint32_t plan_units(const QcacheAttentionParams &p, uint32_t *prefix, uint32_t *scan) {
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    uint32_t total = 0;
    for (int r0 = 0; r0 < p.requests; r0 += THREADS) {
        const int r = r0 + tid;
        uint32_t n = 0;
        if (r < p.requests) {
            const RequestShape s = request_shape<ROWS, TILE>(p, r);
            n = (uint32_t)s.row_tiles * (uint32_t)(s.tiles + SETUP);
        }
        uint32_t a = n;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const uint32_t x = __shfl_up_sync(~0u, a, d);
            if (lane >= d) a = add_units(a, x);
        }
        if (lane == 31) scan[warp] = a;
        __syncthreads();
        uint32_t before = total;
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) {
            if (w < warp) before = add_units(before, scan[w]);
            total = add_units(total, scan[w]);
        }
        if (r < p.requests) prefix[r] = before + a - n;
        __syncthreads();
    }
    if (tid == 0) prefix[p.requests] = total;
    __syncthreads();
    return total < kTooMany ? total : 0;
}

// Units of one thread block: an even share, but no less than a few tiles, below which joining the
// parts costs more than reading alone.
template <int SETUP>
__device__ __forceinline__ uint64_t units_per_block(uint64_t units, uint32_t blocks) {
    return max((units + blocks - 1) / blocks, (uint64_t)(SETUP + 2));
}

// A run of kv tiles [t0, t1) of one row tile of one kv head of one request.
struct AttentionSegment {
    int request, head, row_tile, t0, t1;
    int row0, first, kv, rows, tiles;
    uint64_t unit0;               // the unit of tile 0
};

// The segment at unit u, up to u_end; moves u behind it. Units lie by request, row tile, kv head, kv tile;
// a segment without tiles (t0 == t1) is the share of a setup whose tiles come later.
template <int ROWS, int TILE, int SETUP>
__device__ __forceinline__ AttentionSegment locate(const QcacheAttentionParams &p, const uint32_t *prefix, uint64_t &u,
                                                   uint64_t u_end) {
    int lo = 0, hi = p.requests;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((uint64_t)prefix[mid] * (uint32_t)p.heads <= u) lo = mid; else hi = mid;
    }
    const RequestShape s = request_shape<ROWS, TILE>(p, lo);
    AttentionSegment w;
    w.request = lo;
    w.row0 = s.row0; w.first = s.first; w.kv = s.kv; w.rows = s.rows; w.tiles = s.tiles;
    const uint64_t in = u - (uint64_t)prefix[lo] * (uint32_t)p.heads;
    const uint64_t pair = in / (uint32_t)(s.tiles + SETUP);
    const int at = (int)(in - pair * (uint32_t)(s.tiles + SETUP));
    const int to = (int)min((uint64_t)(s.tiles + SETUP), at + (u_end - u));
    w.t0 = max(0, at - SETUP);
    w.t1 = max(0, to - SETUP);
    w.row_tile = (int)(pair / (uint32_t)p.heads);
    w.head = (int)(pair - (uint64_t)w.row_tile * (uint32_t)p.heads);
    w.unit0 = u - at + SETUP;
    u += to - at;
    return w;
}

// The block of a token and its scales. block < 0: the token is at or past `kv`, or its table
// entry names no block of the pool; such tokens are not attended.
struct BlockEntry {
    int block;
    float k_scale, v_log2, v_inverse;
};

__device__ __forceinline__ BlockEntry block_entry(const QcacheAttentionParams &p, int request, int64_t head, int64_t token, int kv) {
    BlockEntry e{-1, 0.f, 0.f, 0.f};
    if (token < kv) {
        const int b = p.block_table[request * p.table_width + (token >> p.log2_block)];
        if (b >= 0 && b < p.num_blocks) {
            const int64_t at = (int64_t)b * p.scale_stride_block + head * p.scale_stride_head;
            // V scales are read within [2^-60, 2^60], where w / scale stays in fp32's range
            const float v = fminf(fmaxf(p.v_scale[at], 0x1p-60f), 0x1p60f);
            e.block = b;
            e.k_scale = p.k_scale[at];
            e.v_log2 = __log2f(v);
            e.v_inverse = __frcp_rn(v);
        }
    }
    return e;
}

__device__ __forceinline__ BlockEntry shuffle(const BlockEntry &e, int lane) {
    return {__shfl_sync(~0u, e.block, lane), __shfl_sync(~0u, e.k_scale, lane), __shfl_sync(~0u, e.v_log2, lane),
            __shfl_sync(~0u, e.v_inverse, lane)};
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}

// The natural logarithm of a row's sum at maximum m; -inf if it saw no token.
__device__ __forceinline__ float log_sum(float m, float l, float headroom) {
    return l == 0.f ? -INFINITY : (m - headroom + __log2f(l)) * 0.693147180559945309f;
}

// Elements d .. d + 3 of row n (query token n / group, head n % group) of the segment's request.
// A row that saw no token is zero.
__device__ __forceinline__ void write_row(const QcacheAttentionParams &p, const AttentionSegment &w, int n, int d, const float4 &acc,
                                          float m, float l, float headroom) {
    const int64_t row = w.row0 + n / p.group, head = (int64_t)w.head * p.group + n % p.group;
    const float f = l == 0.f ? 0.f : 1.f / l;
    const uint2 x = make_uint2(pack_bf16(acc.x * f, acc.y * f), pack_bf16(acc.z * f, acc.w * f));
    *reinterpret_cast<uint2 *>(p.out + row * p.out_stride_row + head * p.out_stride_head + d) = x;
    if (d == 0 && p.lse)
        p.lse[row * ((int64_t)p.heads * p.group) + head] = log_sum(m, l, headroom);
}

// Joins the parts of rows [0, rows) of a segment's whole range, held by thread blocks c0 .. c1 of the
// grid, in that order; row_at(c, row): the workspace row of block c's part; first: the rows' place
// among the request's. WARPS warps share the rows: lanes weigh the parts, then read them along head_dim.
template <int D, int WARPS, class At>
__device__ __forceinline__ void join_parts(const QcacheAttentionParams &p, const AttentionSegment &w, int first, int rows,
                                           uint32_t c0, uint32_t c1, float headroom, int warp, At row_at) {
    constexpr int kVecs = D >= 128 ? D / 128 : 1;   // 16-byte vectors of a lane
    constexpr int kAhead = 8;              // parts that are read together, the first before they can be weighed
    const int lane = threadIdx.x % 32, n = (int)(c1 - c0 + 1);
    for (int row = warp; row < rows; row += WARPS) {
        auto read_ml = [&](int c) {
            return c < n ? __ldcg(reinterpret_cast<const float2 *>(p.part_ml + row_at(c0 + c, row) * 2)) : make_float2(-INFINITY, 0.f);
        };
        float4 x[kAhead][kVecs], acc[kVecs];
        auto read = [&](int c) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k)
#pragma unroll
                for (int v = 0; v < kVecs; ++v)
                    x[k][v] = (D < 128 && lane >= D / 4) || c + k >= n
                                  ? make_float4(0.f, 0.f, 0.f, 0.f)
                                  : __ldcg(reinterpret_cast<const float4 *>(p.part_o + row_at(c0 + c + k, row) * D) + lane + 32 * v);
        };
        float2 ml = read_ml(lane);
        read(0);
        float m = ml.x, l = 0.f;
        for (int c = 32 + lane; c < n; c += 32) m = fmaxf(m, read_ml(c).x);
#pragma unroll
        for (int d = 16; d; d /= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
#pragma unroll
        for (int v = 0; v < kVecs; ++v) acc[v] = make_float4(0.f, 0.f, 0.f, 0.f);
        float f = 0.f;
#pragma unroll 1
        for (int c = 0; c < n; c += kAhead) {
            if (c > 0) read(c);
            if (c % 32 == 0) {                      // the factors of the next 32 parts, one a lane
                if (c > 0) ml = read_ml(c + lane);
                f = ml.x == m ? 1.f : exp2_fast(ml.x - m);
                float y = ml.y * f;
#pragma unroll
                for (int d = 16; d; d /= 2) y += __shfl_xor_sync(~0u, y, d);
                l += y;
            }
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                const float g = __shfl_sync(~0u, f, (c + k) % 32);
#pragma unroll
                for (int v = 0; v < kVecs; ++v) {
                    acc[v].x = fmaf(x[k][v].x, g, acc[v].x); acc[v].y = fmaf(x[k][v].y, g, acc[v].y);
                    acc[v].z = fmaf(x[k][v].z, g, acc[v].z); acc[v].w = fmaf(x[k][v].w, g, acc[v].w);
                }
            }
        }
#pragma unroll
        for (int v = 0; v < kVecs; ++v)
            if (D >= 128 || lane < D / 4) write_row(p, w, first + row, (lane + 32 * v) * 4, acc[v], m, l, headroom);
    }
}

}  // namespace
}  // namespace cm
