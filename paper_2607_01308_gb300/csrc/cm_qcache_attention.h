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
// hold, so that a wrong one reads nothing outside.
struct RequestShape {
    int row0, q_len, kv;
    int rows, row_tiles, tiles;
};

template <int ROWS, int TILE>
__device__ __forceinline__ RequestShape request_shape(const QcacheAttentionParams &p, int r) {
    RequestShape s;
    const int64_t cap = min(p.table_width << p.log2_block, (int64_t)INT32_MAX - 1024);
    s.row0 = min(max(__ldg(p.row_starts + r), 0), p.total_rows);
    s.q_len = min(max(__ldg(p.row_starts + r + 1), s.row0), p.total_rows) - s.row0;
    s.kv = (int)min((int64_t)max(__ldg(p.kv_lens + r), 0), cap);
    s.rows = s.q_len * p.group;
    s.row_tiles = (s.rows + ROWS - 1) / ROWS;
    s.tiles = max(1, (s.kv + TILE - 1) / TILE);   // one without tokens too: its rows are written
    return s;
}

// The requests' units (row tiles x kv tiles) for one kv head as exclusive prefix sums in
// prefix[0 .. requests]; returns their total. Every thread of the block takes part.
template <int THREADS, int ROWS, int TILE>
__device__ __forceinline__ uint32_t plan_units(const QcacheAttentionParams &p, uint32_t *prefix, uint32_t *scan) {
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    uint32_t total = 0;
    for (int r0 = 0; r0 < p.requests; r0 += THREADS) {
        const int r = r0 + tid;
        uint32_t n = 0;
        if (r < p.requests) {
            const RequestShape s = request_shape<ROWS, TILE>(p, r);
            n = (uint32_t)s.row_tiles * (uint32_t)s.tiles;
        }
        uint32_t a = n;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const uint32_t x = __shfl_up_sync(~0u, a, d);
            if (lane >= d) a += x;
        }
        if (lane == 31) scan[warp] = a;
        __syncthreads();
        uint32_t before = total;
#pragma unroll
        for (int w = 0; w < THREADS / 32; ++w) {
            if (w < warp) before += scan[w];
            total += scan[w];
        }
        if (r < p.requests) prefix[r] = before + a - n;
        __syncthreads();
    }
    if (tid == 0) prefix[p.requests] = total;
    __syncthreads();
    return total;
}

// Units of one thread block: an even share, but no less than a few, below which joining the
// parts costs more than reading alone.
__device__ __forceinline__ uint64_t units_per_block(uint64_t units, uint32_t blocks) {
    return max((units + blocks - 1) / blocks, (uint64_t)2);
}

// A run of kv tiles [t0, t1) of one row tile of one kv head of one request.
struct AttentionSegment {
    int request, head, row_tile, t0, t1;
    int row0, q_len, kv, rows, tiles;
    uint64_t unit0;               // the unit of tile 0
};

// Units lie by request, row tile, kv head, kv tile.
template <int ROWS, int TILE>
__device__ __forceinline__ AttentionSegment locate(const QcacheAttentionParams &p, const uint32_t *prefix, uint64_t u,
                                                   uint64_t u_end) {
    int lo = 0, hi = p.requests;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if ((uint64_t)prefix[mid] * (uint32_t)p.heads <= u) lo = mid; else hi = mid;
    }
    const RequestShape s = request_shape<ROWS, TILE>(p, lo);
    AttentionSegment w;
    w.request = lo;
    w.row0 = s.row0; w.q_len = s.q_len; w.kv = s.kv; w.rows = s.rows; w.tiles = s.tiles;
    const uint64_t in = u - (uint64_t)prefix[lo] * (uint32_t)p.heads;
    const uint64_t pair = in / (uint32_t)s.tiles;
    w.t0 = (int)(in - pair * (uint32_t)s.tiles);
    w.t1 = (int)min((uint64_t)s.tiles, w.t0 + (u_end - u));
    w.row_tile = (int)(pair / (uint32_t)p.heads);
    w.head = (int)(pair - (uint64_t)w.row_tile * (uint32_t)p.heads);
    w.unit0 = u - w.t0;
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
        const int b = __ldg(p.block_table + request * p.table_width + (token >> p.log2_block));
        if (b >= 0 && b < p.num_blocks) {
            const int64_t at = (int64_t)b * p.scale_stride_block + head * p.scale_stride_head;
            // V scales are read within [2^-60, 2^60], where w / scale stays in fp32's range
            const float v = fminf(fmaxf(__ldg(p.v_scale + at), 0x1p-60f), 0x1p60f);
            e.block = b;
            e.k_scale = __ldg(p.k_scale + at);
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

// Adds a part (unnormalised output x, sum l_x, maximum m_x) to one at maximum m >= m_x.
__device__ __forceinline__ void join(float4 &acc, float &l, const float4 &x, float l_x, float m_x, float m) {
    const float f = m_x == m ? 1.f : exp2_fast(m_x - m);
    acc.x = fmaf(x.x, f, acc.x); acc.y = fmaf(x.y, f, acc.y);
    acc.z = fmaf(x.z, f, acc.z); acc.w = fmaf(x.w, f, acc.w);
    l = fmaf(l_x, f, l);
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}

// Elements d .. d + 3 of row n (query token n / group, head n % group) of the segment's request.
// A row that saw no token is zero, its logarithm -inf.
__device__ __forceinline__ void write_row(const QcacheAttentionParams &p, const AttentionSegment &w, int n, int d, const float4 &acc,
                                          float m, float l, float headroom) {
    const int64_t row = w.row0 + n / p.group, head = (int64_t)w.head * p.group + n % p.group;
    const float f = l == 0.f ? 0.f : 1.f / l;
    const uint2 x = make_uint2(pack_bf16(acc.x * f, acc.y * f), pack_bf16(acc.z * f, acc.w * f));
    *reinterpret_cast<uint2 *>(p.out + row * p.out_stride_row + head * p.out_stride_head + d) = x;
    if (d == 0 && p.lse)
        p.lse[row * ((int64_t)p.heads * p.group) + head] =
            l == 0.f ? -INFINITY : (m - headroom + __log2f(l)) * 0.693147180559945309f;
}

// The parts of row n of a segment's whole range, held by thread blocks c0 .. c1, in that order;
// at(c): the workspace row of block c's part.
template <int D, class At>
__device__ __forceinline__ void join_parts(const QcacheAttentionParams &p, const AttentionSegment &w, int n, int d, uint32_t c0,
                                           uint32_t c1, float headroom, At at) {
    float m = -INFINITY;
#pragma unroll 8
    for (uint32_t c = c0; c <= c1; ++c) m = fmaxf(m, __ldcg(p.part_ml + at(c) * 2));
    float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
    float l = 0.f;
#pragma unroll 8
    for (uint32_t c = c0; c <= c1; ++c) {
        const float2 ml = __ldcg(reinterpret_cast<const float2 *>(p.part_ml + at(c) * 2));
        join(acc, l, __ldcg(reinterpret_cast<const float4 *>(p.part_o + at(c) * D + d)), ml.y, ml.x, m);
    }
    write_row(p, w, n, d, acc, m, l, headroom);
}

}  // namespace
}  // namespace cm
