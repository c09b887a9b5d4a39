// New K and V rows into the 8-bit paged cache.
//
// For each (block, layer, head) that gets rows, and for K and V on their own:
//   needed  = the smallest 2^k, k in [-60, 60], with max |x| <= top * 2^k over the finite new
//             values (top = 448 for e4m3, 127 for int8)
//   scale'  = needed if the rows begin at the block's first token, else max(scale, needed)
//   code    = x / scale' to nearest even, clamped to [-top, top]; NaN becomes 0
//   the codes before the first new token are rounded again by scale / scale' where it grew
// Powers of two make every division exact: a code is rounded once, a growing scale costs e4m3
// codes nothing until they become subnormal, and the result does not depend on the order of
// arithmetic. The price is up to one bit of int8's range.
//
// Rows of one block are consecutive in the call (slots ascend by one), so the first of them
// (the leader: its slot does not continue the row before it inside one block) stands for the
// whole run, and one team of warps reads the run, reduces its magnitude, writes the scale and
// the codes. Bound by HBM: 2 bytes in and 1 out per element. A run of up to 2048 elements stays
// in registers between the two steps, so that it is read once.
#include "cm_qcache_kernels.h"

#include "cm_qcache_codes.h"

namespace cm {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kVecs = 8;                      // 16-byte vectors of a lane held in registers
constexpr int kMinExp = -60, kMaxExp = 60;

__device__ __forceinline__ float pow2(int k) { return __int_as_float((k + 127) << 23); }

// Larger of m and the magnitudes (bf16 bits without sign) in w, for each half.
__device__ __forceinline__ uint32_t max_abs(uint32_t m, uint32_t w) { return __vmaxu2(m, w & 0x7fff7fffu); }

__device__ __forceinline__ uint32_t finite_only(uint32_t w) {
    const uint32_t a = w & 0x7fff7fffu;
    return ((a & 0x7f80u) == 0x7f80u ? 0u : a & 0xffffu) | ((a & 0x7f800000u) == 0x7f800000u ? 0u : a & 0xffff0000u);
}

// k of the smallest 2^k that brings a magnitude (bf16 bits) within the format's top, in range.
template <int FORMAT>
__device__ __forceinline__ int scale_exponent(uint32_t bits) {
    const int e = (int)(bits >> 7) - 127;     // a subnormal is far below the range
    const uint32_t m = bits & 0x7f;           // top is 1.75 * 2^8, or 1.984375 * 2^6 (m = 0x7e)
    const int k = FORMAT == CM_QCACHE_E4M3 ? e - 8 + (m > 0x60) : e - 6 + (m > 0x7e);
    return bits == 0 ? kMinExp : min(max(k, kMinExp), kMaxExp);
}

// Four values (already divided by the scale) to codes. CLAMP: values may be out of range or NaN.
template <int FORMAT, bool CLAMP>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d) {
    if constexpr (CLAMP) {
        a = a == a ? a : 0.f; b = b == b ? b : 0.f; c = c == c ? c : 0.f; d = d == d ? d : 0.f;
    }
    if constexpr (FORMAT == CM_QCACHE_E4M3) {
        uint32_t w;
        asm("{\n.reg .b16 lo, hi;\ncvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\ncvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n"
            "mov.b32 %0, {lo, hi};\n}" : "=r"(w) : "f"(a), "f"(b), "f"(c), "f"(d));
        return w;
    } else {
        if constexpr (CLAMP) {
            a = fminf(fmaxf(a, -127.f), 127.f); b = fminf(fmaxf(b, -127.f), 127.f);
            c = fminf(fmaxf(c, -127.f), 127.f); d = fminf(fmaxf(d, -127.f), 127.f);
        }
        // 1.5 * 2^23 + x leaves x, rounded to nearest even, in the low byte
        const uint32_t ua = __float_as_uint(a + 12582912.f), ub = __float_as_uint(b + 12582912.f);
        const uint32_t uc = __float_as_uint(c + 12582912.f), ud = __float_as_uint(d + 12582912.f);
        return prmt(prmt(ua, ub, 0x0040), prmt(uc, ud, 0x0040), 0x5410);
    }
}

__device__ __forceinline__ float half_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float half_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

template <int FORMAT, bool CLAMP>
__device__ __forceinline__ uint2 row_codes(const uint4 &x, float inv) {
    uint2 r;
    r.x = to_codes<FORMAT, CLAMP>(half_lo(x.x) * inv, half_hi(x.x) * inv, half_lo(x.y) * inv, half_hi(x.y) * inv);
    r.y = to_codes<FORMAT, CLAMP>(half_lo(x.z) * inv, half_hi(x.z) * inv, half_lo(x.w) * inv, half_hi(x.w) * inv);
    return r;
}

// Codes times a power of two <= 1, rounded again.
template <int FORMAT>
__device__ __forceinline__ uint32_t shrink(uint32_t w, float ratio) {
    float x[4];
    if constexpr (FORMAT == CM_QCACHE_E4M3) {
        uint32_t lo, hi;
        codes_to_half<FORMAT>(w, lo, hi);
        asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}" : "=f"(x[0]), "=f"(x[1]) : "r"(lo));
        asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}" : "=f"(x[2]), "=f"(x[3]) : "r"(hi));
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = (float)(int8_t)(w >> (8 * i));
    }
    return to_codes<FORMAT, true>(x[0] * ratio, x[1] * ratio, x[2] * ratio, x[3] * ratio);
}

// One (run, layer, head) of K or V by TEAM warps; `t` is the thread in the team. `red`: a word
// per warp of shared memory. All threads of the block take part in the same number of calls
// when TEAM > 1.
template <int FORMAT, int TEAM>
__device__ __forceinline__ void write_run(const QcacheAppendParams &p, int kv, int64_t layer, int64_t head, int64_t row,
                                          int64_t slot, int n, int t, uint32_t *red) {
    constexpr int kTeam = TEAM * 32;
    const int log2_vecs = 31 - __clz(p.head_dim) - 3;          // 16-byte vectors to a row: a power of two
    const int total = n << log2_vecs;                          // of the run
    const uint16_t *src = p.rows[kv] + layer * p.row_stride_layer + head * p.row_stride_head + row * p.row_stride_row;
    const int64_t block = slot >> p.log2_block;
    const int begin = (int)(slot & (((int64_t)1 << p.log2_block) - 1));
    uint8_t *codes = p.codes[kv] + layer * p.stride_layer + head * p.stride_head + block * p.stride_block;
    float *scale = p.scales[kv] + layer * p.scale_stride_layer + head * p.scale_stride_head + block * p.scale_stride_block;
    const float old = begin ? *scale : 0.f;
    const int vec_mask = (1 << log2_vecs) - 1;
    auto load = [&](int i) {
        return __ldcs(reinterpret_cast<const uint4 *>(src + (int64_t)(i >> log2_vecs) * p.row_stride_row + (i & vec_mask) * 8));
    };
    uint4 x[kVecs];
    uint32_t m = 0;
    const int steps = (total + kVecs * kTeam - 1) / (kVecs * kTeam);
    // the last step's vectors are still in registers when they are written
    for (int s = 0; s < steps; ++s) {
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = (s * kVecs + j) * kTeam + t;
            x[j] = i < total ? load(i) : make_uint4(0, 0, 0, 0);
        }
#pragma unroll
        for (int j = 0; j < kVecs; ++j) m = max_abs(max_abs(max_abs(max_abs(m, x[j].x), x[j].y), x[j].z), x[j].w);
    }
    m = max(m & 0xffffu, m >> 16);
    auto reduce = [&](uint32_t v) {
        v = __reduce_max_sync(~0u, v);
        if constexpr (TEAM > 1) {
            if (threadIdx.x % 32 == 0) red[threadIdx.x / 32] = v;
            __syncthreads();
#pragma unroll
            for (int w = 0; w < TEAM; ++w) v = max(v, red[w]);
            __syncthreads();
        }
        return v;
    };
    m = reduce(m);
    bool clamp = false;
    if (m >= 0x7f80u) {                        // an infinity or a NaN: once more without them
        clamp = true;
        m = 0;
        for (int i = t; i < total; i += kTeam) {
            const uint4 v = load(i);
            m = __vmaxu2(m, __vmaxu2(__vmaxu2(finite_only(v.x), finite_only(v.y)), __vmaxu2(finite_only(v.z), finite_only(v.w))));
        }
        m = reduce(max(m & 0xffffu, m >> 16));
    }
    const int k = scale_exponent<FORMAT>(m);
    clamp |= k == kMaxExp;
    const float needed = pow2(k), now = begin ? fmaxf(old, needed) : needed;
    // 1 / now is exact for a power of two; a scale that the caller wrote need not be one
    const float inv = now == needed ? pow2(-k) : __frcp_rn(now);
    for (int s = steps - 1; s >= 0; --s) {
        if (s != steps - 1) {
#pragma unroll
            for (int j = 0; j < kVecs; ++j) {
                const int i = (s * kVecs + j) * kTeam + t;
                if (i < total) x[j] = load(i);
            }
        }
#pragma unroll
        for (int j = 0; j < kVecs; ++j) {
            const int i = (s * kVecs + j) * kTeam + t;
            if (i >= total) break;
            const uint2 c = clamp ? row_codes<FORMAT, true>(x[j], inv) : row_codes<FORMAT, false>(x[j], inv);
            *reinterpret_cast<uint2 *>(codes + (int64_t)(begin + (i >> log2_vecs)) * p.stride_token + (i & vec_mask) * 8) = c;
        }
    }
    if (begin && now > old) {                  // the tokens before the run, rounded to the larger scale
        const float ratio = old * inv;
        for (int i = t; i < begin << log2_vecs; i += kTeam) {
            uint2 *at = reinterpret_cast<uint2 *>(codes + (int64_t)(i >> log2_vecs) * p.stride_token + (i & vec_mask) * 8);
            uint2 c = *at;
            c.x = shrink<FORMAT>(c.x, ratio);
            c.y = shrink<FORMAT>(c.y, ratio);
            *at = c;
        }
    }
    if (TEAM > 1) __syncthreads(); else __syncwarp();   // every thread has read the old scale
    if (t == 0 && now != old) *scale = now;
}

// Grid: windows of rows x groups of heads x layers. TEAM = 1: a warp per run, head and K or V;
// TEAM = 4: the block together.
template <int FORMAT, int TEAM>
__global__ void __launch_bounds__(kThreads) append_kernel(const __grid_constant__ QcacheAppendParams p) {
    __shared__ uint32_t red[kWarps];
    constexpr int kHeads = TEAM == 1 ? 2 : 1;  // per thread block
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    const int64_t layer = blockIdx.z, row0 = (int64_t)blockIdx.x * p.window;
    const int64_t row1 = min(row0 + p.window, p.num_rows);
    const int64_t mask = ((int64_t)1 << p.log2_block) - 1;
    const int heads = min(kHeads, p.heads - (int)blockIdx.y * kHeads);
    int task = 0;
    for (int64_t r0 = row0; r0 < row1; r0 += 32) {
        const int64_t r = r0 + lane;
        const int64_t slot = r < row1 ? __ldg(p.slots + r) : -1;
        const int64_t before = r < row1 && r > 0 ? __ldg(p.slots + r - 1) : -1;
        const bool valid = slot >= 0 && slot < p.num_slots;
        unsigned leaders = __ballot_sync(~0u, valid && (before < 0 || slot != before + 1 || (slot & mask) == 0));
        while (leaders) {
            const int l = __ffs(leaders) - 1;
            leaders &= leaders - 1;
            const int64_t first = __shfl_sync(~0u, slot, l), row = r0 + l;
            // the run's length: rows that continue it inside its block
            const int most = (int)min(mask + 1 - (first & mask), p.num_rows - row);
            int n = 0;
            while (n < most) {
                const bool goes_on = n + lane < most && __ldg(p.slots + row + n + lane) == first + n + lane;
                const unsigned run = __ballot_sync(~0u, goes_on);
                const int more = run == ~0u ? 32 : __ffs(~run) - 1;
                n += more;
                if (more < 32) break;
            }
            for (int i = 0; i < 2 * heads; ++i, ++task)
                if (TEAM > 1 || task % kWarps == warp)
                    write_run<FORMAT, TEAM>(p, i & 1, layer, (int64_t)blockIdx.y * kHeads + (i >> 1), row, first, n,
                                            TEAM > 1 ? (int)threadIdx.x : lane, red);
        }
    }
}

}  // namespace

cudaError_t launch_qcache_append(QcacheAppendParams p, int num_sms, cudaStream_t stream) {
    if (p.num_rows == 0) return cudaSuccess;
    // A warp holds 2048 elements in registers; blocks of more go to four warps together.
    const bool team = ((int64_t)p.head_dim << p.log2_block) > 2048 * 2;
    const int per = team ? 1 : 2;
    const int head_groups = (p.heads + per - 1) / per;
    // Rows per thread block: one while that leaves every SM less than about 16 thread blocks
    // (single tokens: each row is a run of its own), up to a block of tokens, which is one run
    // of a prompt.
    const int64_t blocks_of_one = p.num_rows * head_groups * p.layers;
    int window = 1;
    while (window < 32 && window < (1 << p.log2_block) && blocks_of_one / window > 16ll * num_sms) window *= 2;
    p.window = window;
    const dim3 grid((unsigned)((p.num_rows + window - 1) / window), (unsigned)head_groups, (unsigned)p.layers);
    if (p.format == CM_QCACHE_E4M3) {
        if (team) append_kernel<CM_QCACHE_E4M3, 4><<<grid, kThreads, 0, stream>>>(p);
        else append_kernel<CM_QCACHE_E4M3, 1><<<grid, kThreads, 0, stream>>>(p);
    } else {
        if (team) append_kernel<CM_QCACHE_INT8, 4><<<grid, kThreads, 0, stream>>>(p);
        else append_kernel<CM_QCACHE_INT8, 1><<<grid, kThreads, 0, stream>>>(p);
    }
    return cudaGetLastError();
}

}  // namespace cm
