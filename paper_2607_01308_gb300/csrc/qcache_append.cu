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
// Rows of one block are consecutive in the call (slots ascend by one), so the first of them (its
// slot does not continue the row before it inside one block) stands for the whole run. A thread
// block finds the runs that begin in its window of rows; then a warp takes a run of one head, K or
// V: it reads it into registers, reduces the magnitude, writes the scale and the codes. A run that fits the registers
// (2,048 elements of a warp, 8,192 of four, 16,384 of eight) is read once; of a longer one all but the last
// part is read a second time for its codes (blocks of 128 x 128 and 128 x 256: 1.5 times in all, 256 x 256: 1.75).
// Bound by HBM: 2 bytes in and 1 out per element. Measured: 36 layers of 8 heads of 128, 5,208 tokens in blocks of
// 16 (1,153 MB): 175 us, 6.6 TB/s; 5,000 tokens in blocks of 64 184 us (6.0 TB/s), of 128 217 us (5.1), where a thread
// block's warps write K and V one after the other; 10,300 ragged int8 rows of 12 heads of 64 (47 MB, 2.1 waves of thread
// blocks): 13.5 us; one token of 48 requests: 2.5 us, a launch's latency.
#include "cm_qcache_kernels.h"

#include "cm_qcache_codes.h"

namespace cm {
namespace {

constexpr int kHeld = 4;                      // of codes that are rounded again
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

// Four values times 1 / scale to codes. CLAMP: they may be out of range or NaN.
template <int FORMAT, bool CLAMP>
__device__ __forceinline__ uint32_t to_codes(float a, float b, float c, float d, float inv) {
    constexpr float kRound = 12582912.f;       // 1.5 * 2^23 + x leaves x, rounded to nearest even, in the low byte
    if constexpr (FORMAT == CM_QCACHE_E4M3 || CLAMP) {
        a *= inv; b *= inv; c *= inv; d *= inv;
    }
    if constexpr (CLAMP) {
        a = a == a ? a : 0.f; b = b == b ? b : 0.f; c = c == c ? c : 0.f; d = d == d ? d : 0.f;
    }
    if constexpr (FORMAT == CM_QCACHE_E4M3) {  // the conversion clamps
        uint32_t w;
        asm("{\n.reg .b16 lo, hi;\ncvt.rn.satfinite.e4m3x2.f32 lo, %2, %1;\ncvt.rn.satfinite.e4m3x2.f32 hi, %4, %3;\n"
            "mov.b32 %0, {lo, hi};\n}" : "=r"(w) : "f"(a), "f"(b), "f"(c), "f"(d));
        return w;
    } else {
        if constexpr (CLAMP) {
            a = fminf(fmaxf(a, -127.f), 127.f) + kRound; b = fminf(fmaxf(b, -127.f), 127.f) + kRound;
            c = fminf(fmaxf(c, -127.f), 127.f) + kRound; d = fminf(fmaxf(d, -127.f), 127.f) + kRound;
        } else {                               // the product is exact, or its rounding is this one
            a = __fmaf_rn(a, inv, kRound); b = __fmaf_rn(b, inv, kRound);
            c = __fmaf_rn(c, inv, kRound); d = __fmaf_rn(d, inv, kRound);
        }
        return prmt(prmt(__float_as_uint(a), __float_as_uint(b), 0x0040),
                    prmt(__float_as_uint(c), __float_as_uint(d), 0x0040), 0x5410);
    }
}

__device__ __forceinline__ float half_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float half_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }

template <int FORMAT, bool CLAMP>
__device__ __forceinline__ uint2 row_codes(const uint4 &x, float inv) {
    uint2 r;
    r.x = to_codes<FORMAT, CLAMP>(half_lo(x.x), half_hi(x.x), half_lo(x.y), half_hi(x.y), inv);
    r.y = to_codes<FORMAT, CLAMP>(half_lo(x.z), half_hi(x.z), half_lo(x.w), half_hi(x.w), inv);
    return r;
}

// Codes times a ratio below 1 (a power of two, unless a caller wrote another scale), rounded again.
template <int FORMAT>
__device__ __forceinline__ uint32_t shrink(uint32_t w, float ratio) {
    float x[4];
    if constexpr (FORMAT == CM_QCACHE_E4M3) {
        uint32_t lo, hi;
        codes_to_half<FORMAT>(w, lo, hi);
        asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}" : "=f"(x[0]), "=f"(x[1]) : "r"(lo));
        asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.f32.f16 %0, a;\ncvt.f32.f16 %1, b;\n}" : "=f"(x[2]), "=f"(x[3]) : "r"(hi));
    } else {
        w ^= 0x80808080u;                      // code + 128 as the low byte of 2^23 + code + 128
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(prmt(w, 0x4b000000u, 0x7440 + i)) - 8388736.f;
    }
    // a code that a caller wrote may be NaN, and none is out of range
    return to_codes<FORMAT, FORMAT == CM_QCACHE_E4M3>(x[0], x[1], x[2], x[3], ratio);
}

// One (run, layer, head) of K or V by TEAM warps; `t` is the thread in the team. `red`: a word
// per warp of shared memory. All threads of the block take part in the same number of calls
// when TEAM > 1.
template <int FORMAT, int TEAM, int VECS>
__device__ __forceinline__ void write_run(const QcacheAppendParams &p, int kv, int64_t layer, int64_t head, int64_t row,
                                          int64_t slot, int n, int t, uint32_t *red) {
    constexpr int kTeam = TEAM * 32;
    // A row has 2^log2_vecs vectors of 16 bytes, no more than the team has threads: a thread keeps
    // its column and takes every `step`-th row.
    const int log2_vecs = 31 - __clz(p.head_dim) - 3, vec_mask = (1 << log2_vecs) - 1;
    const int step = kTeam >> log2_vecs, r0 = t >> log2_vecs, column = t & vec_mask;
    const uint16_t *src = p.rows[kv] + layer * p.row_stride_layer + head * p.row_stride_head + (row + r0) * p.row_stride_row + column * 8;
    const int64_t block = slot >> p.log2_block;
    const int begin = (int)(slot & (((int64_t)1 << p.log2_block) - 1));
    uint8_t *codes = p.codes[kv] + layer * p.stride_layer + head * p.stride_head + block * p.stride_block;
    float *scale = p.scales[kv] + layer * p.scale_stride_layer + head * p.scale_stride_head + block * p.scale_stride_block;
    const int64_t src_step = step * p.row_stride_row;
    uint4 x[VECS];
    uint32_t m = 0;
    const int held = VECS * step;             // rows of the run that the team holds at a time
    auto load = [&](int s) {                   // rows s * held + r0 + {0, step, 2 step, ...}
        const uint16_t *at = src + s * VECS * src_step;
        const int left = n - s * held - r0;
#pragma unroll
        for (int j = 0; j < VECS; ++j) {
            x[j] = make_uint4(0, 0, 0, 0);
            if (j * step < left) x[j] = __ldcs(reinterpret_cast<const uint4 *>(at));
            at += src_step;
        }
    };
    const int steps = (n + held - 1) / held;
    const float old = begin ? *scale : 0.f;
    // the last step's vectors are still in registers when they are written
#pragma unroll 1
    for (int s = 0; s < steps; ++s) {
        load(s);
#pragma unroll
        for (int j = 0; j < VECS; ++j) m = max_abs(max_abs(max_abs(max_abs(m, x[j].x), x[j].y), x[j].z), x[j].w);
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
    const bool not_finite = m >= 0x7f80u;
    if (not_finite) {                          // an infinity or a NaN: once more without them
        m = 0;
#pragma unroll 1
        for (int r = 0; r < n - r0; r += step) {
            const uint4 v = *reinterpret_cast<const uint4 *>(src + r * p.row_stride_row);
            m = __vmaxu2(m, __vmaxu2(__vmaxu2(finite_only(v.x), finite_only(v.y)), __vmaxu2(finite_only(v.z), finite_only(v.w))));
        }
        m = reduce(max(m & 0xffffu, m >> 16));
    }
    const int k = scale_exponent<FORMAT>(m);
    const float needed = pow2(k), now = begin ? fmaxf(old, needed) : needed;
    // 1 / now is exact for a power of two; a scale that the caller wrote need not be one
    const float inv = now == needed ? pow2(-k) : __frcp_rn(now);
    uint8_t *to = codes + (int64_t)(begin + r0) * p.stride_token + column * 8;
    const int64_t to_step = step * p.stride_token;
    if (not_finite || k == kMaxExp) {
#pragma unroll 1
        for (int r = 0; r < n - r0; r += step)
            *reinterpret_cast<uint2 *>(to + r * p.stride_token) =
                row_codes<FORMAT, true>(*reinterpret_cast<const uint4 *>(src + r * p.row_stride_row), inv);
    } else {
#pragma unroll 1
        for (int s = steps - 1; s >= 0; --s) {
            if (s != steps - 1) load(s);
            const int left = n - s * held - r0;
            uint8_t *at = to + s * VECS * to_step;
#pragma unroll
            for (int j = 0; j < VECS; ++j) {
                if (j * step >= left) break;
                *reinterpret_cast<uint2 *>(at) = row_codes<FORMAT, false>(x[j], inv);
                at += to_step;
            }
        }
    }
    if (begin && now > old) {                  // the tokens before the run, rounded to the larger scale
        const float ratio = old * inv;
        const int rows = 2 * step;             // half as many vectors of codes to a row
        const int h0 = t >> (log2_vecs - 1);
        uint8_t *base = codes + (t & (vec_mask >> 1)) * 16;
#pragma unroll 1
        for (int r = h0; r < begin; r += kHeld * rows) {       // loads together: one latency for 2 KB of a warp
            uint8_t *at = base + r * p.stride_token;
            uint4 c[kHeld];
#pragma unroll
            for (int j = 0; j < kHeld; ++j)
                if (r + j * rows < begin) c[j] = *reinterpret_cast<const uint4 *>(at + j * rows * p.stride_token);
#pragma unroll
            for (int j = 0; j < kHeld; ++j) {
                if (r + j * rows >= begin) break;
                c[j] = make_uint4(shrink<FORMAT>(c[j].x, ratio), shrink<FORMAT>(c[j].y, ratio),
                                  shrink<FORMAT>(c[j].z, ratio), shrink<FORMAT>(c[j].w, ratio));
                *reinterpret_cast<uint4 *>(at + j * rows * p.stride_token) = c[j];
            }
        }
    }
    if (TEAM > 1) __syncthreads(); else __syncwarp();   // every thread has read the old scale
    if (t == 0 && now != old) *scale = now;
}

// A run: rows [row, row + n) of the call go into slots [slot, slot + n) of one block.
struct Run {
    int64_t slot;
    int32_t row, n;
};

// The runs that begin in rows [row0, row1), row1 <= row0 + 32, found by one warp; their number.
__device__ __forceinline__ int find_runs(const QcacheAppendParams &p, int64_t row0, int64_t row1, Run *runs) {
    const int lane = threadIdx.x % 32;
    const int64_t r = row0 + lane, mask = ((int64_t)1 << p.log2_block) - 1;
    const int64_t slot = r < p.num_rows ? p.slots[r] : -1;
    const int64_t after = r + 32 < p.num_rows ? p.slots[r + 32] : -1;   // where the runs may go on
    int64_t before = __shfl_up_sync(~0u, slot, 1), after_before = __shfl_up_sync(~0u, after, 1);
    const int64_t last = __shfl_sync(~0u, slot, 31);
    if (lane == 0) {
        before = r > 0 ? p.slots[r - 1] : -1;
        after_before = last;
    }
    auto goes_on = [&](int64_t x, int64_t b) { return b >= 0 && x == b + 1 && (x & mask) != 0; };
    const bool leader = r < row1 && slot >= 0 && slot < p.num_slots && !goes_on(slot, before);
    const uint64_t on = __ballot_sync(~0u, goes_on(slot, before)) | (uint64_t)__ballot_sync(~0u, goes_on(after, after_before)) << 32;
    int n = __ffsll(~(on >> (lane + 1)));
    // a run that reaches the last of the 64 rows (blocks of more than 32) is followed further
    const int most = (int)min(mask + 1 - (slot & mask), p.num_rows - r);
    unsigned open = __ballot_sync(~0u, leader && n == 64 - lane && n < most);
    while (open) {
        const int l = __ffs(open) - 1;
        open &= open - 1;
        const int64_t first = __shfl_sync(~0u, slot, l);
        const int limit = __shfl_sync(~0u, most, l);
        int m = 64 - l;
        unsigned more = ~0u;
        while (more == ~0u && m < limit) {
            more = __ballot_sync(~0u, m + lane < limit && p.slots[row0 + l + m + lane] == first + m + lane);
            m += more == ~0u ? 32 : __ffs(~more) - 1;
        }
        if (lane == l) n = m;
    }
    const unsigned leaders = __ballot_sync(~0u, leader);
    if (leader) runs[__popc(leaders & ((1u << lane) - 1))] = {slot, (int32_t)r, n};
    return __popc(leaders);
}

// Grid: windows of rows x groups of heads x layers. A warp per run, head and K or V, or, TEAM > 1 and the
// run too long for one, the block's TEAM warps together.
template <int TEAM>
constexpr int kBlockWarps = TEAM == 1 ? 4 : TEAM;

template <int FORMAT, int TEAM, int VECS>
__global__ void __launch_bounds__(kBlockWarps<TEAM> * 32, (VECS < 8 ? 32 : 24) / kBlockWarps<TEAM>) append_kernel(const __grid_constant__ QcacheAppendParams p) {
    __shared__ uint32_t red[TEAM];
    __shared__ Run runs[32];
    __shared__ int num_runs;
    constexpr int kHeads = TEAM == 1 ? 2 : 1;  // per thread block
    after_kernels_before();
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
    if (warp == 0) {
        const int64_t row0 = (int64_t)blockIdx.x * p.window;
        const int n = find_runs(p, row0, min(row0 + p.window, p.num_rows), runs);
        if (lane == 0) num_runs = n;
    }
    __syncthreads();
    const int head0 = blockIdx.y * kHeads, per_run = 2 * min(kHeads, p.heads - head0);
    const int tasks = num_runs * per_run;
    // a run that one warp holds in registers is written by one, tasks side by side
    constexpr int kAlone = TEAM == 1 ? VECS : 2;
    auto small = [&](const Run &r) { return TEAM == 1 || (p.head_dim <= 256 && r.n * p.head_dim <= 256 * kAlone); };
#pragma unroll 1
    for (int task = warp; task < tasks; task += kBlockWarps<TEAM>) {
        const int i = task % per_run;
        const Run r = runs[task / per_run];
        if (small(r)) write_run<FORMAT, 1, kAlone>(p, i & 1, blockIdx.z, head0 + (i >> 1), r.row, r.slot, r.n, lane, nullptr);
    }
    if constexpr (TEAM > 1) {
#pragma unroll 1
        for (int task = 0; task < tasks; ++task) {
            const int i = task % per_run;
            const Run r = runs[task / per_run];
            if (!small(r)) write_run<FORMAT, TEAM, VECS>(p, i & 1, blockIdx.z, head0 + (i >> 1), r.row, r.slot, r.n, threadIdx.x, red);
        }
    }
}

template <int FORMAT, int TEAM, int VECS>
cudaError_t launch(const QcacheAppendParams &p, const dim3 &grid, cudaStream_t stream) {
    return launch_behind(append_kernel<FORMAT, TEAM, VECS>, grid, kBlockWarps<TEAM> * 32, 0, stream, p);
}

}  // namespace

cudaError_t launch_qcache_append(QcacheAppendParams p, int num_sms, cudaStream_t stream) {
    if (p.num_rows == 0) return cudaSuccess;
    // Who holds a run in registers, by the elements of a block of one head:
    //   to 1024    a warp with 4 vectors a lane, 32 warps to an SM (blocks of 16 x 64, 886 MB of int8:
    //              158 us; with 40 warps a quarter more, with 24 a sixth)
    //   to 4096    a warp with 8 vectors a lane, 24 warps to an SM
    //   above      four warps, of more than 16384 eight (blocks of 128 x 256: 242 us, with four 257,
    //              with sixteen, of which fewer fit an SM, 381); all head_dim above 256 are here. Short
    //              runs in such blocks go to single warps all the same (one token of 128 requests, 36
    //              layers, blocks of 128 x 128: 48 us against 142)
    const int64_t block = (int64_t)p.head_dim << p.log2_block;
    const int team = block <= 4096 ? 1 : block <= 16384 ? 4 : 8, per = team == 1 ? 2 : 1;
    const int head_groups = (p.heads + per - 1) / per;
    // Rows per thread block: one while that leaves every SM less than about 16 thread blocks (single
    // tokens: each row is a run of its own), up to 32, of which a warp looks at the slots in one go. (With 64
    // thread blocks to an SM the ragged int8 rows take 16.1 us, with 16 13.8; with windows of no more than a block
    // of tokens the merge takes 183 us, with 32 rows 175, with 64 the same.)
    const int64_t blocks_of_one = p.num_rows * head_groups * p.layers;
    int window = 1;
    while (window < 32 && blocks_of_one / window > 16ll * num_sms) window *= 2;
    p.window = window;
    const dim3 grid((unsigned)((p.num_rows + window - 1) / window), (unsigned)head_groups, (unsigned)p.layers);
    const bool e4m3 = p.format == CM_QCACHE_E4M3;
    if (block <= 1024) return e4m3 ? launch<CM_QCACHE_E4M3, 1, 4>(p, grid, stream) : launch<CM_QCACHE_INT8, 1, 4>(p, grid, stream);
    if (team == 1) return e4m3 ? launch<CM_QCACHE_E4M3, 1, 8>(p, grid, stream) : launch<CM_QCACHE_INT8, 1, 8>(p, grid, stream);
    if (team == 4) return e4m3 ? launch<CM_QCACHE_E4M3, 4, 8>(p, grid, stream) : launch<CM_QCACHE_INT8, 4, 8>(p, grid, stream);
    return e4m3 ? launch<CM_QCACHE_E4M3, 8, 8>(p, grid, stream) : launch<CM_QCACHE_INT8, 8, 8>(p, grid, stream);
}

}  // namespace cm
