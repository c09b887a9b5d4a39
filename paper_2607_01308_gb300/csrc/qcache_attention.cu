// Attention over the 8-bit paged cache for few query rows per request (single tokens, drafts).
//
// For a query row q of head g of kv head h, over its request's tokens j the row may see:
//   s_j = scale * sum_d q_d * K_jd,   out = sum_j e^{s_j} V_j / sum_j e^{s_j}
// with K_jd = kc_jd * ks_b and V_jd = vc_jd * vs_b, b the block of token j. The codes go into
// the matrix instructions as they are (exact in fp16); the K scale multiplies the finished sum
// and the V scale joins the exponent:
//   t_j = (q . kc_j) * (scale * log2 e * ks_b) + log2 vs_b,   w_j = 2^(t_j - M)
//   out = sum_j w_j vc_j / sum_j (w_j / vs_b)
// so a block's scale costs one fused multiply-add per score and nothing per element of V. M, the
// running maximum of t, the sums and the outputs are fp32. Roundings: q is taken to fp16 after a
// power-of-two scaling of its row that puts the largest element at 2^14 (bf16's 8 bits are kept
// down to 2^-28 of it), w to fp16 with M set so that w <= 2^15 (11 bits; w below 2^-40 of the
// largest are lost), the result to bf16.
//
// Layout. A warp takes 16 tokens at a time through a ring of its own in shared memory, copied one to
// three stages ahead (64 KB and more on their way per SM), into the fragments of mma.m16n8k16: scores as
// K (16 tokens) x Q^T (8 rows), outputs as V^T (16 of head_dim) x w^T. Which element of head_dim a
// fragment position stands for is free as long as K and Q (V and the output) agree, so every lane
// reads whole vectors and no code is transposed. The work, every (request, kv head, tile of 64 tokens),
// is laid out on one line and cut evenly over a grid that just fills the GPU; where a cut falls inside a (request, head), the
// parts meet in the workspace and whoever comes last joins them in their order, so that the
// result does not depend on timing.
//
// Bound by HBM once the requests are long (above), by the chain of dependent reads (lengths, table, scales,
// tokens, parts) when they are short: one token over 1,041 cached 8.8 us; 64 requests of 600 to 12,000 tokens 84 us
// (5.9 TB/s); 29 requests, int8 drafts of 3 or 4 rows, 18 us. At head_dim 32 and 64 neither HBM nor issue is full (64: 47
// and 52 % over 32 x 4,096 tokens): a warp's own chain of copy, conversion and products per 16 tokens.
#include "cm_qcache_kernels.h"

#include <atomic>

#include "cm_qcache_codes.h"
#include "cm_qcache_attention.h"

namespace cm {
namespace {

constexpr int kWarps = 4;
constexpr int kThreads = kWarps * 32;
constexpr int kTile = 16 * kWarps;          // tokens of a tile
constexpr float kRaise = 8.f;               // M moves when a score passes it by more
constexpr float kHeadroom = 7.f;            // w <= 2^(kRaise + kHeadroom)

__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3,
                                        uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
                 "{%0, %1, %2, %3};"
                 : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
                 : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

__device__ __forceinline__ uint32_t transpose8x8(uint32_t x) {
    uint32_t y;
    asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

template <int N>
__device__ __forceinline__ void load_words(uint32_t *w, const unsigned char *p) {
    if constexpr (N == 16) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        w[0] = v.x; w[1] = v.y; w[2] = v.z; w[3] = v.w;
    } else if constexpr (N == 8) {
        const uint2 v = *reinterpret_cast<const uint2 *>(p);
        w[0] = v.x; w[1] = v.y;
    } else {
        w[0] = *reinterpret_cast<const uint32_t *>(p);
    }
}

__device__ __forceinline__ void copy16(unsigned char *to, const uint8_t *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((uint32_t)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_end_group() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

template <int D, int FORMAT, int NT>
struct Decode {
    static constexpr int kRows = 8 * NT;                      // query rows of a tile
    static constexpr int kVecK = D / 4 < 16 ? D / 4 : 16;     // bytes of a K read: a lane has D / 4 of a row
    static constexpr int kVecV = D / 8 < 16 ? D / 8 : 16;     // bytes of a V read: D / 8 of a row
    static constexpr int kWordsK = D / 16, kWordsV = D / 32;
    static constexpr int kPitch = D + 4;                      // floats of a row in shared memory
    static constexpr int kBlocksPerSm = D == 256 ? 2 : NT == 2 ? 3 : 4;
    static constexpr int kSetup = D >= 128 ? 2 : 256 / D;     // about 2.5 us in tiles of 128 D bytes at a block's share of HBM
    static constexpr int kStageBytes = 32 * D;                // 16 tokens of K, then of V
    // More on its way at once is slower: 32 requests of 16,384 tokens, head_dim 128, take 167 us (6.4 TB/s) with two
    // stages, 180 with three; head_dim 64 91 us with three, 95 with four, 103 with two; head_dim 256 170 with two, 181
    // with three. So are more blocks with fewer registers (head_dim 64: five 101 us) and fewer blocks (three 103).
    static constexpr int kStages = D >= 128 ? 2 : D == 64 ? 3 : 4;
    static constexpr int kRing = kWarps * kStages * kStageBytes;
    static constexpr int kMerge = kWarps * kRows * (kPitch + 2) * 4;   // over the ring, once it has been read
    static constexpr size_t kShared = kRing > kMerge ? kRing : kMerge;
    // Places of a row's 16-byte chunks, so that the lanes that read together (K: two rows and four chunks; V: four
    // rows two apart and two chunks) meet no bank twice.
    static __device__ __forceinline__ int place_k(int row, int chunk) { return D >= 128 ? chunk ^ (row & 1) << 2 : chunk; }
    static __device__ __forceinline__ int place_v(int row, int chunk) {
        return D >= 128 ? chunk ^ (row >> 1 & 3) << 1 : D == 64 ? chunk ^ (row >> 1 & 3) : chunk;
    }
};

template <int D, int FORMAT, int NT, bool TREE>
__global__ void __launch_bounds__(kThreads, Decode<D, FORMAT, NT>::kBlocksPerSm)
    decode_kernel(const __grid_constant__ QcacheAttentionParams p) {
    using C = Decode<D, FORMAT, NT>;
    extern __shared__ __align__(16) unsigned char smem[];
    float *merge_o = reinterpret_cast<float *>(smem);                        // [warps][rows][pitch]
    float *merge_ml = merge_o + kWarps * C::kRows * C::kPitch;               // [warps][rows][2]
    uint32_t *prefix = reinterpret_cast<uint32_t *>(smem + C::kShared);
    __shared__ float4 ring_scales[kWarps][C::kStages];                       // k_scale, log2 v_scale, 1 / v_scale, block
    __shared__ uint32_t scan[kWarps];
    __shared__ uint32_t last_one;
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, g = lane / 4, t = lane % 4;
    after_kernels_before();

    const uint32_t per_head = plan_units<kThreads, C::kRows, kTile, C::kSetup>(p, prefix, scan);
    const uint64_t units = (uint64_t)per_head * (uint32_t)p.heads;
    const uint64_t per = units_per_block<C::kSetup>(units, gridDim.x);
    uint64_t u = (uint64_t)blockIdx.x * per;
    const uint64_t u_end = min(u + per, units);

    while (u < u_end) {
        const AttentionSegment w = locate<C::kRows, kTile, C::kSetup>(p, prefix, u, u_end);
        if (w.t0 == w.t1) continue;
        const int64_t kv_head = w.head;

        // The warp's own ring: 16 tokens of K and V a stage, copied some stages ahead. A lane looks up the block of
        // one tile, for 32 tiles at a time; a tile without a block is passed over.
        const uint8_t *k_head = p.k + kv_head * p.stride_head, *v_head = p.v + kv_head * p.stride_head;
        const int in_block = (1 << p.log2_block) - 1;
        unsigned char *ring = smem + warp * (C::kStages * C::kStageBytes);
        BlockEntry mine;
        auto issue = [&](int ti) {
            if (ti < w.t1) {
                const int at = (ti - w.t0) % 32;
                if (at == 0)
                    mine = block_entry(p, w.request, kv_head, (int64_t)(ti + lane) * kTile + warp * 16, ti + lane < w.t1 ? w.kv : 0);
                const BlockEntry e = shuffle(mine, at);
                const int stage = (ti - w.t0) % C::kStages;
                if (lane == 0) ring_scales[warp][stage] = make_float4(e.k_scale, e.v_log2, e.v_inverse, __int_as_float(e.block));
                if (e.block >= 0) {
                    constexpr int kPerRow = D / 16, kStep = 32 / kPerRow;   // chunks of a row, rows of one copy
                    const int row = lane / kPerRow, chunk = lane % kPerRow;
                    const int64_t from = (int64_t)e.block * p.stride_block +
                                         (int64_t)(((ti * kTile + warp * 16) & in_block) + row) * p.stride_token + chunk * 16;
                    unsigned char *to = ring + stage * C::kStageBytes + row * D;
#pragma unroll
                    for (int r = 0; r < 16; r += kStep) {
                        copy16(to + r * D + C::place_k(row + r, chunk) * 16, k_head + from + r * p.stride_token);
                        copy16(to + (16 + r) * D + C::place_v(row + r, chunk) * 16, v_head + from + r * p.stride_token);
                    }
                }
            }
            copies_end_group();
        };
#pragma unroll
        for (int i = 0; i < C::kStages - 1; ++i) issue(w.t0 + i);

        // the query rows of this lane's fragments, as fp16 with a power of two per row
        uint32_t qf[NT][D / 8];
        float row_factor[NT][2];
        int limit[NT][2];                       // tokens that rows 2t and 2t + 1 may see
        int least = w.kv;                       // of the rows in the tile
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
            const int n = w.row_tile * C::kRows + nt * 8 + g;
            const bool valid = n < w.rows;
            const int i = n / p.group;
            const uint16_t *q = p.q + (int64_t)(w.row0 + i) * p.q_stride_row +
                                (kv_head * p.group + n % p.group) * p.q_stride_head;
            uint32_t raw[D / 8];
#pragma unroll
            for (int c = 0; c < D / (4 * C::kVecK); ++c)
#pragma unroll
                for (int e = 0; e < C::kVecK / 8; ++e) {
                    const uint4 x = valid ? *reinterpret_cast<const uint4 *>(q + c * 4 * C::kVecK + t * C::kVecK + e * 8)
                                          : make_uint4(0, 0, 0, 0);
                    const int at = c * C::kVecK / 2 + e * 4;
                    raw[at] = x.x; raw[at + 1] = x.y; raw[at + 2] = x.z; raw[at + 3] = x.w;
                }
            uint32_t m = 0;
#pragma unroll
            for (int x = 0; x < D / 8; ++x) m = __vmaxu2(m, raw[x] & 0x7fff7fffu);
            m = max(m & 0xffffu, m >> 16);
            m = max(m, __shfl_xor_sync(~0u, m, 1));
            m = max(m, __shfl_xor_sync(~0u, m, 2));
            const int e = max((int)(m >> 7) - 127, -100);
            const float up = pow2f(14 - e);
#pragma unroll
            for (int x = 0; x < D / 8; ++x)
                qf[nt][x] = pack_half(__uint_as_float(raw[x] << 16) * up, __uint_as_float(raw[x] & 0xffff0000u) * up);
            const float f = p.scale_log2 * pow2f(e - 14);
            const int lim = !valid ? 0 : p.causal ? min(w.kv, max(0, w.first + i + 1)) : w.kv;
            if (valid) least = min(least, lim);
#pragma unroll
            for (int b = 0; b < 2; ++b) {
                row_factor[nt][b] = __shfl_sync(~0u, f, (2 * t + b) * 4);
                limit[nt][b] = __shfl_sync(~0u, lim, (2 * t + b) * 4);
            }
        }
        least = TREE ? min(least, w.first) : __reduce_min_sync(~0u, least);

        float o[D / 16][NT][4];
        float top[NT][2], sum[NT][2];
#pragma unroll
        for (int i = 0; i < D / 16; ++i)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                for (int x = 0; x < 4; ++x) o[i][nt][x] = 0.f;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) top[nt][0] = top[nt][1] = -INFINITY, sum[nt][0] = sum[nt][1] = 0.f;

        for (int ti = w.t0; ti < w.t1; ++ti) {
            const int token = ti * kTile + warp * 16, stage = (ti - w.t0) % C::kStages;
            copies_wait<C::kStages - 2>();
            __syncwarp();                         // the warp's copies are there, and the stage before has been read
            issue(ti + C::kStages - 1);
            const float4 z = ring_scales[warp][stage];
            const BlockEntry b{__float_as_int(z.w), z.x, z.y, z.z};
            if (b.block < 0) continue;
            const unsigned char *k_at = ring + stage * C::kStageBytes, *v_at = k_at + 16 * D;

            // what of the request's own rows the rows see, in its last tiles: on its way while the scores are computed
            uint32_t seen[NT][2];
            if (TREE && token + 16 > least) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        const int n = w.row_tile * C::kRows + nt * 8 + 2 * t + b;
                        seen[nt][b] = 0;
                        if (n < w.rows)
                            seen[nt][b] = tree_window(p.tree + (int64_t)(w.row0 + n / p.group) * p.tree_words, p.tree_words, token - w.first);
                    }
            }
            float s[NT][4];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) s[nt][0] = s[nt][1] = s[nt][2] = s[nt][3] = 0.f;
#pragma unroll
            for (int c = 0; c < C::kWordsK * 4 / C::kVecK; ++c) {
                uint32_t kw[2][C::kVecK / 4];
#pragma unroll
                for (int x = 0; x < 2; ++x)
                    load_words<C::kVecK>(kw[x], C::kVecK == 16 ? k_at + (g + 8 * x) * D + C::place_k(g, c * 4 + t) * 16
                                                               : k_at + (g + 8 * x) * D + t * C::kVecK);
#pragma unroll
                for (int i = 0; i < C::kVecK / 4; ++i) {
                    const int j = c * (C::kVecK / 4) + i;
                    uint32_t a0, a1, a2, a3;
                    codes_to_half<FORMAT>(kw[0][i], a0, a2);
                    codes_to_half<FORMAT>(kw[1][i], a1, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(s[nt], a0, a1, a2, a3, qf[nt][2 * j], qf[nt][2 * j + 1]);
                }
            }
            bool raise = false;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float f0 = row_factor[nt][0] * b.k_scale, f1 = row_factor[nt][1] * b.k_scale;
                s[nt][0] = fmaf(s[nt][0], f0, b.v_log2);
                s[nt][1] = fmaf(s[nt][1], f1, b.v_log2);
                s[nt][2] = fmaf(s[nt][2], f0, b.v_log2);
                s[nt][3] = fmaf(s[nt][3], f1, b.v_log2);
                if (TREE && token + 16 > least) {
#pragma unroll
                    for (int b = 0; b < 2; ++b) {
                        if (!(seen[nt][b] >> g & 1) || token + g >= w.kv) s[nt][b] = -INFINITY;
                        if (!(seen[nt][b] >> (g + 8) & 1) || token + g + 8 >= w.kv) s[nt][2 + b] = -INFINITY;
                    }
                } else if (token + 16 > least) {
                    if (token + g >= limit[nt][0]) s[nt][0] = -INFINITY;
                    if (token + g >= limit[nt][1]) s[nt][1] = -INFINITY;
                    if (token + g + 8 >= limit[nt][0]) s[nt][2] = -INFINITY;
                    if (token + g + 8 >= limit[nt][1]) s[nt][3] = -INFINITY;
                }
                raise |= fmaxf(s[nt][0], s[nt][2]) > top[nt][0] + kRaise || fmaxf(s[nt][1], s[nt][3]) > top[nt][1] + kRaise;
            }
            if (__any_sync(~0u, raise)) {
#pragma unroll
                for (int nt = 0; nt < NT; ++nt)
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        float m = fmaxf(s[nt][c], s[nt][c + 2]);
#pragma unroll
                        for (int d = 4; d < 32; d *= 2) m = fmaxf(m, __shfl_xor_sync(~0u, m, d));
                        m = fmaxf(m, top[nt][c]);
                        const float f = top[nt][c] == m ? 1.f : exp2_fast(top[nt][c] - m);
                        top[nt][c] = m;
                        sum[nt][c] *= f;
#pragma unroll
                        for (int i = 0; i < D / 16; ++i) o[i][nt][c] *= f, o[i][nt][c + 2] *= f;
                    }
            }
            uint32_t w0[NT], w1[NT];
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                const float m0 = (top[nt][0] == -INFINITY ? 0.f : top[nt][0]) - kHeadroom;
                const float m1 = (top[nt][1] == -INFINITY ? 0.f : top[nt][1]) - kHeadroom;
                const float e0 = exp2_fast(s[nt][0] - m0), e1 = exp2_fast(s[nt][1] - m1);
                const float e2 = exp2_fast(s[nt][2] - m0), e3 = exp2_fast(s[nt][3] - m1);
                sum[nt][0] = fmaf(e0 + e2, b.v_inverse, sum[nt][0]);
                sum[nt][1] = fmaf(e1 + e3, b.v_inverse, sum[nt][1]);
                w0[nt] = transpose8x8(pack_half(e0, e1));
                w1[nt] = transpose8x8(pack_half(e2, e3));
            }
#pragma unroll
            for (int c = 0; c < C::kWordsV * 4 / C::kVecV; ++c) {
                uint32_t vw[4][C::kVecV / 4];
#pragma unroll
                for (int x = 0; x < 4; ++x) {
                    const int row = 2 * t + (x & 1) + 8 * (x >> 1), byte = c * 8 * C::kVecV + g * C::kVecV;
                    load_words<C::kVecV>(vw[x], v_at + row * D + C::place_v(row, byte / 16) * 16 + byte % 16);
                    if (token + 16 > w.kv && token + row >= w.kv)   // what lies behind the last token may be anything
#pragma unroll
                        for (int i = 0; i < C::kVecV / 4; ++i) vw[x][i] = 0;
                }
#pragma unroll
                for (int j = 0; j < C::kVecV / 4; ++j) {
                    const int i = c * (C::kVecV / 4) + j;
                    uint32_t a0, a1, a2, a3;    // bytes 4i, 4i + 1: fragment rows g and g + 8
                    codes_to_half<FORMAT>(prmt(vw[0][j], vw[1][j], 0x5140), a0, a1);
                    codes_to_half<FORMAT>(prmt(vw[2][j], vw[3][j], 0x5140), a2, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(o[2 * i][nt], a0, a1, a2, a3, w0[nt], w1[nt]);
                    codes_to_half<FORMAT>(prmt(vw[0][j], vw[1][j], 0x7362), a0, a1);
                    codes_to_half<FORMAT>(prmt(vw[2][j], vw[3][j], 0x7362), a2, a3);
#pragma unroll
                    for (int nt = 0; nt < NT; ++nt) mma_f16(o[2 * i + 1][nt], a0, a1, a2, a3, w0[nt], w1[nt]);
                }
            }
        }
        copies_wait<0>();
        __syncthreads();                          // every warp has read its ring: the parts go over it

        // the four warps' parts through shared memory
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int c = 0; c < 2; ++c) {
#pragma unroll
                for (int d = 4; d < 32; d *= 2) sum[nt][c] += __shfl_xor_sync(~0u, sum[nt][c], d);
                const int n = nt * 8 + 2 * t + c;
                if (g == 0) {
                    merge_ml[(warp * C::kRows + n) * 2] = top[nt][c];
                    merge_ml[(warp * C::kRows + n) * 2 + 1] = sum[nt][c];
                }
                float *row = merge_o + (warp * C::kRows + n) * C::kPitch;
#pragma unroll
                for (int i = 0; i < C::kWordsV; ++i) {
                    const int byte = 4 * i, d = byte / C::kVecV * 8 * C::kVecV + g * C::kVecV + byte % C::kVecV;
                    *reinterpret_cast<float4 *>(row + d) =
                        make_float4(o[2 * i][nt][c], o[2 * i][nt][c + 2], o[2 * i + 1][nt][c], o[2 * i + 1][nt][c + 2]);
                }
            }
        __syncthreads();
        const int rows = min(C::kRows, w.rows - w.row_tile * C::kRows);
        const bool whole = w.t0 == 0 && w.t1 == w.tiles;
        const int64_t part = 2 * (int64_t)blockIdx.x + (w.t0 == 0);
        for (int x = tid; x < rows * (D / 4); x += kThreads) {
            const int n = x / (D / 4), d = x % (D / 4) * 4;
            float m = -INFINITY;
#pragma unroll
            for (int y = 0; y < kWarps; ++y) m = fmaxf(m, merge_ml[(y * C::kRows + n) * 2]);
            float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
            float l = 0.f;
#pragma unroll
            for (int y = 0; y < kWarps; ++y) {
                const float m_y = merge_ml[(y * C::kRows + n) * 2], f = m_y == m ? 1.f : exp2_fast(m_y - m);
                const float4 x = *reinterpret_cast<const float4 *>(merge_o + (y * C::kRows + n) * C::kPitch + d);
                acc.x = fmaf(x.x, f, acc.x); acc.y = fmaf(x.y, f, acc.y);
                acc.z = fmaf(x.z, f, acc.z); acc.w = fmaf(x.w, f, acc.w);
                l = fmaf(merge_ml[(y * C::kRows + n) * 2 + 1], f, l);
            }
            if (whole) {
                write_row(p, w, w.row_tile * C::kRows + n, d, acc, m, l, kHeadroom);
            } else {
                __stcg(reinterpret_cast<float4 *>(p.part_o + (part * C::kRows + n) * D + d), acc);
                if (d == 0) __stcg(reinterpret_cast<float2 *>(p.part_ml + (part * C::kRows + n) * 2), make_float2(m, l));
            }
        }
        if (!whole) {
            const uint64_t begin = w.unit0, end = w.unit0 + w.tiles;
            const uint32_t c0 = (uint32_t)(begin / per), c1 = (uint32_t)((end - 1) / per);
            __threadfence();
            __syncthreads();
            if (tid == 0) last_one = atomicInc(p.arrived + c0, c1 - c0) == c1 - c0;
            __syncthreads();
            if (last_one) {
                __threadfence();
                join_parts<D, kWarps>(p, w, w.row_tile * C::kRows, rows, c0, c1, kHeadroom, warp,
                                      [&](uint32_t c, int n) { return (2 * (int64_t)c + (c == c0)) * C::kRows + n; });
            }
        }
        __syncthreads();
    }
}

template <int D, int FORMAT, int NT, bool TREE>
cudaError_t launch(const QcacheAttentionParams &p, int num_sms, int device, cudaStream_t stream) {
    using C = Decode<D, FORMAT, NT>;
    static std::atomic<uint64_t> allowed{0};   // devices on which the shared memory limit is raised
    const size_t smem = C::kShared + ((size_t)p.requests + 1) * 4;
    // whatever this call needs: the limit without it covers the static bytes too
    if (device >= 64 || !(allowed.load() >> device & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(decode_kernel<D, FORMAT, NT, TREE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)(C::kShared + (kQcacheMaxAttentionRequests + 1) * 4));
        if (e != cudaSuccess) return e;
        if (device < 64) allowed.fetch_or(1ull << device);
    }
    return launch_behind(decode_kernel<D, FORMAT, NT, TREE>, dim3(num_sms * C::kBlocksPerSm), kThreads, smem, stream, p);
}

}  // namespace

// Part rows of a whole launch, of either kernel.
static size_t part_rows(int head_dim, int num_sms) {
    const size_t decode = (size_t)num_sms * kQcacheDecodeBlocksPerSm * 16, prefill = num_sms * qcache_prefill_part_rows(head_dim);
    return 2 * (decode > prefill ? decode : prefill);
}

// What comes first, at the same place for every head_dim: the arrival counters, which have to be
// zero, and the splits.
static size_t counter_bytes(int num_sms) { return (size_t)num_sms * kQcacheDecodeBlocksPerSm * 4; }
static size_t head_bytes(int num_sms) { return counter_bytes(num_sms) + ((size_t)num_sms * sizeof(QcacheSplit) + 15) / 16 * 16; }

size_t qcache_workspace_bytes(int head_dim, int num_sms) {
    return head_bytes(num_sms) + part_rows(head_dim, num_sms) * ((size_t)head_dim + 2) * 4;
}

void qcache_workspace_split(QcacheAttentionParams &p, void *workspace, int num_sms) {
    unsigned char *at = static_cast<unsigned char *>(workspace);
    p.arrived = reinterpret_cast<unsigned int *>(at);
    p.splits = reinterpret_cast<QcacheSplit *>(at + counter_bytes(num_sms));
    p.part_o = reinterpret_cast<float *>(at + head_bytes(num_sms));
    p.part_ml = p.part_o + part_rows(p.head_dim, num_sms) * p.head_dim;
}

#define CM_EACH_DECODE(X) \
    X(32, CM_QCACHE_E4M3) X(64, CM_QCACHE_E4M3) X(128, CM_QCACHE_E4M3) X(256, CM_QCACHE_E4M3) \
    X(32, CM_QCACHE_INT8) X(64, CM_QCACHE_INT8) X(128, CM_QCACHE_INT8) X(256, CM_QCACHE_INT8)

cudaError_t launch_qcache_attention(const QcacheAttentionParams &p, int rows_per_request, int num_sms, int device,
                                    cudaStream_t stream) {
    // Rows of a request and kv head: to 8 in one fragment, to 16 in two at once, to 32 (not at head_dim 256) in two
    // tiles of those, which read the cache twice; above, the other kernel. Measured, 32 requests of 4,096 tokens, 8 kv heads:
    //   head_dim 128 e4m3   8 rows 52 us, as two fragments 56; 16 rows 60 us, as two tiles of one 91;
    //                       32 rows 97 us, by the other kernel 105 (one request of 131,072 tokens: 101 by either)
    //   head_dim 64 int8    8 rows 33 us, as two fragments 40; 32 rows 72 us, by the other kernel 90
    //   head_dim 32 e4m3    32 rows 50 us, by the other kernel 83
    //   head_dim 256 e4m3   (16 requests, 4 kv heads) 32 rows 59 us, by the other kernel 48
    // Trees, whose other kernel has two streams for up to 128 rows:
    //   head_dim 128 e4m3   32 rows 103 us, by the other kernel 95; int8 115 and 99
    //   head_dim 64 e4m3    32 rows 69 us, by the other kernel 71; head_dim 32 53 and 66
    if (rows_per_request > (p.head_dim == 256 || (p.tree && p.head_dim == 128) ? 16 : 32)) return launch_qcache_prefill(p, rows_per_request, num_sms, device, stream);
#define CM_LAUNCH(D, F) \
    if (p.head_dim == D && p.format == F) \
        return rows_per_request <= 8 ? p.tree ? launch<D, F, 1, true>(p, num_sms, device, stream) : launch<D, F, 1, false>(p, num_sms, device, stream) \
               : p.tree ? launch<D, F, 2, true>(p, num_sms, device, stream) : launch<D, F, 2, false>(p, num_sms, device, stream);
    CM_EACH_DECODE(CM_LAUNCH)
#undef CM_LAUNCH
    return cudaErrorInvalidValue;
}

}  // namespace cm
