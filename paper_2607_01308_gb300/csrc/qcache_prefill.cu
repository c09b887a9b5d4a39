// Attention over the 8-bit paged cache for many query rows per request (prompts, chunks of them).
// The mathematics and the roundings are those of qcache_attention.cu: codes enter the matrix
// instructions as fp16, the K scale multiplies the finished score, the V scale joins the exponent.
//
// One thread block per SM, on the tcgen05 tensor cores, with up to 256 query rows (rows are query
// tokens x heads of a group) in two tiles of 128, so that each K and V tile that is brought in and
// taken to fp16 serves both:
//   warps 0-3, 4-7   softmax of query tile 0 and 1, one row per thread: a kv tile (64 scores) from tensor
//                    memory into registers, weights back into the same columns as fp16, the output
//                    rescaled when the running maximum is raised, the row normalised and written
//   warps 8-11       K tiles, from global memory through registers to fp16 in shared memory, in the 128-byte
//                    swizzle, the next tile's codes on their way meanwhile
//   warps 12-15      V tiles
//   warp 16 (, 18)   issue the matrix instructions (at head_dim 128 a warp for each query tile):
//                    S = Q K^T (both operands from shared memory), O += P V (P from tensor memory, V as it
//                    lies, tokens x head_dim)
//   warp 17          looks up blocks and scales of every 16 tokens, several tiles ahead
// Scores are computed two kv tiles ahead, into two buffers for each query tile, so that the softmax warps
// always have a tile at hand while the tensor cores take the last one's weights. Products of 128 x 64 leave
// a third of the tensor cores' time to the operands' way from shared memory; with tiles of 128 tokens, for
// which there is one buffer, softmax and products wait for each other (513 us against 464 for the chunk
// below). The softmax warps take registers over from the others. Work is cut as in qcache_attention.cu, over
// kv tiles that the rows of a tile may see at all; a second, small kernel joins the ranges that were cut
// between thread blocks, over the whole GPU (one thread block alone took 95 us for 256 rows in 19 parts).
//
// Bound by the tensor cores and the softmax's latency together (the tensor pipe is 56 % busy with 1,024 rows x 4 over
// 8,192 tokens): 2,048 rows x 4 heads of a group over 16,384 tokens, 8 kv heads of 128, 465 us (1,256 TFLOP/s); by
// latency where prompts are short: 64 tokens of that shape 17.6 us, eight of 700 80 us, five ragged ones of
// head_dim 256 48 us. What a range costs besides its tiles is spent in series: output out, queries in, first product.
#include "cm_qcache_kernels.h"

#include <atomic>
#include <type_traits>

#include "cm_qcache_attention.h"
#include "cm_qcache_codes.h"

namespace cm {
namespace {

constexpr int kSoftmaxWarps = 8, kLoadWarps = 4;              // load warps: for K, and as many for V
constexpr int kMmaWarp = kSoftmaxWarps + 2 * kLoadWarps, kEntryWarp = kMmaWarp + 1, kSecondMmaWarp = kMmaWarp + 2;
constexpr int kThreads = 20 * 32;           // whole warpgroups: registers change hands by warpgroup
constexpr int kLaunchRegs = 96;
constexpr int kLoadThreads = kLoadWarps * 32;
constexpr float kRaise = 8.f, kHeadroom = 7.f;

constexpr int kTile = 64;                   // tokens of a kv tile
constexpr int kBlocks = kTile / 16;         // its scale entries
constexpr int kEntryTiles = 32 / kBlocks, kEntryStages = 2 * kEntryTiles;   // tiles looked up at a time; held

template <int D>
struct Shape {
    // tensor memory, 512 columns: two buffers of scores for each query tile, and the outputs
    static constexpr int kQTiles = D == 256 ? 1 : 2;
    // Warps that issue: one for each query tile at head_dim 128, where one for both waits for the weights of one
    // tile while those of the other are there (2,048 tokens over 16,384: 467 us against 520); below, where the
    // products are short, one (head_dim 64: 433 us against 461), which keeps the two tiles' softmax apart.
    static constexpr int kIssuers = D == 128 ? 2 : 1;
    static constexpr int kRows = 128 * kQTiles;
    static constexpr int kOColumn = kQTiles * 2 * kTile;
    static constexpr int kSetup = 4;                          // a segment's queries and its end, in tiles: 8,700 to 11,000 cycles
    static constexpr int kPanels = D < 64 ? 1 : D / 64;       // 64 columns (128 bytes) of fp16 each
    static constexpr int kStages = D == 256 ? 2 : 4;          // tiles of K, of V
    static constexpr int kQPanel = 128 * 128, kKvPanel = kTile * 128;   // bytes
    static constexpr int kQBytes = kQTiles * kPanels * kQPanel;
    static constexpr int kKvBytes = kPanels * kKvPanel;       // a tile of K, of V
    static constexpr int kChunks = kTile * D / 16 / kLoadThreads;   // 16-code loads of a thread for a tile
    static constexpr size_t kSmem = kQBytes + 2 * kStages * kKvBytes;
    // registers of the softmax, the converting and the issuing warps; where the second half of the softmax
    // warps has no tile, the converting ones have its
    static constexpr int kSoftmaxRegs = 120, kIdleRegs = 32, kLoadRegs = kQTiles == 1 ? 128 : 88, kIssueRegs = 64;
    static_assert(128 * kSoftmaxRegs + 128 * (kQTiles == 1 ? kIdleRegs : kSoftmaxRegs) + 256 * kLoadRegs + 128 * kIssueRegs <=
                      kThreads * kLaunchRegs, "registers at launch");
    static_assert(kChunks >= 1, "every load thread has work");
    static_assert(kOColumn + kQTiles * D <= 512, "tensor memory");
};

// ---------------------------------------------------------------- barriers, bounded

__device__ __forceinline__ uint32_t smem_u32(const void *p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void bar_init(uint64_t *b, int n) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_u32(b)), "r"(n) : "memory");
}

__device__ __forceinline__ void bar_arrive(uint64_t *b) {
    asm volatile("{\n.reg .b64 t;\nmbarrier.arrive.shared::cta.b64 t, [%0];\n}" ::"r"(smem_u32(b)) : "memory");
}

__device__ __forceinline__ bool bar_try(uint64_t *b, uint32_t parity) {
    uint32_t ok;
    asm volatile("{\n.reg .pred p;\nmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, 1000000;\nselp.u32 %0, 1, 0, p;\n}"
                 : "=r"(ok) : "r"(smem_u32(b)), "r"(parity) : "memory");
    return ok != 0;
}

// Waits for the phase of the given parity. A wait that runs out (2 * 10^9 cycles, about a second) is recorded, and every
// later one then gives up after two tries (measured: 864 tiles of three such waits end 7 ms after the first), so that the
// block runs to its end with a wrong result that the host can learn of.
__device__ __forceinline__ void bar_wait_slow(uint64_t *b, uint32_t parity, volatile int *failed, unsigned int *error) {
    const long long t0 = clock64();
    while (!bar_try(b, parity)) {
        if (*failed) return;
        if (clock64() - t0 > 2000000000ll) {
            *failed = 1;
            atomicOr(error, 1u);
            return;
        }
    }
}

struct Waiter {
    int *failed;
    unsigned int *error;
    __device__ __forceinline__ void operator()(uint64_t *b, uint32_t parity) const {
        if (!bar_try(b, parity)) bar_wait_slow(b, parity, failed, error);
    }
    // of a whole warp, which goes on together
    __device__ __forceinline__ void warp(uint64_t *b, uint32_t parity) const {
        (*this)(b, parity);
        __syncwarp();
    }
};

// ---------------------------------------------------------------- tcgen05

__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_async_smem() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }

// One lane of a converged warp, the same each time.
__device__ __forceinline__ uint32_t elect() {
    uint32_t leader;
    asm volatile("{\n.reg .pred p;\nelect.sync _|p, 0xffffffff;\nselp.u32 %0, 1, 0, p;\n}" : "=r"(leader));
    return leader;
}

// The whole warp runs the code around these, so that addresses and descriptors stay uniform; the
// leader alone acts.
__device__ __forceinline__ void commit(uint64_t *b, uint32_t leader) {
    asm volatile("{\n.reg .pred p;\nsetp.ne.u32 p, %1, 0;\n"
                 "@p tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(smem_u32(b)), "r"(leader) : "memory");
}

#define CM_REGS16(x, i) \
    "=r"(x[i]), "=r"(x[i + 1]), "=r"(x[i + 2]), "=r"(x[i + 3]), "=r"(x[i + 4]), "=r"(x[i + 5]), "=r"(x[i + 6]), "=r"(x[i + 7]), \
    "=r"(x[i + 8]), "=r"(x[i + 9]), "=r"(x[i + 10]), "=r"(x[i + 11]), "=r"(x[i + 12]), "=r"(x[i + 13]), "=r"(x[i + 14]), "=r"(x[i + 15])
#define CM_IN16(x, i) \
    "r"(x[i]), "r"(x[i + 1]), "r"(x[i + 2]), "r"(x[i + 3]), "r"(x[i + 4]), "r"(x[i + 5]), "r"(x[i + 6]), "r"(x[i + 7]), \
    "r"(x[i + 8]), "r"(x[i + 9]), "r"(x[i + 10]), "r"(x[i + 11]), "r"(x[i + 12]), "r"(x[i + 13]), "r"(x[i + 14]), "r"(x[i + 15])

#define CM_INOUT16(x, i) \
    "+r"(x[i]), "+r"(x[i + 1]), "+r"(x[i + 2]), "+r"(x[i + 3]), "+r"(x[i + 4]), "+r"(x[i + 5]), "+r"(x[i + 6]), "+r"(x[i + 7]), \
    "+r"(x[i + 8]), "+r"(x[i + 9]), "+r"(x[i + 10]), "+r"(x[i + 11]), "+r"(x[i + 12]), "+r"(x[i + 13]), "+r"(x[i + 14]), "+r"(x[i + 15])

// Columns of the warp's 32 lanes, one row per thread; the values are there after ld_wait.
__device__ __forceinline__ void tmem_ld(uint32_t (&x)[32], uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
                 "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
                 : CM_REGS16(x, 0), CM_REGS16(x, 16) : "r"(at));
}
__device__ __forceinline__ void tmem_ld(uint32_t (&x)[8], uint32_t at) {
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
                 : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]), "=r"(x[4]), "=r"(x[5]), "=r"(x[6]), "=r"(x[7]) : "r"(at));
}
// Waits for the loads; what is done with x comes after that, copies of its registers too.
__device__ __forceinline__ void ld_wait(uint32_t (&x)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    asm volatile("" : CM_INOUT16(x, 0), CM_INOUT16(x, 16) :: "memory");
}
__device__ __forceinline__ void ld_wait(uint32_t (&x)[8]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
    asm volatile("" : "+r"(x[0]), "+r"(x[1]), "+r"(x[2]), "+r"(x[3]), "+r"(x[4]), "+r"(x[5]), "+r"(x[6]), "+r"(x[7]) :: "memory");
}
__device__ __forceinline__ void tmem_st8(uint32_t at, const uint32_t (&x)[8]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
                 ::"r"(at), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]), "r"(x[4]), "r"(x[5]), "r"(x[6]), "r"(x[7]) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t at, const uint32_t (&x)[16]) {
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
                 ::"r"(at), CM_IN16(x, 0) : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Shared memory operand in 128-byte swizzled atoms of 8 rows x 128 bytes. Rows of K (and Q) are
// tokens (query rows) and the contraction runs along a row; for V the contraction runs over rows.
// The descriptor's lower word moves with the address, in units of 16 bytes.
__device__ __forceinline__ uint32_t operand_lo(uint32_t addr, uint32_t leading) { return (addr & 0x3ffff) >> 4 | (leading >> 4) << 16; }
__device__ __forceinline__ uint64_t operand(uint32_t lo) {
    uint64_t d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "r"(lo), "n"(1024u >> 4 | 1u << 14 | 2u << 29));   // 1024 bytes to the next eight rows
    return d;
}

// fp32 accumulator, fp16 operands; b_rows: B's contraction runs over rows.
__host__ __device__ constexpr uint32_t instruction(int m, int n, bool b_rows) {
    return 1u << 4 | (b_rows ? 1u << 16 : 0u) | (uint32_t)(n / 8) << 17 | (uint32_t)(m / 16) << 24;
}

__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t leader) {
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %5, 0;\n"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate, uint32_t leader) {
    asm volatile("{\n.reg .pred p, q;\nsetp.ne.u32 p, %4, 0;\nsetp.ne.u32 q, %5, 0;\n"
                 "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate), "r"(leader) : "memory");
}

// 16 codes, read once by this block.
__device__ __forceinline__ uint4 load_codes(const uint8_t *p) {
    uint4 x;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w) : "l"(p));
    return x;
}

// ---------------------------------------------------------------- softmax

// A pair of fp32 values in one 64-bit register, for the two-wide instructions.
__device__ __forceinline__ uint64_t pair(float x, float y) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
    return v;
}
__device__ __forceinline__ void unpair(uint64_t v, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
    uint64_t v;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(v) : "l"(a), "l"(b), "l"(c));
    return v;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
    uint64_t v;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(v) : "l"(a), "l"(b));
    return v;
}

// What a tile needs to know of each 16 tokens: the scales, and where their codes begin in a head's plane, in
// bytes (negative: in a block that is not there, or past the request's tokens).
struct alignas(16) Entries {      // read 16 bytes at a time
    float2 scale[kBlocks];        // k_scale, log2 v_scale
    float v_inverse[kBlocks];
    int64_t offset[kBlocks];
};
static_assert(sizeof(Entries) % 16 == 0 && kBlocks % 4 == 0, "every tile's entries are aligned alike");

// What a softmax thread keeps of its row. The weights of a tile are 2^(t - top + headroom); `limit` is the
// largest exponent that is let pass: without bound until the row has seen a token, which then sets `top`.
struct RowState {
    float top, sum, limit;
};

__device__ __forceinline__ float max3(float a, float b, float c) {
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(a), "f"(b), "f"(c));
    return m;
}

// A kv tile of one row: scores x to weights w (fp16 pairs). left: columns that the row sees (only if
// `masked`, which is the warp's). Where the largest exponent of some row passes its limit, that row's maximum is
// raised by as much, its sum and, unless this is the first tile (behind `wait_output`), its output rescaled.
template <int D, class Wait, class Store>
__device__ __forceinline__ void softmax_tile(uint32_t (&x)[2][32], uint32_t (&w)[2][16], uint32_t o_at, const float4 *scale,
                                             const float4 &inverse, float factor, bool masked, int left, bool first, RowState &r,
                                             Wait wait_output, Store store) {
    const float base = kHeadroom - r.top;
#pragma unroll
    for (int c = 0; c < 2; ++c) {
        const float4 z = scale[c];                                // of two blocks
        if (c == 1) ld_wait(x[1]);
#pragma unroll
        for (int k = 0; k < 32; k += 2) {
            const float a = factor * (k < 16 ? z.x : z.z), d = (k < 16 ? z.y : z.w) + base;
            float e0, e1;
            unpair(fma2(pair(__uint_as_float(x[c][k]), __uint_as_float(x[c][k + 1])), pair(a, a), pair(d, d)), e0, e1);
            x[c][k] = __float_as_uint(e0);
            x[c][k + 1] = __float_as_uint(e1);
        }
    }
    if (masked) {
#pragma unroll
        for (int k = 0; k < kTile; ++k)
            if (k >= left) x[k / 32][k % 32] = 0xff800000u;
    }
    float high[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        high[i] = __uint_as_float(x[i / 2][i % 2 * 16]);
#pragma unroll
        for (int k = 1; k < 15; k += 2) high[i] = max3(high[i], __uint_as_float(x[i / 2][i % 2 * 16 + k]), __uint_as_float(x[i / 2][i % 2 * 16 + k + 1]));
        high[i] = fmaxf(high[i], __uint_as_float(x[i / 2][i % 2 * 16 + 15]));
    }
    const float most = fmaxf(max3(high[0], high[1], high[2]), high[3]);
    if (__any_sync(~0u, most > r.limit)) {
        const bool raise = most > r.limit;
        const float by = raise ? most - kHeadroom : 0.f;
        const float f = !raise ? 1.f : r.limit == -INFINITY ? 0.f : exp2_fast(-by);
        r.top += by;
        r.sum *= f;
        if (raise) r.limit = kRaise + kHeadroom;
#pragma unroll
        for (int k = 0; k < kTile; ++k) x[k / 32][k % 32] = __float_as_uint(__uint_as_float(x[k / 32][k % 32]) - by);
        if (!first) {
            wait_output();
            fence_after();
#pragma unroll 1
            for (int c = 0; c < D / 8; ++c) {
                uint32_t y[8];
                tmem_ld(y, o_at + 8 * c);
                ld_wait(y);
#pragma unroll
                for (int k = 0; k < 8; ++k) y[k] = __float_as_uint(__uint_as_float(y[k]) * f);
                tmem_st8(o_at + 8 * c, y);
            }
        }
    }
#pragma unroll
    for (int c = 0; c < 2; ++c) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
            uint64_t part = 0;
#pragma unroll
            for (int k = 16 * b; k < 16 * b + 16; k += 2) {
                const float e0 = exp2_fast(__uint_as_float(x[c][k])), e1 = exp2_fast(__uint_as_float(x[c][k + 1]));
                part = add2(part, pair(e0, e1));
                w[c][k / 2] = pack_half(e0, e1);
            }
            float p0, p1;
            unpair(part, p0, p1);
            r.sum = fmaf(p0 + p1, c ? (b ? inverse.w : inverse.z) : (b ? inverse.y : inverse.x), r.sum);
        }
        store(c);
    }
}

// The warp's 32 query rows, rows first .. first + 31 of the request, to fp16 with a power of two per row,
// into rows at .. at + 31 of the swizzled tile: copied there as they are, each 16 bytes to the place that
// they will keep, then taken to fp16 in place, a row per lane. `row` points at this lane's row (null: none).
// Returns the factor that turns a product of this lane's row into a score.
template <int D>
__device__ __forceinline__ float load_queries(const QcacheAttentionParams &p, const uint16_t *row, unsigned char *tile, int at) {
    using C = Shape<D>;
    constexpr int kLanes = D / 8, kStep = 32 / kLanes;            // lanes to a row, rows of one copy
    const int lane = threadIdx.x % 32, sub = lane / kLanes, col = lane % kLanes;
    const uint32_t to = smem_u32(tile) + col / 8 * C::kQPanel + at * 128;
#pragma unroll 8
    for (int k = 0; k < 32 / kStep; ++k) {
        const int r = k * kStep + sub;
        const uint16_t *from = reinterpret_cast<const uint16_t *>(__shfl_sync(~0u, reinterpret_cast<uint64_t>(row), r));
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to + r * 128 + ((col % 8) ^ (r & 7)) * 16),
                     "l"(from ? from + col * 8 : p.q), "r"(from ? 16 : 0) : "memory");
    }
    asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
    __syncwarp();
    unsigned char *mine = tile + (at + lane) * 128;
    uint32_t m = 0;
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
        const uint4 x = *reinterpret_cast<const uint4 *>(mine + c / 8 * C::kQPanel + ((c % 8) ^ (lane & 7)) * 16);
        m = __vmaxu2(m, __vmaxu2(__vmaxu2(x.x & 0x7fff7fffu, x.y & 0x7fff7fffu), __vmaxu2(x.z & 0x7fff7fffu, x.w & 0x7fff7fffu)));
    }
    m = max(m & 0xffffu, m >> 16);
    const int e = max((int)(m >> 7) - 127, -100);
    // a negative softmax scale turns Q around, so that larger products are larger scores
    const float up = p.scale_log2 < 0.f ? -pow2f(14 - e) : pow2f(14 - e);
#pragma unroll
    for (int c = 0; c < D / 8; ++c) {
        uint4 *place = reinterpret_cast<uint4 *>(mine + c / 8 * C::kQPanel + ((c % 8) ^ (lane & 7)) * 16);
        uint4 x = *place;
        x.x = pack_half(__uint_as_float(x.x << 16) * up, __uint_as_float(x.x & 0xffff0000u) * up);
        x.y = pack_half(__uint_as_float(x.y << 16) * up, __uint_as_float(x.y & 0xffff0000u) * up);
        x.z = pack_half(__uint_as_float(x.z << 16) * up, __uint_as_float(x.z & 0xffff0000u) * up);
        x.w = pack_half(__uint_as_float(x.w << 16) * up, __uint_as_float(x.w & 0xffff0000u) * up);
        *place = x;
    }
    return fabsf(p.scale_log2) * pow2f(e - 14);
}

// The warp's 32 rows of 16-byte chunks, placed as load_queries places them, to their rows in global memory
// (`row`: this lane's; null: none).
template <int D>
__device__ __forceinline__ void store_rows(uint16_t *row, const unsigned char *tile) {
    using C = Shape<D>;
    constexpr int kLanes = D / 8, kStep = 32 / kLanes;            // lanes to a row, rows of one store
    const int lane = threadIdx.x % 32, sub = lane / kLanes, col = lane % kLanes;
#pragma unroll 8
    for (int k = 0; k < 32 / kStep; ++k) {
        const int r = k * kStep + sub;
        uint16_t *to = reinterpret_cast<uint16_t *>(__shfl_sync(~0u, reinterpret_cast<uint64_t>(row), r));
        const uint4 x = *reinterpret_cast<const uint4 *>(tile + col / 8 * C::kQPanel + r * 128 + ((col % 8) ^ (r & 7)) * 16);
        if (to) *reinterpret_cast<uint4 *>(to + col * 8) = x;
    }
    __syncwarp();
}

// ---------------------------------------------------------------- work

// kv tiles that row tile rt of a request may see (one at least: its rows are written).
template <int ROWS, int TILE>
__device__ __forceinline__ int visible_tiles(const QcacheAttentionParams &p, const RequestShape &s, int rt) {
    int limit = s.kv;
    if (p.causal) limit = min(limit, max(0, s.first + (min(s.rows, (rt + 1) * ROWS) - 1) / p.group + 1));
    return max(1, (limit + TILE - 1) / TILE);
}

struct Start {
    uint64_t u, end, per;
    int request, row_tile, head, at;
};

// The walk through a block's share, and the segment that it is at: each warp makes it for itself, in
// shared memory, so that neither takes registers from the loops.
template <int ROWS, int TILE, int SETUP>
struct Walk {
    AttentionSegment w;
    int at, left;                 // units: done of this (row tile, head), its setup first; of the share behind w
    bool more;

    __device__ void begin(const QcacheAttentionParams &p, const Start &start) {
        left = (int)(start.end > start.u ? start.end - start.u : 0);
        if (left == 0) return;
        w.request = start.request; w.head = start.head; w.row_tile = start.row_tile;
        at = start.at;
        w.unit0 = start.u - start.at + SETUP;
        request(p);
    }

    __device__ __forceinline__ void request(const QcacheAttentionParams &p) {
        const RequestShape s = request_shape<ROWS, TILE>(p, w.request);
        w.row0 = s.row0; w.first = s.first; w.kv = s.kv; w.rows = s.rows;
        w.tiles = visible_tiles<ROWS, TILE>(p, s, w.row_tile);
    }

    // The next segment with tiles into w, for the whole warp; false at the end.
    __device__ __forceinline__ bool next(const QcacheAttentionParams &p) {
        __syncwarp();
        if (threadIdx.x % 32 == 0) {
            more = false;
            while (left > 0 && !more) {
                if (at == w.tiles + SETUP) {
                    w.unit0 += w.tiles + SETUP;
                    at = 0;
                    if (++w.head == p.heads) {
                        w.head = 0;
                        if (++w.row_tile * ROWS >= w.rows) {
                            w.row_tile = 0;
                            do ++w.request, request(p); while (w.rows == 0);
                        } else {
                            request(p);
                        }
                    }
                }
                const int n = min(w.tiles + SETUP - at, left);
                w.t0 = max(0, at - SETUP);
                at += n;
                left -= n;
                w.t1 = max(0, at - SETUP);
                more = w.t1 > w.t0;
            }
        }
        __syncwarp();
        return more;
    }
};

// The parity of each of a few stages' barriers, flipped at every use. Stages are counted from the first tile
// of a segment: a loop whose counter starts at a constant keeps its addresses in uniform registers, which the
// tensor instructions want.
struct Parity {
    uint32_t bits = 0;
    __device__ __forceinline__ uint32_t peek(uint32_t stage) const { return bits >> stage & 1; }
    __device__ __forceinline__ uint32_t use(uint32_t stage) {
        const uint32_t p = bits >> stage & 1;
        bits ^= 1u << stage;
        return p;
    }
};

struct Barriers {
    // A step brings the K tile of the scores and the V tile of the weights, two tiles behind, in one stage.
    uint64_t kv_full[4], kv_empty[4];
    uint64_t entry_full[kEntryStages], entry_empty[2];   // tiles; half of the stages
    uint64_t q_full[2], o_full[2];
    uint64_t s_full[2][2], p_full[2][2];      // query tile, score buffer
    uint64_t o_done[2];                       // all but the segment's last tile is in the output
    uint64_t drained[2];                      // all that an issuing warp has issued is done
};

template <int D, int FORMAT>
__global__ void __launch_bounds__(kThreads, 1) prefill_kernel(const __grid_constant__ QcacheAttentionParams p) {
    using C = Shape<D>;
    extern __shared__ __align__(1024) unsigned char smem[];
    __shared__ Barriers bars;
    __shared__ Entries entries[kEntryStages];
    __shared__ uint32_t scan[kThreads / 32];
    __shared__ Start start;
    __shared__ Walk<C::kRows, kTile, C::kSetup> walks[kThreads / 32];
    __shared__ uint32_t tmem_base;
    __shared__ int failed;
    unsigned char *q_smem = smem, *k_smem = q_smem + C::kQBytes, *v_smem = k_smem + C::kStages * C::kKvBytes;
    const int tid = threadIdx.x, warp = tid / 32, lane = tid % 32;

    after_kernels_before();
    // the plan: one thread per request, prefix sums in the (still unused) tile memory
    uint32_t *prefix = reinterpret_cast<uint32_t *>(smem);
    uint32_t total = 0;
    for (int r0 = 0; r0 < p.requests; r0 += kThreads) {
        const int r = r0 + tid;
        uint32_t n = 0;
        if (r < p.requests) {
            const RequestShape s = request_shape<C::kRows, kTile>(p, r);
#pragma unroll 4
            for (int rt = 0; rt < s.row_tiles; ++rt) n += visible_tiles<C::kRows, kTile>(p, s, rt) + C::kSetup;
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
        for (int w = 0; w < kThreads / 32; ++w) {
            if (w < warp) before = add_units(before, scan[w]);
            total = add_units(total, scan[w]);
        }
        if (r < p.requests) prefix[r] = before + a - n;
        __syncthreads();
    }
    if (total >= kTooMany) total = 0;
    if (warp == kMmaWarp) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_base)), "n"(512) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
    }
    if (tid == 0) {
        for (int i = 0; i < C::kStages; ++i) {
            bar_init(&bars.kv_full[i], 2 * kLoadWarps);
            bar_init(&bars.kv_empty[i], C::kIssuers);
        }
        for (int i = 0; i < kEntryStages; ++i) bar_init(&bars.entry_full[i], 1);
        for (int i = 0; i < 2; ++i) {
            for (int j = 0; j < 2; ++j) {
                bar_init(&bars.s_full[i][j], 1);
                bar_init(&bars.p_full[i][j], 128);
            }
            bar_init(&bars.q_full[i], 128 + (p.withhold == kQcacheWithholdQueries && blockIdx.x == 0));   // one more never comes
            bar_init(&bars.o_full[i], 1);
            bar_init(&bars.o_done[i], 1);
            bar_init(&bars.drained[i], 1);
            bar_init(&bars.entry_empty[i], C::kIssuers);
        }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        failed = 0;
    }
    // after a wait that ran out the loads may come to a tile that was never looked up: it is one without blocks
    for (int i = tid; i < kEntryStages * kBlocks; i += kThreads) entries[i / kBlocks].offset[i % kBlocks] = -1;
    if (warp == 1) {
        // where the block's share begins: the request by halving, the row tile 32 at a time
        const uint64_t units = (uint64_t)total * (uint32_t)p.heads;
        Start s;
        s.per = units_per_block<C::kSetup>(units, gridDim.x);
        s.u = (uint64_t)blockIdx.x * s.per;
        s.end = min(s.u + s.per, units);
        s.request = s.row_tile = s.head = s.at = 0;
        if (s.u < s.end) {
            int lo = 0, hi = p.requests;
            while (hi - lo > 1) {
                const int mid = (lo + hi) >> 1;
                if ((uint64_t)prefix[mid] * (uint32_t)p.heads <= s.u) lo = mid; else hi = mid;
            }
            s.request = lo;
            const RequestShape q = request_shape<C::kRows, kTile>(p, lo);
            uint64_t in = s.u - (uint64_t)prefix[lo] * (uint32_t)p.heads;
            for (int rt = 0; rt < q.row_tiles; rt += 32) {
                const uint32_t n = visible_tiles<C::kRows, kTile>(p, q, min(rt + lane, q.row_tiles - 1)) + C::kSetup;
                uint64_t all = (uint64_t)n * (uint32_t)p.heads;       // of the row tiles so far
#pragma unroll
                for (int d = 1; d < 32; d *= 2) {
                    const uint64_t x = __shfl_up_sync(~0u, all, d);
                    if (lane >= d) all += x;
                }
                const unsigned behind = __ballot_sync(~0u, in < all);
                const int l = behind ? __ffs(behind) - 1 : 32;
                if (l < 32 && rt + l < q.row_tiles) {
                    const uint32_t n_l = __shfl_sync(~0u, n, l);
                    const uint64_t in_l = in - (__shfl_sync(~0u, all, l) - (uint64_t)n_l * (uint32_t)p.heads);
                    s.row_tile = rt + l;
                    s.head = (int)(in_l / n_l);
                    s.at = (int)(in_l - (uint64_t)s.head * n_l);
                    break;
                }
                in -= __shfl_sync(~0u, all, 31);
            }
        }
        if (lane == 0) start = s;
    }
    fence_before();
    __syncthreads();
    fence_after();
    const Waiter wait{&failed, p.error};
    // all 512 columns: they begin at 0, which is what the addresses below take them to do
    if (tmem_base != 0 && tid == 0) atomicOr(p.error, 1u);
    constexpr uint32_t tmem = 0;
    Walk<C::kRows, kTile, C::kSetup> &walk = walks[warp];
    const AttentionSegment &w = walk.w;
    if (lane == 0) walk.begin(p, start);

    if (C::kQTiles == 1 && warp >= 4 && warp < kSoftmaxWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kIdleRegs));
    } else if (warp < kSoftmaxWarps) {
        // ------------------------------------------------ softmax: one row per thread
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kSoftmaxRegs));
        const int qt = warp / 4, row = tid % 128;
        const uint32_t lanes = (uint32_t)(warp % 4 * 32) << 16;
        const uint32_t s_at = tmem + lanes + qt * 2 * kTile, o_at = tmem + lanes + C::kOColumn + qt * D;
        uint32_t n_tile = 0;          // kv tiles of the block so far
        uint32_t o_phase = 0, done = 0;
        Parity scored;
        while (walk.next(p)) {
            const int first = w.row_tile * C::kRows + qt * 128;   // of the tile, among the request's rows
            if (first >= w.rows) {
                // Counted on without waiting, n_tile may get a round and more ahead of the lookups, and the wait for the
                // entries below then end early, on the parity of the round before. They are there all the same once the tile's
                // scores are: the loads had them before the products could begin.
                n_tile += w.t1 - w.t0;
                continue;
            }
            const int n = first + row;
            const bool valid = n < w.rows;
            const int64_t token = w.row0 + n / p.group, head = (int64_t)w.head * p.group + n % p.group;
            const float factor = load_queries<D>(p, valid ? p.q + token * p.q_stride_row + head * p.q_stride_head : nullptr,
                                                 q_smem + qt * C::kPanels * C::kQPanel, warp % 4 * 32);
            fence_async_smem();
            bar_arrive(&bars.q_full[qt]);

            // a row that is not there sees everything, so that no tile is masked for its sake
            const int limit = !valid ? INT32_MAX : p.causal ? min(w.kv, max(0, w.first + (int)(token - w.row0) + 1)) : w.kv;
            const int least = __reduce_min_sync(~0u, limit);      // of the warp's rows
            RowState r{0.f, 0.f, -INFINITY};
            const int t0 = w.t0, t1 = w.t1;
            for (int t = t0; t < t1; ++t, ++n_tile) {
                const uint32_t buffer = (t - t0) & 1;
                wait.warp(&bars.entry_full[n_tile % kEntryStages], n_tile / kEntryStages & 1);
                wait.warp(&bars.s_full[qt][buffer], scored.use(buffer));
                fence_after();
                const Entries &entry = entries[n_tile % kEntryStages];
                const uint32_t tile = s_at + buffer * kTile;
                uint32_t x[2][32], y[2][16];
                tmem_ld(x[0], tile);
                ld_wait(x[0]);
                tmem_ld(x[1], tile + 32);                         // on its way while the first half is scaled
                softmax_tile<D>(x, y, o_at, reinterpret_cast<const float4 *>(entry.scale), *reinterpret_cast<const float4 *>(entry.v_inverse),
                                factor, (t + 1) * kTile > least, limit - t * kTile, t == t0, r,
                                // the tile before is in the output when the next tile's scores are there, which came after it
                                [&] {
                                    if (t + 1 < t1) wait.warp(&bars.s_full[qt][buffer ^ 1], scored.peek(buffer ^ 1));
                                    else wait.warp(&bars.o_done[qt], done);
                                },
                                // into columns whose scores have been read, the first half while the second is computed
                                [&](int c) { tmem_st16(tile + 16 * c, y[c]); });
                st_wait();
                fence_before();
                bar_arrive(&bars.p_full[qt][buffer]);
            }
            if (t1 - t0 > 1) done ^= 1;
            const float top = r.top, sum = r.sum;
            wait.warp(&bars.o_full[qt], o_phase);
            o_phase ^= 1;
            fence_after();
            const bool whole = w.t0 == 0 && w.t1 == w.tiles;
            const int64_t part = 2 * (int64_t)blockIdx.x + (w.t0 == 0);
            if (whole) {
                // through the query rows' places in shared memory, so that the warp stores whole rows
                const float scale = sum == 0.f ? 0.f : 1.f / sum;
                unsigned char *tile = q_smem + qt * C::kPanels * C::kQPanel + warp % 4 * 32 * 128;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t x[32];
                    tmem_ld(x, o_at + 32 * c);
                    ld_wait(x);
#pragma unroll
                    for (int k = 0; k < 4; ++k) {
                        uint32_t y[4];
#pragma unroll
                        for (int j = 0; j < 4; ++j)
                            y[j] = pack_bf16(__uint_as_float(x[8 * k + 2 * j]) * scale, __uint_as_float(x[8 * k + 2 * j + 1]) * scale);
                        const int chunk = 4 * c + k;
                        *reinterpret_cast<uint4 *>(tile + chunk / 8 * C::kQPanel + lane * 128 + ((chunk % 8) ^ (lane & 7)) * 16) =
                            make_uint4(y[0], y[1], y[2], y[3]);
                    }
                }
                __syncwarp();
                store_rows<D>(valid ? p.out + token * p.out_stride_row + head * p.out_stride_head : nullptr, tile);
            } else {
                // 4 columns of all rows after another: a warp's stores lie together
                float *to = p.part_o + (part * C::kRows * (D / 4) + qt * 128 + row) * 4;
#pragma unroll
                for (int c = 0; c < D / 32; ++c) {
                    uint32_t x[32];
                    tmem_ld(x, o_at + 32 * c);
                    ld_wait(x);
#pragma unroll
                    for (int k = 0; k < 32; k += 4)
                        __stcg(reinterpret_cast<uint4 *>(to + (8 * c + k / 4) * (C::kRows * 4)), make_uint4(x[k], x[k + 1], x[k + 2], x[k + 3]));
                }
            }
            if (valid && whole && p.lse) p.lse[token * ((int64_t)p.heads * p.group) + head] = log_sum(top, sum, kHeadroom);
            if (!whole)
                __stcg(reinterpret_cast<float2 *>(p.part_ml + (part * C::kRows + qt * 128 + row) * 2), make_float2(sum == 0.f ? -INFINITY : top, sum));
        }
    } else if (warp < kMmaWarp) {
        if constexpr (C::kLoadRegs < kLaunchRegs) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kLoadRegs));
        else asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(C::kLoadRegs));
        // ------------------------------------------------ K (the first four warps) and V tiles to fp16
        const bool is_v = warp >= kSoftmaxWarps + kLoadWarps;
        const int lt = tid % kLoadThreads;
        constexpr int kPerRow = D / 16;                           // 16-code chunks of a token
        constexpr int kRowStep = kLoadThreads / kPerRow;          // tokens between a thread's chunks: a multiple of 8
        const int row = lt / kPerRow, d = lt % kPerRow * 16;
        // the lanes of a store that are in odd panels take their second half first: no bank twice
        const bool swap = D > 64 && d / 64 % 2;
        const int at16 = d % 64 / 8 + swap;
        unsigned char *to0 = (is_v ? v_smem : k_smem) + d / 64 * C::kKvPanel + row * 128;
        unsigned char *to1 = to0 + ((at16 ^ 1) ^ (row & 7)) * 16;
        to0 += (at16 ^ (row & 7)) * 16;
        const uint8_t *codes = (is_v ? p.v : p.k) + (row % 16) * p.stride_token + d;
        uint32_t n_tile = 0;
        Parity freed;
        while (walk.next(p)) {
            const int tiles = w.t1 - w.t0;
            const uint8_t *head = codes + (int64_t)w.head * p.stride_head;
            // the segment's tile i; a token past the request's, or in a block that is not there, is zero
            auto fetch = [&](uint4 (&x)[C::kChunks], int i) {
                wait.warp(&bars.entry_full[(n_tile + i) % kEntryStages], (n_tile + i) / kEntryStages & 1);
                const int64_t *offset = entries[(n_tile + i) % kEntryStages].offset;
                const int left = w.kv - (w.t0 + i) * kTile;
#pragma unroll
                for (int c = 0; c < C::kChunks; ++c) {
                    const int r = row + c * kRowStep;
                    const int64_t at = offset[r / 16];
                    x[c] = make_uint4(0, 0, 0, 0);
                    if (at >= 0 && r < left) x[c] = load_codes(head + at + (kRowStep % 16 ? c % 2 * 8 * p.stride_token : 0));
                }
            };
            auto begin_step = [&](int step) {
                const uint32_t stage = step % C::kStages;
                wait.warp(&bars.kv_empty[stage], freed.use(stage) ^ 1);
                return stage;
            };
            auto end_step = [&](int step) {
                __syncwarp();
                if (lane == 0) bar_arrive(&bars.kv_full[step % C::kStages]);
            };
            auto empty_step = [&](int step) {                     // V has none in the first two steps, K in the last two
                begin_step(step);
                end_step(step);
            };
            auto convert = [&](uint4 (&x)[C::kChunks], int i) {
                const int to = begin_step(is_v ? i + 2 : i) * C::kKvBytes;
#pragma unroll
                for (int c = 0; c < C::kChunks; ++c) {
                    if (swap) x[c] = make_uint4(x[c].z, x[c].w, x[c].x, x[c].y);
                    uint4 y0, y1;
                    codes_to_half<FORMAT>(x[c].x, y0.x, y0.y);
                    codes_to_half<FORMAT>(x[c].y, y0.z, y0.w);
                    codes_to_half<FORMAT>(x[c].z, y1.x, y1.y);
                    codes_to_half<FORMAT>(x[c].w, y1.z, y1.w);
                    *reinterpret_cast<uint4 *>(to0 + to + c * kRowStep * 128) = y0;
                    *reinterpret_cast<uint4 *>(to1 + to + c * kRowStep * 128) = y1;
                }
                fence_async_smem();
                end_step(is_v ? i + 2 : i);
            };
            // a tile's codes are on their way while the one before is converted (at head_dim 256, with registers for one
            // tile, 2,048 tokens over 16,384 take 1,134 us instead of 1,059)
            uint4 x[C::kChunks], y[C::kChunks];
            fetch(x, 0);
            if (is_v) {
                empty_step(0);
                empty_step(1);
            }
            for (int i = 0; i < tiles; i += 2) {
                if (i + 1 < tiles) fetch(y, i + 1);
                convert(x, i);
                if (i + 1 == tiles) break;
                if (i + 2 < tiles) fetch(x, i + 2);
                convert(y, i + 1);
            }
            if (!is_v) {
                empty_step(tiles);
                empty_step(tiles + 1);
            }
            n_tile += tiles;
        }
        // no arrival of the tensor cores is under way when the block ends
        for (int stage = 0; stage < C::kStages; ++stage) wait.warp(&bars.kv_empty[stage], freed.use(stage) ^ 1);
    } else {
      asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(C::kIssueRegs));
      // ------------------------------------------------ the matrix instructions of query tiles Q0 .. Q1 - 1
      // (a whole warp goes through it, one of its threads issues)
      auto issue = [&](auto q0, auto q1) {
        constexpr int Q0 = decltype(q0)::value, Q1 = decltype(q1)::value;
        constexpr uint32_t s_instruction = instruction(128, kTile, false), o_instruction = instruction(128, D, true);
        const uint32_t q_at = smem_u32(q_smem), k_at = smem_u32(k_smem), v_at = smem_u32(v_smem);
        const uint32_t leader = elect();
        uint32_t n_tile = 0, segment[2] = {0, 0};                // segment: those with rows in the query tile
        Parity filled, weighted[2];
        bool split = false;
        while (__any_sync(~0u, walk.next(p))) {
            if (Q0 == 0 && w.t0 == 0 && w.t1 < w.tiles) {
                // the part that begins a range which the next blocks go on with: for the joining kernel
                split = true;
                if (leader)
                    p.splits[blockIdx.x] = {w.request, w.head, w.row_tile, w.row0, w.rows, (int)((w.unit0 + w.tiles - 1) / start.per)};
            }
            // votes, so that the branches are uniform
            const int tiles = w.t1 - w.t0;
            const bool both = C::kQTiles == 2 && __any_sync(~0u, w.rows - w.row_tile * C::kRows > 128);
#pragma unroll
            for (int qt = Q0; qt < Q1; ++qt)
                if (qt == 0 || both) wait.warp(&bars.q_full[qt], segment[qt]++ & 1);
            // Scores two tiles ahead of the products, one query tile after the other.
            for (int i = -2; __any_sync(~0u, i < tiles); ++i) {
                const uint32_t buffer = i & 1, stage = (i + 2) & (C::kStages - 1);
                const bool ahead = __any_sync(~0u, i + 2 < tiles);
                wait.warp(&bars.kv_full[stage], filled.use(stage));
                fence_after();
#pragma unroll
                for (int qt = Q0; qt < Q1; ++qt) {
                    if (qt == 1 && !both) break;
                    if (i >= 0) {
                        wait.warp(&bars.p_full[qt][buffer], weighted[qt].use(buffer));
                        fence_after();
                        const uint32_t a = (qt * 2 + buffer) * kTile, b = operand_lo(v_at + stage * C::kKvBytes, C::kKvPanel);
#pragma unroll
                        for (int j = 0; j < kTile / 16; ++j)
                            mma_ts(C::kOColumn + qt * D, a + j * 8, operand(b + j * 128), o_instruction, j > 0 || i > 0, leader);
                        if (!ahead) {
                            if (__any_sync(~0u, i + 2 == tiles)) commit(&bars.o_done[qt], leader);
                            else commit(&bars.o_full[qt], leader);
                        }
                    }
                    if (ahead) {
                        const uint32_t a = operand_lo(q_at + qt * C::kPanels * C::kQPanel, 16), b = operand_lo(k_at + stage * C::kKvBytes, 16);
#pragma unroll
                        for (int k = 0; k < D / 16; ++k)
                            mma_ss((qt * 2 + buffer) * kTile, operand(a + k / 4 * (C::kQPanel / 16) + k % 4 * 2),
                                   operand(b + k / 4 * (C::kKvPanel / 16) + k % 4 * 2), s_instruction, k > 0, leader);
                        commit(&bars.s_full[qt][buffer], leader);
                    }
                }
                commit(&bars.kv_empty[stage], leader);
                if (i >= 0) {
                    // these tiles' softmax threads have read the kv tile's entries, and so have the loads long before
                    if (n_tile % kEntryTiles == kEntryTiles - 1 && leader) bar_arrive(&bars.entry_empty[n_tile / kEntryTiles % 2]);
                    ++n_tile;
                }
            }
        }
        if (Q0 == 0 && !split && leader) p.splits[blockIdx.x].rows = 0;
        // whatever waits were passed over before, nothing is under way into this block's memory when it ends
        int late = 0;
        commit(&bars.drained[Q0], leader);
        if (!bar_try(&bars.drained[Q0], 0)) bar_wait_slow(&bars.drained[Q0], 0, &late, p.error);
        __syncwarp();
      };
      using First = std::integral_constant<int, 0>;
      using Second = std::integral_constant<int, 1>;
      using All = std::integral_constant<int, C::kQTiles>;
      if (warp == kEntryWarp) {
        // ------------------------------------------------ blocks and scales, kEntryTiles tiles at a time
        uint32_t n_tile = 0;
        const bool withheld = p.withhold == kQcacheWithholdEntries && blockIdx.x == 0;
        while (!withheld && walk.next(p)) {
            for (int t = w.t0; t < w.t1;) {
                // up to the next multiple of kEntryTiles of the count, so that the stages stay together
                const int n = min(w.t1 - t, (int)(kEntryTiles - n_tile % kEntryTiles));
                const int mine = lane / kBlocks, group = lane % kBlocks;
                const uint32_t half = n_tile / kEntryTiles % 2, slot = (n_tile + mine) % kEntryStages;
                // the first tile of a half of the stages waits for that half
                if (n_tile % kEntryTiles == 0) wait.warp(&bars.entry_empty[half], (n_tile / kEntryStages & 1) ^ 1);
                if (mine < n) {
                    const int64_t token = (int64_t)(t + mine) * kTile + group * 16;
                    const BlockEntry b = block_entry(p, w.request, w.head, token, w.kv);
                    // an absent block's tokens get weight 2^-inf
                    entries[slot].scale[group] = make_float2(b.k_scale, b.block < 0 ? -INFINITY : b.v_log2);
                    entries[slot].v_inverse[group] = b.v_inverse;
                    entries[slot].offset[group] = b.block < 0 ? -1 : (int64_t)b.block * p.stride_block +
                                                                         (token & ((1 << p.log2_block) - 1)) * p.stride_token;
                }
                __syncwarp();
                if (mine < n && group == 0) bar_arrive(&bars.entry_full[slot]);
                t += n;
                n_tile += n;
            }
        }
      } else if (warp == kMmaWarp) {
        if constexpr (C::kIssuers == 2) issue(First{}, Second{});
        else issue(First{}, All{});
      } else if (warp == kSecondMmaWarp) {
        if constexpr (C::kIssuers == 2) issue(Second{}, All{});
      }
    }
    fence_before();
    __syncthreads();
    fence_after();
    __syncwarp();
    if (warp == kMmaWarp)
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(512));
}

// The parts of ranges that were cut: a thread block for a sixteenth of a row tile, of the range that begins
// in block blockIdx.x of the kernel before. A thread has 4 columns of a row at a time, a warp those of 8 or
// 16 rows, whose parts lie together; the parts are weighed and added in the blocks' order. Bound by
// latency: the two reads and the launch. (Half as many rows, so twice the blocks: 1 us more where nothing
// was cut, 11.6 us for 64 tokens; twice as many: 2 us more for the head_dim 256 prompts.)
constexpr int kJoinThreads = 256, kJoinAhead = 4;   // parts that are read before they can be weighed

template <int D>
__global__ void __launch_bounds__(kJoinThreads) join_kernel(const __grid_constant__ QcacheAttentionParams p) {
    using C = Shape<D>;
    constexpr int kJoinRows = C::kRows / 16, kColumns = kJoinThreads / kJoinRows, kVecs = D / 4 > kColumns ? D / 4 / kColumns : 1;
    after_kernels_before();
    const QcacheSplit z = p.splits[blockIdx.x];
    const int row = blockIdx.y * kJoinRows + threadIdx.x % kJoinRows, column = threadIdx.x / kJoinRows;
    if (z.row_tile * C::kRows + row >= z.rows || column >= D / 4) return;
    const int n = z.last_block - (int)blockIdx.x + 1;
    auto part = [&](int c) { return (2 * (int64_t)(blockIdx.x + c) + (c == 0)) * C::kRows; };
    auto read_ml = [&](int c) { return __ldcg(reinterpret_cast<const float2 *>(p.part_ml + (part(c) + row) * 2)); };
    auto read = [&](int c, int v) {
        return __ldcg(reinterpret_cast<const float4 *>(p.part_o) + part(c) * (D / 4) + (int64_t)(column + v * kColumns) * C::kRows + row);
    };
    float2 ml[kJoinAhead];
    float4 x[kJoinAhead][kVecs], acc[kVecs];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int c = 0; c < kJoinAhead; ++c) {
        ml[c] = make_float2(-INFINITY, 0.f);
        if (c < n) {
            ml[c] = read_ml(c);
#pragma unroll
            for (int v = 0; v < kVecs; ++v) x[c][v] = read(c, v);
        }
    }
#pragma unroll
    for (int c = 0; c < kJoinAhead; ++c) m = fmaxf(m, ml[c].x);
#pragma unroll 4
    for (int c = kJoinAhead; c < n; ++c) m = fmaxf(m, read_ml(c).x);
#pragma unroll
    for (int v = 0; v < kVecs; ++v) acc[v] = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](const float2 &y, const float4 (&z)[kVecs]) {
        const float f = y.x == m ? 1.f : exp2_fast(y.x - m);
        l = fmaf(y.y, f, l);
#pragma unroll
        for (int v = 0; v < kVecs; ++v) {
            acc[v].x = fmaf(z[v].x, f, acc[v].x); acc[v].y = fmaf(z[v].y, f, acc[v].y);
            acc[v].z = fmaf(z[v].z, f, acc[v].z); acc[v].w = fmaf(z[v].w, f, acc[v].w);
        }
    };
#pragma unroll
    for (int c = 0; c < kJoinAhead; ++c)
        if (c < n) add(ml[c], x[c]);
#pragma unroll 4
    for (int c = kJoinAhead; c < n; ++c) {
        float4 y[kVecs];
#pragma unroll
        for (int v = 0; v < kVecs; ++v) y[v] = read(c, v);
        add(read_ml(c), y);
    }
    AttentionSegment w{};
    w.head = z.head;
    w.row0 = z.row0;
#pragma unroll
    for (int v = 0; v < kVecs; ++v) write_row(p, w, z.row_tile * C::kRows + row, (column + v * kColumns) * 4, acc[v], m, l, kHeadroom);
}

template <int D, int FORMAT>
cudaError_t launch(const QcacheAttentionParams &p, int num_sms, int device, cudaStream_t stream) {
    using C = Shape<D>;
    // more than half of an SM's shared memory: one block per SM, which holds all of its tensor memory
    const size_t smem = C::kSmem > 120 * 1024 ? C::kSmem : 120 * 1024;
    static std::atomic<uint64_t> allowed{0};   // devices on which the shared memory limit is raised
    if (device >= 64 || !(allowed.load() >> device & 1)) {
        const cudaError_t e = cudaFuncSetAttribute(prefill_kernel<D, FORMAT>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
        if (e != cudaSuccess) return e;
        if (device < 64) allowed.fetch_or(1ull << device);
    }
    const cudaError_t e = launch_behind(prefill_kernel<D, FORMAT>, dim3(num_sms), kThreads, smem, stream, p);
    return e != cudaSuccess ? e : launch_behind(join_kernel<D>, dim3(num_sms, 16), kJoinThreads, 0, stream, p);
}

}  // namespace

size_t qcache_prefill_part_rows(int head_dim) { return head_dim == 256 ? 128 : 256; }

cudaError_t launch_qcache_prefill(const QcacheAttentionParams &p, int num_sms, int device, cudaStream_t stream) {
#define CM_LAUNCH(D) \
    if (p.head_dim == D) \
        return p.format == CM_QCACHE_E4M3 ? launch<D, CM_QCACHE_E4M3>(p, num_sms, device, stream) \
                                          : launch<D, CM_QCACHE_INT8>(p, num_sms, device, stream);
    CM_LAUNCH(32) CM_LAUNCH(64) CM_LAUNCH(128) CM_LAUNCH(256)
#undef CM_LAUNCH
    return cudaErrorInvalidValue;
}

}  // namespace cm
