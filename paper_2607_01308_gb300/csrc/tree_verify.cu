// Drafted tokens against the target's probabilities, from given random numbers.
//
// The walk begins at a request's first row. At row x: w = target[x], z = 1; the rows drafted behind it, in
// their order, are accepted where
//   u_c * q(t_c) * z < w(t_c),        q = draft[x]
// and the walk goes on there. One that is rejected leaves w = max(w - q z, 0) and z = sum w, unless that is 0.
// Without draft probabilities q is 1 at t_c: w(t_c) becomes 0 and z less by it. Where no row is left, the next
// token is the first whose cumulative w passes u_r * sum w. So the tokens that come out are distributed as the
// target's own.
//
// The result must not depend on the order of additions, or a number next to a border would choose by it. Elements
// are fp32, each operation rounded alone; a sum adds the whole multiples of 2^-42 that its elements reach, in 64-bit
// integers (up to 2^20 elements of at most 1: below 2^62), and is exact. Tests multiply in fp64.
//
// A cluster of thread blocks has a request. What the walk may ask of single elements (the probabilities of every
// drafted token at its parent) is read at once, and each block walks for itself, so that blocks only meet
// where a whole row has to be summed: after a rejection, and at the end. Then each takes a share of the vocabulary,
// and the shares' sums are put into every block's shared memory. The last share's sums lead to the token: the block,
// its warp's piece, and the element within it, read once more.
//
// While all requests sum their first rows, that takes as long as the rows take from HBM (and some eleven instructions an
// element just as long); then it is the chain of a walk with several rejections, 4 us for each, in which a thread's own chain
// through its share counts: two vectors at once take 5,900 cycles where one after the other takes 6,550. 64 trees over 152,000
// tokens, up to four rows to sum one after another, 42 us (1.2 pairs of rows a request are read: 92 MB); one such tree 18 us; 16 chains
// over 32,003 tokens without draft rows 7.3 us (7.6 with fp64 products for the children asked first: that pipe is slow).
// Tried and no faster: more vectors on their way; blocks of 512 threads, which leave less than a third of the requests
// room to walk (55 us).
#include "cm_tree_kernels.h"

#include <cooperative_groups.h>

namespace cm {
namespace {

namespace cg = cooperative_groups;

constexpr int kMaxCluster = 8;
constexpr int kMaxVocab = 1 << 20, kAlone = 4096;              // elements that one block takes alone
constexpr int kMaxSteps = kMaxVocab / (32 * 4 * 8 * kMaxCluster) + 1;   // of a warp, with eight of them to a block
static_assert(kAlone / (32 * 4 * 8) + 1 <= kMaxSteps, "a smaller cluster's warps have no more");
constexpr int kThreads = 256, kWarps = kThreads / 32;   // four blocks to an SM: 64 requests with a cluster of eight each are there at once
constexpr int kSlot = 2 * kThreads * 16;                // a vector of each row for every thread
constexpr double kUnit = 0x1p-42;

__device__ __forceinline__ float clean(float x) { return __saturatef(x); }      // to [0, 1], a NaN to 0

// max(w - q z, 0) of values in [0, 1], each operation rounded.
__device__ __forceinline__ float less(float w, float q, float z) {
    const float product = __fmul_rn(q, z);
    float rest;
    asm("sub.rn.sat.f32 %0, %1, %2;" : "=f"(rest) : "f"(w), "f"(product));
    return rest;
}

// u q < w without rounding, for q and w in [0, 1]. A product that rounds to another value than w is on the same side of
// it; else its rounding's error says. 2^60 keeps that error above the least fp32 value, unless w is 0.
__device__ __forceinline__ bool product_below(float u, float q, float w) {
    const float a = q * 0x1p60f, b = w * 0x1p60f, product = __fmul_rn(u, a);
    return product < b || (product == b && __fmaf_rn(u, a, -product) < 0.f) || (u < 0.f && q > 0.f);
}

template <int TYPE>
struct Row;
template <>
struct Row<CM_PROB_F32> {
    using Element = float;
    static constexpr int kVec = 4;            // elements of a vector
    static constexpr int kAtOnce = 2, kAhead = 2;   // vectors of each row that a thread takes at once, and of those on their way (32 KB of a block)
    static __device__ __forceinline__ float one(const float *p) { return clean(*p); }
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&x)[4]) {
        x[0] = clean(__uint_as_float(v.x)); x[1] = clean(__uint_as_float(v.y));
        x[2] = clean(__uint_as_float(v.z)); x[3] = clean(__uint_as_float(v.w));
    }
};
template <>
struct Row<CM_PROB_BF16> {
    using Element = uint16_t;
    static constexpr int kVec = 8, kAtOnce = 1, kAhead = 3;
    static __device__ __forceinline__ float one(const uint16_t *p) { return clean(__uint_as_float((uint32_t)*p << 16)); }
    static __device__ __forceinline__ void unpack(const uint4 &v, float (&x)[8]) {
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = clean(__uint_as_float(w[i] << 16));
            x[2 * i + 1] = clean(__uint_as_float(w[i] & 0xffff0000u));
        }
    }
};

// The whole multiples of 2^-42 in x, 0 <= x <= 1, are hi * 2^21 + lo: additions that round towards zero leave
// floor(x * 2^21) in the low bits of 4 + x, then the same of what is left. Both come with kBits of 4 on top, which a sum
// takes off at its end (modulo 2^32).
constexpr uint32_t kBits = 0x40800000u;
__device__ __forceinline__ void split(float x, uint32_t &hi, uint32_t &lo) {
    const float y = __fadd_rz(x, 4.f);
    hi = __float_as_uint(y);
    lo = __float_as_uint(__fmaf_rz(__fsub_rn(x, __fsub_rn(y, 4.f)), 0x1p21f, 4.f));
}
template <int N>
__device__ __forceinline__ uint64_t whole(const float (&x)[N]) {
    uint32_t hi = 0, lo = 0;
#pragma unroll
    for (int i = 0; i < N; ++i) {
        uint32_t a, b;
        split(x[i], a, b);
        hi += a;
        lo += b;
    }
    return ((uint64_t)(hi - N * kBits) << 21) + (lo - N * kBits);
}
__device__ __forceinline__ uint64_t whole(float x) {
    const float one[1] = {x};
    return whole(one);
}

// Sum over a warp's lanes of numbers below 2^59.
__device__ __forceinline__ uint64_t over_warp(uint64_t x) {
    constexpr uint32_t kLow = (1u << 27) - 1;
    const uint32_t a = __reduce_add_sync(~0u, (uint32_t)x & kLow), b = __reduce_add_sync(~0u, (uint32_t)(x >> 27) & kLow),
                   c = __reduce_add_sync(~0u, (uint32_t)(x >> 54));
    return a + ((uint64_t)b << 27) + ((uint64_t)c << 54);
}

// Two elements in a 64-bit register, for the two-wide instructions.
__device__ __forceinline__ uint64_t pair(float x, float y) {
    uint64_t v;
    asm("mov.b64 %0, {%1, %2};" : "=l"(v) : "f"(x), "f"(y));
    return v;
}
__device__ __forceinline__ void unpair(uint64_t v, float &x, float &y) { asm("mov.b64 {%0, %1}, %2;" : "=f"(x), "=f"(y) : "l"(v)); }

// less() of both, the factor negated.
__device__ __forceinline__ uint64_t less2(uint64_t w, uint64_t q, uint64_t minus_z) {
    uint64_t product, rest;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(product) : "l"(q), "l"(minus_z));
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(rest) : "l"(w), "l"(product));
    float a, b;
    unpair(rest, a, b);
    return pair(fmaxf(a, 0.f), fmaxf(b, 0.f));
}

// split() of both, added up.
__device__ __forceinline__ void split2(uint64_t x, uint32_t &hi, uint32_t &lo) {
    const uint64_t four = pair(4.f, 4.f), minus_four = pair(-4.f, -4.f), minus_one = pair(-1.f, -1.f), up = pair(0x1p21f, 0x1p21f);
    uint64_t y, t, rest, z;
    asm("add.rz.f32x2 %0, %1, %2;" : "=l"(y) : "l"(x), "l"(four));
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(t) : "l"(y), "l"(minus_four));
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(rest) : "l"(t), "l"(minus_one), "l"(x));
    asm("fma.rz.f32x2 %0, %1, %2, %3;" : "=l"(z) : "l"(rest), "l"(up), "l"(four));
    hi += (uint32_t)y + (uint32_t)(y >> 32);
    lo += (uint32_t)z + (uint32_t)(z >> 32);
}

__device__ __forceinline__ void copy16(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ uint4 load16(uint32_t from) {
    uint4 v;
    asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(from) : "memory");
    return v;
}

// A row and what the rejections at it leave of it.
template <int TYPE>
struct Rest {
    using E = typename Row<TYPE>::Element;
    static constexpr int kVec = Row<TYPE>::kVec;
    const E *target, *draft;      // draft may be null
    int vocab, levels;
    bool wide;                    // both rows begin alike within a vector
    const float *level;           // z of each rejection, with a draft
    const int32_t *out;           // tokens taken out, without

    // Elements e, e + 1, ... (0 outside the row) where speed does not count, and their sum.
    __device__ __forceinline__ uint64_t get(int e, float (&w)[kVec]) const {
        const bool drawn = draft && levels > 0;
        float q[kVec];
        if (wide && e >= 0 && e + kVec <= vocab) {
            Row<TYPE>::unpack(*reinterpret_cast<const uint4 *>(target + e), w);
            if (drawn) Row<TYPE>::unpack(*reinterpret_cast<const uint4 *>(draft + e), q);
        } else {
#pragma unroll
            for (int k = 0; k < kVec; ++k) {
                const bool there = e + k >= 0 && e + k < vocab;
                w[k] = there ? Row<TYPE>::one(target + e + k) : 0.f;
                q[k] = there && drawn ? Row<TYPE>::one(draft + e + k) : 0.f;
            }
        }
        for (int l = 0; l < levels; ++l)
#pragma unroll
            for (int k = 0; k < kVec; ++k) w[k] = drawn ? less(w[k], q[k], level[l]) : out[l] == e + k ? 0.f : w[k];
        return whole(w);
    }
};

// Where the walk is, in shared memory.
struct Walk {
    int node, child;              // the row, and its next child (kTreeMaxNodes: none)
    int levels;                   // of z, with draft rows; tokens taken out, without
    int depth;                    // rows accepted so far, the first among them
    int64_t z;                    // in multiples of 2^-42
    bool ends;                    // no child is left: the next token is chosen here
};

template <int TYPE>
__global__ void __launch_bounds__(kThreads, 4) verify_kernel(const __grid_constant__ TreeVerifyParams p) {
    using R = Row<TYPE>;
    using E = typename R::Element;
    constexpr int kVec = R::kVec, kAtOnce = R::kAtOnce, kAhead = R::kAhead, kRing = kAhead * kAtOnce * kSlot;
    extern __shared__ __align__(16) unsigned char copies[];   // [kAhead][kAtOnce][target, draft][thread] vectors
    const uint32_t ring = (uint32_t)__cvta_generic_to_shared(copies) + threadIdx.x * 16;
    __shared__ int16_t parent[kTreeMaxNodes], walked[kTreeMaxNodes];
    __shared__ int32_t token[kTreeMaxNodes];
    __shared__ float target_at[kTreeMaxNodes], draft_at[kTreeMaxNodes], accept_at[kTreeMaxNodes];
    __shared__ float level[kTreeMaxNodes];              // z of each subtraction at this node
    __shared__ int32_t first_child[kTreeMaxNodes];      // kTreeMaxNodes: none
    __shared__ bool accepted[kTreeMaxNodes];            // where nothing was rejected at its parent
    __shared__ int32_t out[kTreeMaxNodes];              // tokens taken out, without draft rows
    __shared__ uint64_t warp_sum[kWarps], block_sum[2][kMaxCluster], step_sum[kMaxSteps];
    __shared__ Walk walk;
    __shared__ RequestRows rows_here;
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), r = blockIdx.x / blocks;
    after_kernels_before();

    // The first block reads what the walk goes by and puts it into each block's memory: the blocks' barriers only meet if all
    // walk alike, whatever happens to the inputs meanwhile. (Every block reading for itself is no faster.)
    for (int i = tid; i < p.max_nodes; i += kThreads) first_child[i] = kTreeMaxNodes;
    cluster.barrier_arrive();                   // waited for before the first write to another block's memory
    RequestRows given{};
    if (rank == 0) given = request_rows(p.row_starts, r, p.total_rows);
    const int m = min(given.n, p.max_nodes);
    struct Node {
        int parent, token;
        float target, draft, accept;
    };
    auto read = [&](int i) {
        const int a = p.parents[given.first + i], t = p.tokens[given.first + i];
        if (a < 0 || a >= i || t < 0 || t >= p.vocab) return Node{-1, t, 0.f, 1.f, 0.f};
        return Node{a, t, R::one(static_cast<const E *>(p.target) + (given.first + a) * p.target_stride + t),
                    p.draft ? R::one(static_cast<const E *>(p.draft) + (given.first + a) * p.draft_stride + t) : 1.f, p.accept[given.first + i]};
    };
    auto put = [&](int i, const Node &x) {
        for (int b = 0; b < blocks; ++b) {
            cluster.map_shared_rank(parent, b)[i] = (int16_t)x.parent;
            cluster.map_shared_rank(token, b)[i] = x.token;
            cluster.map_shared_rank(target_at, b)[i] = x.target;
            cluster.map_shared_rank(draft_at, b)[i] = x.draft;
            cluster.map_shared_rank(accept_at, b)[i] = x.accept;
        }
    };
    Node mine{};
    if (tid < m) mine = read(tid);
    cluster.barrier_wait();
    if (tid < m) put(tid, mine);
    for (int i = tid + kThreads; i < m; i += kThreads) put(i, read(i));
    if (rank == 0 && tid < blocks) *cluster.map_shared_rank(&rows_here, tid) = given;
    const float sample = p.sample[r];
    cluster.sync();
    const RequestRows rows = rows_here;
    const int n = min(rows.n, p.max_nodes);
    if (n == 0) {
        if (rank == 0 && tid == 0) {
            p.kept[r] = 0;
            p.next_token[r] = -1;
        }
        return;
    }
    const E *target = static_cast<const E *>(p.target) + rows.first * p.target_stride;
    const E *draft = p.draft ? static_cast<const E *>(p.draft) + rows.first * p.draft_stride : nullptr;
    for (int i = tid; i < n; i += kThreads) {
        const int a = parent[i];
        if (a >= 0 && i < first_child[a]) atomicMin(&first_child[a], i);
        accepted[i] = product_below(accept_at[i], draft_at[i], target_at[i]);
    }
    if (tid == 0) walked[0] = 0;
    __syncthreads();
    if (tid == 0) walk = {0, first_child[0], 0, 1, (int64_t)1 << 42, false};
    __syncthreads();

    // The block's share of a row, and its warps' pieces of it, one behind the other, in steps of 32 vectors. (A row
    // may begin within a vector.)
    constexpr int kStep = 32 * kVec;
    const int warp_steps = ((p.vocab + kVec + kStep - 1) / kStep + blocks * kWarps - 1) / (blocks * kWarps);
    const int begin = rank * kWarps * warp_steps * kStep;      // counted from the row's first vector

    int pass = 0;
    while (true) {
        // ------------------------------------------------ the walk, by one warp of each block
        if (warp == 0) {
            Walk w = walk;
            auto next_child = [&](int after) {
                for (int base = after + 1; base < n; base += 32) {
                    const unsigned found = __ballot_sync(~0u, base + lane < n && parent[min(base + lane, n - 1)] == w.node);
                    if (found) return base + __ffs(found) - 1;
                }
                return kTreeMaxNodes;
            };
            while (true) {
                const int c = w.child;
                if (c == kTreeMaxNodes) {
                    w.ends = true;
                    break;
                }
                float have = target_at[c];
                bool yes;
                if (w.levels == 0) {
                    yes = accepted[c];          // z is 1
                } else if (draft) {
                    const float q = draft_at[c], z = (float)((double)w.z * kUnit);
                    for (int k = 0; k < w.levels; ++k) have = less(have, q, level[k]);
                    yes = __dmul_rn(__dmul_rn((double)accept_at[c], (double)q), (double)z) < (double)have;
                } else {
                    for (int k = 0; k < w.levels; ++k)
                        if (out[k] == token[c]) have = 0.f;
                    yes = __dmul_rn((double)accept_at[c], (double)w.z * kUnit) < (double)have;
                }
                if (yes) {
                    if (lane == 0) walked[w.depth] = (int16_t)c;
                    w = {c, first_child[c], 0, w.depth + 1, (int64_t)1 << 42, false};
                    continue;
                }
                w.child = next_child(c);
                if (draft) {
                    if (lane == 0) level[w.levels] = (float)((double)w.z * kUnit);
                    ++w.levels;
                    w.ends = w.child == kTreeMaxNodes;
                    break;                      // what is left of the row has to be summed
                }
                if (have > 0.f) {
                    if (lane == 0) out[w.levels] = token[c];
                    ++w.levels;
                    w.z -= (int64_t)whole(have);
                }
                __syncwarp();
            }
            __syncwarp();
            if (lane == 0) walk = w;
        }
        __syncthreads();
        const int node = walk.node;
        const bool ends = walk.ends;

        // ------------------------------------------------ sums of w over the block's share
        const E *t_row = target + node * p.target_stride, *d_row = draft ? draft + node * p.draft_stride : nullptr;
        const int skew = (int)((reinterpret_cast<uintptr_t>(t_row) / sizeof(E)) % kVec);
        const bool wide = !d_row || (int)((reinterpret_cast<uintptr_t>(d_row) / sizeof(E)) % kVec) == skew;
        Rest<TYPE> rest{t_row, d_row, p.vocab, walk.levels, wide, level, out};
        uint64_t total, before;                 // of the whole row; of the blocks in front of this one
        auto sum_row = [&] {
            // the warp's piece: from step s0 to s1 every lane's vector is within the row
            const int first = begin + warp * warp_steps * kStep - skew;
            const int s1 = wide ? min(warp_steps, max(p.vocab - first, 0) / kStep) : 0, s0 = min(first < 0 ? 1 : 0, s1);
            const bool drawn = d_row && rest.levels > 0;
            const E *t_at = t_row + first + lane * kVec, *d_at = drawn ? d_row + first + lane * kVec : t_at;
            const float minus_z = drawn ? -level[0] : 0.f;
            uint64_t sum = 0;
            uint32_t hi = 0, lo = 0;            // less kBits for each element, modulo 2^32
            // vectors on their way lie in shared memory, each for the thread that asked for it
            const int n = max(s1 - s0, 0);
            t_at += s0 * kStep;
            d_at += s0 * kStep;
            int asked = 0;
            uint32_t to = ring, from = ring;
            auto ask = [&] {
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
                    if (asked + j < n) {
                        copy16(to + j * kSlot, t_at + j * kStep);
                        if (drawn) copy16(to + j * kSlot + kThreads * 16, d_at + j * kStep);
                    }
                asked += kAtOnce;
                t_at += kAtOnce * kStep;
                d_at += kAtOnce * kStep;
                to = to == ring + kRing - kAtOnce * kSlot ? ring : to + kAtOnce * kSlot;
                asm volatile("cp.async.commit_group;" ::: "memory");
            };
            for (int i = 0; i < kAhead; ++i) ask();
            // the row's ends, or all of rows that do not begin alike
#pragma unroll 1
            for (int i = 0; i < s0 + warp_steps - s1; ++i) {
                const int e = first + (i < s0 ? i : s1 + i - s0) * kStep + lane * kVec;
                float w[kVec];
                if (e < p.vocab) sum += rest.get(e, w);
            }
            int taken = 0;
#pragma unroll 1
            for (; taken < n; taken += kAtOnce) {
                asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 1) : "memory");
                uint64_t x[kAtOnce][kVec / 2];
                float w[kAtOnce][kVec], q[kAtOnce][kVec];
                auto unpack = [&](int j, int row, float (&v)[kVec]) {   // zeros behind the last
                    R::unpack(taken + j < n ? load16(from + j * kSlot + row * kThreads * 16) : make_uint4(0, 0, 0, 0), v);
                };
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j) {
                    unpack(j, 0, w[j]);
#pragma unroll
                    for (int k = 0; k < kVec / 2; ++k) x[j][k] = pair(w[j][2 * k], w[j][2 * k + 1]);
                }
                if (drawn) {
#pragma unroll
                    for (int j = 0; j < kAtOnce; ++j) unpack(j, 1, q[j]);
                    float z = minus_z;
                    for (int l = 1;; ++l) {
#pragma unroll
                        for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                            for (int k = 0; k < kVec / 2; ++k) x[j][k] = less2(x[j][k], pair(q[j][2 * k], q[j][2 * k + 1]), pair(z, z));
                        if (l == rest.levels) break;
                        z = -level[l];
                    }
                }
                from = from == ring + kRing - kAtOnce * kSlot ? ring : from + kAtOnce * kSlot;
#pragma unroll
                for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                    for (int k = 0; k < kVec / 2; ++k) split2(x[j][k], hi, lo);
                ask();
            }
            const uint32_t elements = (uint32_t)(taken * kVec);
            sum += ((uint64_t)(hi - elements * kBits) << 21) + (lo - elements * kBits);
            // without draft rows the steps above have counted the tokens that are taken out
            if (!d_row)
                for (int l = 0; l < rest.levels; ++l) {
                    const int at = out[l] - first, step = at / kStep;
                    if (at >= 0 && step >= s0 && step < s1 && at % kStep / kVec == lane) sum -= whole(R::one(t_row + out[l]));
                }
            sum = over_warp(sum);
            if (lane == 0) warp_sum[warp] = sum;
            __syncthreads();
            if (tid < blocks) {
                uint64_t all = 0;
                for (int w = 0; w < kWarps; ++w) all += warp_sum[w];
                *cluster.map_shared_rank(&block_sum[pass & 1][rank], tid) = all;
            }
            cluster.sync();
            total = before = 0;
            for (int b = 0; b < blocks; ++b) {
                const uint64_t x = block_sum[pass & 1][b];
                if (b < rank) before += x;
                total += x;
            }
            ++pass;
        };
        bool taken_back = false;
        while (true) {
            sum_row();
            if (total != 0 || rest.levels == 0 || taken_back) break;
            // a rejection that leaves nothing is taken back; without draft rows, all of them
            rest.levels = draft ? rest.levels - 1 : 0;
            taken_back = true;
            if (!ends) break;
        }
        if (!ends) {
            if (tid == 0) {
                if (taken_back) walk.levels = rest.levels;
                else walk.z = (int64_t)total;
            }
            __syncwarp();
            continue;
        }

        // ------------------------------------------------ the next token
        if (rank == 0) {
            for (int i = tid; i < rows.n; i += kThreads) p.path[rows.first + i] = i < walk.depth ? walked[i] : -1;
            if (tid == 0) {
                p.kept[r] = walk.depth;
                if (total == 0) p.next_token[r] = -1;
            }
        }
        uint64_t point = __umul64hi(total, (uint64_t)__float2uint_rz(clean(sample) * 0x1p32f) << 32);
        if (total == 0 || point < before) return;
        point -= before;
        int piece = 0;
        uint64_t sums[kWarps];
#pragma unroll
        for (int i = 0; i < kWarps; ++i) sums[i] = warp_sum[i];
#pragma unroll
        for (int i = 0; i < kWarps; ++i)
            if (piece == i && point >= sums[i]) point -= sums[i], ++piece;
        if (piece == kWarps) return;            // another block's
        // its steps, shared by the block's warps
        const int first = begin + piece * warp_steps * kStep + lane * kVec - skew;   // this lane's
        float w[kVec];
        for (int s = warp; s < warp_steps; s += kWarps) {
            const int e = first + s * kStep;
            if (e >= 0 && e < p.vocab) {        // all of them on their way before the first is waited for
                asm volatile("prefetch.global.L1 [%0];" ::"l"(t_row + e));
                if (draft) asm volatile("prefetch.global.L1 [%0];" ::"l"(d_row + e));
            }
        }
        for (int s = warp; s < warp_steps; s += kWarps) {
            const uint64_t sum = over_warp(rest.get(first + s * kStep, w));
            if (lane == 0) step_sum[s] = sum;
        }
        __syncthreads();
        if (warp != 0) return;
        // the step, its lane, its element: where the sum passes the point
        auto scan = [&](uint64_t x) {
#pragma unroll
            for (int d = 1; d < 32; d *= 2) {
                const uint64_t y = __shfl_up_sync(~0u, x, d);
                if (lane >= d) x += y;
            }
            return x;
        };
        for (int s0 = 0; s0 < warp_steps; s0 += 32) {
            const uint64_t mine = s0 + lane < warp_steps ? step_sum[s0 + lane] : 0, upto = scan(mine);
            const unsigned passed = __ballot_sync(~0u, point < upto);
            if (!passed) {
                point -= __shfl_sync(~0u, upto, 31);
                continue;
            }
            const int l = __ffs(passed) - 1, e = first + (s0 + l) * kStep;
            point -= __shfl_sync(~0u, upto - mine, l);
            const uint64_t own = rest.get(e, w), all = scan(own);
            if (point < all && point >= all - own) {
                point -= all - own;
                int k = 0;
#pragma unroll
                for (int i = 0; i < kVec - 1; ++i)
                    if (k == i && point >= whole(w[i])) point -= whole(w[i]), ++k;
                p.next_token[r] = e + k;
            }
            return;
        }
        return;
    }
}

template <int TYPE>
cudaError_t launch(const TreeVerifyParams &p, int blocks, cudaStream_t stream) {
    cudaLaunchAttribute attrs[2];
    attrs[0].id = cudaLaunchAttributeClusterDimension;
    attrs[0].val.clusterDim = {(unsigned)blocks, 1, 1};
    attrs[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attrs[1].val.programmaticStreamSerializationAllowed = 1;
    cudaLaunchConfig_t config{};
    config.gridDim = dim3((unsigned)p.requests * blocks);
    config.blockDim = dim3(kThreads);
    config.dynamicSmemBytes = Row<TYPE>::kAhead * Row<TYPE>::kAtOnce * kSlot;
    config.stream = stream;
    config.attrs = attrs;
    config.numAttrs = 2;
    return cudaLaunchKernelEx(&config, verify_kernel<TYPE>, p);
}

}  // namespace

cudaError_t launch_tree_verify(const TreeVerifyParams &p, cudaStream_t stream) {
    int blocks = 1;
    while (blocks < kMaxCluster && p.vocab > kAlone * blocks) blocks *= 2;
    return p.type == CM_PROB_F32 ? launch<CM_PROB_F32>(p, blocks, stream) : launch<CM_PROB_BF16>(p, blocks, stream);
}

}  // namespace cm
