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
// A cluster of thread blocks has a request. Each block reads, at once, what the walk may ask of single
// elements (the probabilities of every drafted token at its parent) and walks for itself, so that blocks only meet
// where a whole row has to be summed: after a rejection, and at the end. Then each takes a share of the vocabulary,
// and the shares' sums are put into every block's shared memory. The last share's sums lead to the token: the block,
// its warp, and the element within the warp's piece, read once more.
#include "cm_tree_kernels.h"

#include <cooperative_groups.h>

namespace cm {
namespace {

namespace cg = cooperative_groups;

constexpr int kThreads = 512, kWarps = kThreads / 32;
constexpr int kMaxCluster = 8;
constexpr int kMaxVocab = 1 << 20;
constexpr int kMaxSteps = kMaxVocab / (32 * 4 * kWarps) + 1;   // of a warp, if one block has the whole row
constexpr double kUnit = 0x1p-42;

__device__ __forceinline__ float clean(float x) { return fminf(fmaxf(x, 0.f), 1.f); }      // a NaN becomes 0

template <int TYPE>
struct Row;
template <>
struct Row<CM_PROB_F32> {
    using Element = float;
    static constexpr int kVec = 4;
    static __device__ __forceinline__ float one(const float *p) { return clean(*p); }
    static __device__ __forceinline__ void vec(const float *p, float (&x)[4]) {
        const float4 v = *reinterpret_cast<const float4 *>(p);
        x[0] = clean(v.x); x[1] = clean(v.y); x[2] = clean(v.z); x[3] = clean(v.w);
    }
};
template <>
struct Row<CM_PROB_BF16> {
    using Element = uint16_t;
    static constexpr int kVec = 8;
    static __device__ __forceinline__ float one(const uint16_t *p) { return clean(__uint_as_float((uint32_t)*p << 16)); }
    static __device__ __forceinline__ void vec(const uint16_t *p, float (&x)[8]) {
        const uint4 v = *reinterpret_cast<const uint4 *>(p);
        const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = clean(__uint_as_float(w[i] << 16));
            x[2 * i + 1] = clean(__uint_as_float(w[i] & 0xffff0000u));
        }
    }
};

// The whole multiples of 2^-42 in x, 0 <= x <= 1, as hi * 2^21 + lo: additions that round towards zero leave
// floor(x * 2^21) in the low bits of 4 + x, then the same of what is left.
__device__ __forceinline__ void split(float x, uint32_t &hi, uint32_t &lo) {
    const float y = __fadd_rz(x, 4.f);
    hi = __float_as_uint(y) - 0x40800000u;
    const float rest = __fmul_rn(__fsub_rn(x, __fsub_rn(y, 4.f)), 0x1p21f);
    lo = __float_as_uint(__fadd_rz(rest, 4.f)) - 0x40800000u;
}
__device__ __forceinline__ uint64_t whole(float x) {
    uint32_t hi, lo;
    split(x, hi, lo);
    return ((uint64_t)hi << 21) + lo;
}

// Where the walk is, in shared memory.
struct Walk {
    int node, child;              // the row, and its next child (-1: none)
    int levels;                   // of z, with draft rows; tokens taken out, without
    int depth;                    // rows accepted so far, the first among them
    int64_t z;                    // in multiples of 2^-42
    bool ends;                    // no child is left: the next token is chosen here
};

template <int TYPE>
__global__ void __launch_bounds__(kThreads) verify_kernel(const __grid_constant__ TreeVerifyParams p) {
    using R = Row<TYPE>;
    using E = typename R::Element;
    constexpr int kVec = R::kVec;
    __shared__ int16_t parent[kTreeMaxNodes], walked[kTreeMaxNodes];
    __shared__ int32_t token[kTreeMaxNodes];
    __shared__ float target_at[kTreeMaxNodes], draft_at[kTreeMaxNodes], accept_at[kTreeMaxNodes];
    __shared__ float level[kTreeMaxNodes];              // z of each subtraction at this node
    __shared__ int32_t out[kTreeMaxNodes];              // tokens taken out, without draft rows
    __shared__ uint64_t warp_sum[kWarps], block_sum[2][kMaxCluster], step_sum[kMaxSteps];
    __shared__ Walk walk;
    cg::cluster_group cluster = cg::this_cluster();
    const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
    const int blocks = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), r = blockIdx.x / blocks;
    after_kernels_before();

    const RequestRows rows = request_rows(p.row_starts, r, p.total_rows);
    const int n = min(rows.n, p.max_nodes);
    const E *target = static_cast<const E *>(p.target) + rows.first * p.target_stride;
    const E *draft = p.draft ? static_cast<const E *>(p.draft) + rows.first * p.draft_stride : nullptr;
    if (n == 0) {
        if (rank == 0 && tid == 0) {
            p.kept[r] = 0;
            p.next_token[r] = -1;
        }
        return;
    }
    cluster.barrier_arrive();                   // waited for before the first write to another block's memory
    for (int i = tid; i < n; i += kThreads) {
        int a = p.parents[rows.first + i];
        const int t = p.tokens[rows.first + i];
        if (a < 0 || a >= i || t < 0 || t >= p.vocab) a = -1;
        parent[i] = (int16_t)a;
        token[i] = t;
        if (a >= 0) {
            target_at[i] = R::one(target + a * p.target_stride + t);
            draft_at[i] = draft ? R::one(draft + a * p.draft_stride + t) : 1.f;
            accept_at[i] = p.accept[rows.first + i];
        }
    }
    __syncthreads();
    if (warp == 0) {
        int child = -1;
        for (int base = 1; base < n && child < 0; base += 32) {
            const unsigned found = __ballot_sync(~0u, base + lane < n && parent[min(base + lane, n - 1)] == 0);
            if (found) child = base + __ffs(found) - 1;
        }
        if (lane == 0) {
            walk = {0, child, 0, 1, (int64_t)1 << 42, false};
            walked[0] = 0;
        }
        __syncwarp();
    }
    cluster.barrier_wait();

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
                return -1;
            };
            while (true) {
                const int c = w.child;
                if (c < 0) {
                    w.ends = true;
                    break;
                }
                float have = target_at[c];
                double bar;
                if (draft) {
                    const float q = draft_at[c], z = (float)((double)w.z * kUnit);
                    for (int k = 0; k < w.levels; ++k) have = fmaxf(__fsub_rn(have, __fmul_rn(q, level[k])), 0.f);
                    bar = __dmul_rn(__dmul_rn((double)accept_at[c], (double)q), (double)z);
                } else {
                    for (int k = 0; k < w.levels; ++k)
                        if (out[k] == token[c]) have = 0.f;
                    bar = __dmul_rn((double)accept_at[c], (double)w.z * kUnit);
                }
                if (bar < (double)have) {
                    if (lane == 0) walked[w.depth] = (int16_t)c;
                    w = {c, -1, 0, w.depth + 1, (int64_t)1 << 42, false};
                    w.child = next_child(c);
                    continue;
                }
                w.child = next_child(c);
                if (draft) {
                    if (lane == 0) level[w.levels] = (float)((double)w.z * kUnit);
                    ++w.levels;
                    w.ends = w.child < 0;
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
        int levels = walk.levels;
        // element e of the row is number e + skew of its vectors
        auto weights = [&](int at, float (&w)[kVec]) {
            const int e = at - skew;
            float q[kVec];
            if (wide && e >= 0 && e + kVec <= p.vocab) {
                R::vec(t_row + e, w);
                if (d_row && levels) R::vec(d_row + e, q);
            } else {
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    const bool there = e + k >= 0 && e + k < p.vocab;
                    w[k] = there ? R::one(t_row + e + k) : 0.f;
                    q[k] = there && d_row && levels ? R::one(d_row + e + k) : 0.f;
                }
            }
            if (d_row) {
                for (int l = 0; l < levels; ++l) {
                    const float z = level[l];
#pragma unroll
                    for (int k = 0; k < kVec; ++k) w[k] = fmaxf(__fsub_rn(w[k], __fmul_rn(q[k], z)), 0.f);
                }
            } else {
                for (int l = 0; l < levels; ++l)
#pragma unroll
                    for (int k = 0; k < kVec; ++k)
                        if (out[l] == e + k) w[k] = 0.f;
            }
        };
        auto vector_sum = [&](const float (&w)[kVec]) {
            uint32_t hi = 0, lo = 0;
#pragma unroll
            for (int k = 0; k < kVec; ++k) {
                uint32_t x, y;
                split(w[k], x, y);
                hi += x;
                lo += y;
            }
            return ((uint64_t)hi << 21) + lo;
        };
        uint64_t total, before;                 // of the whole row; of the blocks in front of this one
        auto sum_row = [&] {
            uint64_t sum = 0;
#pragma unroll 4
            for (int s = 0; s < warp_steps; ++s) {
                const int at = begin + (warp * warp_steps + s) * kStep + lane * kVec;
                if (at - skew >= p.vocab) break;
                float w[kVec];
                weights(at, w);
                sum += vector_sum(w);
            }
#pragma unroll
            for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
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
        sum_row();
        if (total == 0 && levels > 0) {
            // a rejection that leaves nothing is taken back; without draft rows, all of them
            levels = draft ? levels - 1 : 0;
            if (ends) sum_row();
            else if (tid == 0) walk.levels = levels;
        } else if (!ends && tid == 0) {
            walk.z = (int64_t)total;
        }
        if (!ends) {
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
        const double number = (double)fminf(fmaxf(p.sample[r], 0.f), 1.f) * 0x1p32;
        uint64_t point = __umul64hi(total, min((uint64_t)number, (uint64_t)0xffffffffu) << 32);
        if (total == 0 || point < before) return;
        point -= before;
        int piece = 0;
        while (piece < kWarps && point >= warp_sum[piece]) point -= warp_sum[piece++];
        if (piece == kWarps) return;            // another block's
        // its steps, shared by the block's warps
        const int piece_begin = begin + piece * warp_steps * kStep;
        for (int s = warp; s < warp_steps; s += kWarps) {
            float w[kVec];
            weights(piece_begin + s * kStep + lane * kVec, w);
            uint64_t sum = vector_sum(w);
#pragma unroll
            for (int d = 16; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
            if (lane == 0) step_sum[s] = sum;
        }
        __syncthreads();
        if (warp != 0) return;
        int s = 0;
        while (s < warp_steps - 1 && point >= step_sum[s]) point -= step_sum[s++];
        float w[kVec];
        const int at = piece_begin + s * kStep + lane * kVec;
        weights(at, w);
        const uint64_t mine = vector_sum(w);
        uint64_t upto = mine;
#pragma unroll
        for (int d = 1; d < 32; d *= 2) {
            const uint64_t x = __shfl_up_sync(~0u, upto, d);
            if (lane >= d) upto += x;
        }
        if (point < upto && point >= upto - mine) {
            point -= upto - mine;
            int k = 0;
#pragma unroll
            for (int i = 0; i < kVec - 1; ++i)
                if (k == i && point >= whole(w[i])) point -= whole(w[i]), ++k;
            p.next_token[r] = at - skew + k;
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
    config.stream = stream;
    config.attrs = attrs;
    config.numAttrs = 2;
    return cudaLaunchKernelEx(&config, verify_kernel<TYPE>, p);
}

}  // namespace

cudaError_t launch_tree_verify(const TreeVerifyParams &p, int num_sms, cudaStream_t stream) {
    (void)num_sms;
    int blocks = 1;
    while (blocks < kMaxCluster && p.vocab > 4096 * blocks) blocks *= 2;
    return p.type == CM_PROB_F32 ? launch<CM_PROB_F32>(p, blocks, stream) : launch<CM_PROB_BF16>(p, blocks, stream);
}

}  // namespace cm
