// Norm of every head's row of q and k, and the rotation to its position, in one pass.
//
//   y = x * rsqrt(mean x^2 + eps) * w          (without a weight y = x)
//   a_j = position * theta^(-2j/d),  out_j = y_j cos a_j - y_{j+d/2} sin a_j,
//                                    out_{j+d/2} = y_{j+d/2} cos a_j + y_j sin a_j
// fp32 throughout, rounded once to bf16. Angles lose nothing at far positions: turns_j = 2^64 theta^(-2j/d) / 2 pi
// is a 64-bit whole number, position * turns_j modulo 2^64 is the angle's fraction of a turn, and its upper 32
// bits, within [-1, 1) half turns, go to sincospi.
//
// A thread has 8 elements of a row's lower half and their partners in the upper one (two 16-byte vectors), d / 16
// threads a row of a head. A thread block takes some tokens' rows of all heads, computes their d / 2 angles once, and
// has the next row's vectors on their way while it computes. Bound by HBM (2 bytes in, 2 out an element) and issue
// together for prompts (16,384 tokens of 40 heads of 128: 56.5 us, 5.9 TB/s, the issue slots 72 % busy), by latency for single
// tokens (48 of them: 2.3 us). Tried and no faster: a token's angles in registers for five of its heads (57.4 us), two-wide
// arithmetic with the sines negated beside them (58.8, shared memory 77 % busy), five blocks to an SM (59.9), streaming
// loads and stores (56.7).
#include "cm_tree_kernels.h"

namespace cm {
namespace {

constexpr int kThreads = 256;
constexpr int kBlocksPerSm = 4;

__device__ __forceinline__ float bf16_lo(uint32_t w) { return __uint_as_float(w << 16); }
__device__ __forceinline__ float bf16_hi(uint32_t w) { return __uint_as_float(w & 0xffff0000u); }
__device__ __forceinline__ uint32_t to_bf16(float lo, float hi) {
    uint32_t w;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(w) : "f"(hi), "f"(lo));
    return w;
}
__device__ __forceinline__ void unpack(const uint4 &v, float (&x)[8]) {
    x[0] = bf16_lo(v.x); x[1] = bf16_hi(v.x); x[2] = bf16_lo(v.y); x[3] = bf16_hi(v.y);
    x[4] = bf16_lo(v.z); x[5] = bf16_hi(v.z); x[6] = bf16_lo(v.w); x[7] = bf16_hi(v.w);
}
__device__ __forceinline__ uint4 pack(const float (&x)[8]) {
    return make_uint4(to_bf16(x[0], x[1]), to_bf16(x[2], x[3]), to_bf16(x[4], x[5]), to_bf16(x[6], x[7]));
}

constexpr uint32_t kLeastMean = (127 - 60) << 23, kLargestMean = (127 + 100) << 23;   // as bits

// x / sqrt(mean x^2 + eps) of a row whose mean, eps with it, is too small or too large for sums of its squares: these
// are taken of x times 2^80 or 2^-70. Small: eps and all elements are below 2^-25, their squares below 2^110, and at 2^-106 or more
// (bf16 ends at 2^-133). Large: squares to 2^116, of which those that vanish are below the mean's rounding. All lanes of the warp come here,
// `odd`: those whose row it is.
template <int D>
__device__ __forceinline__ void normed_far(float (&a)[8], float (&b)[8], float mean, float eps, bool odd) {
    const bool small = mean < 1.f;
    const float by = small ? 0x1p80f : 0x1p-70f;
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float x = a[i] * by, y = b[i] * by;
        sum = fmaf(x, x, fmaf(y, y, sum));
    }
#pragma unroll
    for (int d = D / 32; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
    if (!odd) return;
    const float scaled = sum * (1.f / D) + eps * by * by, root = scaled == 0.f ? 0.f : rsqrtf(scaled);
    // small elements are made larger, large ones meet a smaller factor: neither passes fp32's ends on the way
    const float first = small ? by : 1.f, second = small ? root : root * by;
#pragma unroll
    for (int i = 0; i < 8; ++i) a[i] = a[i] * first * second, b[i] = b[i] * first * second;
}

// D: head_dim. Tokens [blockIdx.x * tokens, + tokens).
template <int D>
__global__ void __launch_bounds__(kThreads, kBlocksPerSm) rotate_kernel(const __grid_constant__ RotateParams p, int tokens) {
    constexpr int kLanes = D / 16, kGroups = kThreads / kLanes;   // threads of a head's row; rows side by side
    extern __shared__ __align__(16) float angles[];               // [tokens][2][D / 2]: cosines, sines
    after_kernels_before();
    const int64_t row0 = (int64_t)blockIdx.x * tokens;
    const int n = (int)min((int64_t)tokens, p.rows - row0), heads = p.heads[0] + p.heads[1];
    const int lane = threadIdx.x % kLanes, group = threadIdx.x / kLanes;
    // items: tokens x heads, in that order; this thread's are group, group + kGroups, ...
    int token = group / heads, head = group - token * heads;
    uint4 lo = make_uint4(0, 0, 0, 0), hi = lo;
    auto load = [&](int t, int h) {
        if (t >= n) return;
        const int which = h >= p.heads[0];
        const uint16_t *x = p.in[which] + (row0 + t) * p.in_row[which] + (h - (which ? p.heads[0] : 0)) * p.in_head[which] + lane * 8;
        lo = *reinterpret_cast<const uint4 *>(x);
        hi = *reinterpret_cast<const uint4 *>(x + D / 2);
    };
    load(token, head);
    const bool norms = p.weight[0] || p.weight[1];
    uint4 wl[2], wh[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        wl[i] = wh[i] = make_uint4(0, 0, 0, 0);
        if (p.weight[i]) {
            wl[i] = *reinterpret_cast<const uint4 *>(p.weight[i] + lane * 8);
            wh[i] = *reinterpret_cast<const uint4 *>(p.weight[i] + D / 2 + lane * 8);
        }
    }
    for (int i = threadIdx.x; i < n * (D / 2); i += kThreads) {
        const int t = i / (D / 2), j = i % (D / 2);
        const uint64_t turn = (uint64_t)(int64_t)p.positions[row0 + t] * p.turns[j];
        float s, c;
        sincospif((float)(int32_t)(turn >> 32) * 0x1p-31f, &s, &c);
        angles[t * D + j] = c;
        angles[t * D + D / 2 + j] = s;
    }
    __syncthreads();
    // as many steps for every thread of the block: the sums below take whole warps
    for (int step = 0; step < n * heads; step += kGroups) {
        const int t = token, which = head >= p.heads[0], h = head - (which ? p.heads[0] : 0);
        float a[8], b[8];
        unpack(lo, a);
        unpack(hi, b);
        head += kGroups;
        while (head >= heads) head -= heads, ++token;
        load(token, head);
        if (norms) {
            float sum = 0.f;
#pragma unroll
            for (int i = 0; i < 8; ++i) sum = fmaf(a[i], a[i], fmaf(b[i], b[i], sum));
#pragma unroll
            for (int d = kLanes / 2; d; d /= 2) sum += __shfl_xor_sync(~0u, sum, d);
            const float mean = sum * (1.f / D) + p.eps;
            float f = rsqrtf(mean);
            // outside of [2^-60, 2^100] (or NaN): squares that fp32 does not hold
            const bool odd = p.weight[which] && __float_as_uint(mean) - kLeastMean > kLargestMean - kLeastMean;
            if (__any_sync(~0u, odd)) {
                normed_far<D>(a, b, mean, p.eps, odd);
                if (odd) f = 1.f;
            }
            if (p.weight[which]) {
                float wa[8], wb[8];
                unpack(which ? wl[1] : wl[0], wa);
                unpack(which ? wh[1] : wh[0], wb);
#pragma unroll
                for (int i = 0; i < 8; ++i) a[i] *= f * wa[i], b[i] *= f * wb[i];
            }
        }
        if (t >= n) break;                    // in the last step
        const float *cosine = angles + t * D + lane * 8, *sine = cosine + D / 2;
        float c[8], s[8], x[8], y[8];
#pragma unroll
        for (int i = 0; i < 8; i += 4) {
            const float4 u = *reinterpret_cast<const float4 *>(cosine + i), v = *reinterpret_cast<const float4 *>(sine + i);
            c[i] = u.x; c[i + 1] = u.y; c[i + 2] = u.z; c[i + 3] = u.w;
            s[i] = v.x; s[i + 1] = v.y; s[i + 2] = v.z; s[i + 3] = v.w;
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            x[i] = fmaf(a[i], c[i], -(b[i] * s[i]));
            y[i] = fmaf(b[i], c[i], a[i] * s[i]);
        }
        uint16_t *out = p.out[which] + (row0 + t) * p.out_row[which] + h * p.out_head[which] + lane * 8;
        *reinterpret_cast<uint4 *>(out) = pack(x);
        *reinterpret_cast<uint4 *>(out + D / 2) = pack(y);
    }
}

template <int D>
cudaError_t launch(const RotateParams &p, int num_sms, cudaStream_t stream) {
    // One token to a thread block while that leaves none waiting, then more, to eight (16,384 tokens of 40 heads of 128: one
    // 79.5 us, two 62, four and eight 56.5, sixteen 58; 48 tokens: one 2.3 us, four 4.0).
    int tokens = 1;
    while (tokens < 8 && p.rows > (int64_t)tokens * kBlocksPerSm * num_sms) tokens *= 2;
    const dim3 grid((unsigned)((p.rows + tokens - 1) / tokens));
    return launch_behind(rotate_kernel<D>, grid, kThreads, (size_t)tokens * D * 4, stream, p, tokens);
}

}  // namespace

cudaError_t launch_rotate(const RotateParams &p, int num_sms, cudaStream_t stream) {
    switch (p.head_dim) {
        case 16: return launch<16>(p, num_sms, stream);
        case 32: return launch<32>(p, num_sms, stream);
        case 64: return launch<64>(p, num_sms, stream);
        case 128: return launch<128>(p, num_sms, stream);
        case 256: return launch<256>(p, num_sms, stream);
        case 512: return launch<512>(p, num_sms, stream);
    }
    return cudaErrorInvalidValue;
}

}  // namespace cm
