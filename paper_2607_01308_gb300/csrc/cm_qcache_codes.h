// The two 8-bit formats of the cache: codes to and from fp16 / fp32. A stored value is
// code * scale. Every code of either format is exact in fp16 (e4m3: 4 significant bits from
// 2^-9 to 448; int8: whole numbers to 127), so only the write rounds.
#pragma once

#include <cstdint>

#include <cuda_runtime.h>

namespace cm {
namespace {

__device__ __forceinline__ uint32_t prmt(uint32_t a, uint32_t b, uint32_t sel) { return __byte_perm(a, b, sel); }

// Four codes (bytes 0..3 of w) as two fp16 pairs.
template <int FORMAT>
__device__ __forceinline__ void codes_to_half(uint32_t w, uint32_t &lo, uint32_t &hi) {
    if constexpr (FORMAT == CM_QCACHE_E4M3) {
        asm("{\n.reg .b16 a, b;\nmov.b32 {a, b}, %2;\ncvt.rn.f16x2.e4m3x2 %0, a;\ncvt.rn.f16x2.e4m3x2 %1, b;\n}"
            : "=r"(lo), "=r"(hi) : "r"(w));
    } else {
        // 0x6400 + u is 1024 + u in fp16, u = code + 128 in 0..255: minus 1152 is exact
        const uint32_t u = w ^ 0x80808080u;
        const uint32_t bias = 0x64806480u;
        uint32_t a = prmt(u, 0x64646464u, 0x4140), b = prmt(u, 0x64646464u, 0x4342);
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(lo) : "r"(a), "r"(bias));
        asm("sub.rn.f16x2 %0, %1, %2;" : "=r"(hi) : "r"(b), "r"(bias));
    }
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

}  // namespace
}  // namespace cm
