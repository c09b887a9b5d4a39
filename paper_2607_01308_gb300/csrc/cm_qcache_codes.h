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

}  // namespace
}  // namespace cm
