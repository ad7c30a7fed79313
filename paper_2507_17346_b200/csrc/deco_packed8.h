// The layout of activations kept in 8 bits, for the files that read or write it: a row of `cols` entries is
// ceil(cols / 32) blocks, each 32 signed bytes (0 beyond the row's end) and one exponent byte b;
// entry j stands for q_j 2^(b - 127), b = 255 for NaN.  (b = 0, which is never written, reads as a step of 0.)
#pragma once

#include <stdint.h>

namespace deco {

constexpr uint32_t BLOCK8 = 32;

// 2^(b - 127), or NaN, as bf16.
__device__ __forceinline__ uint32_t bf16_step(uint32_t b) { return b == 255u ? 0x7FC0u : b << 7; }

// Eight codes times their step (bf16, twice) as bf16.  A code's low seven bits in the place of a bf16 fraction with the exponent of
// 128 are 128 + those bits; its sign bit in the place of the lowest exponent bit makes 256 of 128: the
// difference is the code, exactly.
__device__ __forceinline__ uint4 converted(uint32_t c0, uint32_t c1, uint32_t step)
{
    uint32_t o[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const uint32_t p = __byte_perm(i < 2 ? c0 : c1, 0, i & 1 ? 0x4342 : 0x4140);
        const uint32_t a = (p & 0x007F007Fu) | 0x43004300u, b = (p & 0x00800080u) | 0x43004300u;
        uint32_t d;
        asm("sub.rn.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
        asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(o[i]) : "r"(d), "r"(step));
    }
    return make_uint4(o[0], o[1], o[2], o[3]);
}

}  // namespace deco
