// Rounding to 8-bit floats (OCP FP8 E4M3).
#pragma once

#include "gelo_internal.h"

namespace gelo {

// float -> E4M3 code (1 sign, 4 exponent bits with bias 7, 3 fraction bits; largest finite value 448 = 0x7E),
// round to nearest even, saturating, subnormals spaced 2^-9
__device__ __forceinline__ uint32_t e4m3_code(float t) {
    const uint32_t bits = __float_as_uint(t);
    const uint32_t sign = (bits >> 24) & 0x80u;
    const float a = fabsf(t);
    uint32_t code;
    if (a < 0.015625f) {                                     // below 2^-6: multiples of 2^-9; 8 of them is the first normal
        code = (uint32_t)rintf(a * 512.0f);
    } else {
        uint32_t m = __float_as_uint(a);
        m += 0x7FFFFu + ((m >> 20) & 1u);                    // round the 23-bit fraction to 3 bits, ties to even
        const uint32_t e = (m >> 23) - 120u;                 // rebias: 127 -> 7
        code = (e << 3) | ((m >> 20) & 7u);
        code = code > 0x7Eu ? 0x7Eu : code;                  // saturate at 448 (0x7F would be NaN)
    }
    return sign | code;
}

// How values of up to `top` are scaled to codes: times 448 / top, and back by top / 448 (1 where there are only zeros).  From 1.3e-36 down the
// first would be infinite; numbers of that size are scaled by 2^126, to at most 112.
struct E4m3Scale { float back, times; };
__device__ __forceinline__ E4m3Scale e4m3_scale(float top) {
    if (top == 0.f) return {1.f, 1.f};
    const float times = 448.0f / top;
    return times == __builtin_inff() ? E4m3Scale{0x1p-126f, 0x1p126f} : E4m3Scale{top / 448.0f, times};
}

}  // namespace gelo
