// Keys and values of 4 bits: a block of 32 values of a head's row is codes - a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6 - times 2^(byte - 127), the
// block's scale byte (255: the block is NaN).  Codes go two to a byte, the value of even number in the lower half.
//
// A head's piece of a page, 17 / 32 of a byte for each of its values: the codes of its rows, then their scale bytes.  A wave reads 16 rows at a time
// with one load of codes, D / 8 bytes to a lane, and one or two of scales:
//   keys    row by row, D / 2 bytes of codes and D / 32 scale bytes to each.  Lane (g, c) of an attention kernel takes a quarter of row c.
//   values  four rows at a time.  Their codes: of each row the first D / 32 bytes, then of each the next D / 32, 16 times.  Their scale bytes: of each row that of
//           the first block, then of each that of the next.  Lane (g, c) has to have D / 16 components of each of the rows 4 g ... 4 g + 3: they lie side by side.
#pragma once

#include "gelo_internal.h"

namespace gelo {

__device__ __forceinline__ int fp4_scales_at(int d, int page_shift) { return (d / 2) << page_shift; }       // bytes of a piece before its scales

constexpr uint32_t kFp4MostScale = 125 + 127;                // bytes beyond it are not finite: 255, and 253 and 254, which are never written

// the float 2^(byte - 127); 255: what the conversions take for a NaN scale
__device__ __forceinline__ float fp4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// The two bfloat16 of byte B of `codes`, exact: the conversion looks at the scale's exponent only.
template <int B>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float scale) {
    typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
    const bf16x2_t x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B);
    return __builtin_bit_cast(uint32_t, x);
}

// v with its last bit set if it is not a float: towards zero, and then odd.  Compares with anything of fewer bits as v does, so codes made of it are those of v.
__device__ __forceinline__ float odd_float(double v) {
    const float f = (float)v;
    uint32_t u = __float_as_uint(f);
    if (fabs((double)f) > fabs(v)) --u;
    return __uint_as_float((double)f == v ? u : u | 1u);
}

// Scale byte of a block whose largest |value| is `top`: the least 2^e with top <= 7 2^e, so that no value is off by more than 2^e, half of the largest
// step; e from -110 on (products of such values stay normal floats; smaller blocks are off by 2^-111 at most) to 125 (6 2^125 is one; larger values become it).
__device__ __forceinline__ uint32_t fp4_scale_byte(float top) {
    const uint32_t u = __float_as_uint(top);
    const int e = (int)(u >> 23) - 127 - ((u & 0x7FFFFFu) > 0x600000u ? 1 : 2);
    return (uint32_t)(min(max(e, -110), 125) + 127);
}

// Codes of 8 values, to nearest, ties to the even code.
__device__ __forceinline__ uint32_t fp4_codes(const float (&v)[8], float scale) {
    uint32_t w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0, v[0], v[1], scale, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], scale, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], scale, 2);
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], scale, 3);
}

}  // namespace gelo
