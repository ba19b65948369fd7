// The 4-bit rows of the key/value cache: codes of sign, two exponent bits and one mantissa bit (0, 1/2, 1, 3/2, 2, 3,
// 4, 6), one power of two per 32 values as a biased exponent byte.
#pragma once
#include "mfma.h"

namespace mvla {

// Scale operand of the conversions from a word of exponent bytes: byte `blk` rotated to the exponent's place.  (The
// conversions read only the exponent bits of their scale operand: found by running all 256 bytes with and without the
// others set.)
__device__ __forceinline__ float fp4_scale(uint32_t bytes, int blk) {
    return __uint_as_float(__builtin_amdgcn_alignbit(bytes, bytes, 9 + 8 * blk));
}

// two values of byte SEL of a word of eight codes, the even one in the low half (exact: bf16 holds every level times
// every power)
template <int SEL>
__device__ __forceinline__ uint32_t fp4_pair(uint32_t codes, float scale) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL));
}

// the eight values of a word of codes
__device__ __forceinline__ uint4 fp4_values(uint32_t codes, float scale) {
    return make_uint4(fp4_pair<0>(codes, scale), fp4_pair<1>(codes, scale), fp4_pair<2>(codes, scale),
                      fp4_pair<3>(codes, scale));
}

// eight bf16 values (finite) as a word of codes, rounded to nearest, ties to the even code; from 7 * scale on in magnitude,
// which only the largest power meets, the largest level
__device__ __forceinline__ uint32_t fp4_codes(const uint4& x, float scale) {
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.x), scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.y), scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.z), scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, __builtin_bit_cast(bf16x2_t, x.w), scale, 3);
    return c;
}

// Exponent byte of a block whose largest magnitude has the bf16 bits `top` (sign off): the smallest power under which
// it stays below 7 (from 7 on, 6 would no longer be the nearest level), but none above FP4_LARGEST, whose levels are the
// last that all stay below 2^128; 255 where it is no finite number.
constexpr uint32_t FP4_LARGEST = 252;
__device__ __forceinline__ uint32_t fp4_exponent(uint32_t top) {
    if (top >= 0x7f80u) return 255u;
    const int e = (int)(top >> 7) - 2 + ((top & 0x7fu) >= 0x60u ? 1 : 0);
    return e < 0 ? 0u : min((uint32_t)e, FP4_LARGEST);
}

// whether a block of this power may hold what is no finite number
__device__ __forceinline__ bool fp4_unbounded(uint32_t power) { return power > FP4_LARGEST; }
// ... one of the four of a word of powers (low seven bits from 125 on carry into the top one, which has to be set already)
__device__ __forceinline__ bool fp4_some_unbounded(uint32_t powers) {
    return (((powers & 0x7f7f7f7fu) + 0x03030303u) & powers & 0x80808080u) != 0;
}

}  // namespace mvla
