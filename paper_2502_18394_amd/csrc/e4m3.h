// Numbers of 8 bits (e4m3: up to 448, spacing 2^-3 of the leading bit, subnormals down to 2^-9, NaN 0x7f and 0xff) with scales that are powers of two.
// gfx950 converts two at a time with the scale's exponent in the same instruction: encoding rounds x / scale to nearest even (non-finite x: NaN), decoding
// gives code * scale, exact as a bf16 number.
#pragma once
#include "common.h"

namespace spectre {

constexpr float kE4m3Most = 448.f;
constexpr float kMostScale = 0x1p120f;             // the largest bf16 number's
constexpr float kCut = 1.875f * 0x1p127f;          // 240 at that scale: the next code would be 2^128

// The smallest power of two s with x <= 448 s, from 2^-100 on; x finite, not negative: 448 = 1.75 * 2^8.
__device__ __forceinline__ float e4m3_scale(float x) {
    const uint32_t b = __float_as_uint(x);
    const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
    return __uint_as_float((uint32_t)(e < 27 ? 27 : e) << 23);
}

typedef short e4m3x4_t __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t e4m3_encode4(float a, float b, float c, float d, float scale) {
    e4m3x4_t w = {0, 0};
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, a, b, scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(w, c, d, scale, true);
    return __builtin_bit_cast(uint32_t, w);
}
__device__ __forceinline__ uint2 e4m3_encode8(const float (&x)[8], float scale) {
    return make_uint2(e4m3_encode4(x[0], x[1], x[2], x[3], scale), e4m3_encode4(x[4], x[5], x[6], x[7], scale));
}
// Codes of the scale `from` as codes of the larger scale `to`: exact but for subnormals.
__device__ __forceinline__ uint32_t e4m3_rescale4(uint32_t w, float from, float to) {
    const f32x2_t a = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, from, false), b = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(w, from, true);
    return e4m3_encode4(a.x, a.y, b.x, b.y, to);
}
// Eight codes as bf16 numbers.
__device__ __forceinline__ uint4 e4m3_decode8(uint32_t lo, uint32_t hi, float scale) {
    return make_uint4(__builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, scale, true)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, false)),
                      __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, scale, true)));
}
__device__ __forceinline__ float e4m3_decode1(uint32_t code, float scale) { return __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(code, scale, false)[0]; }

// The highest bit of each byte that is a NaN.
__device__ __forceinline__ uint32_t e4m3_nan_bits(uint32_t w) { return ((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }
// NaNs replaced by zeros.
__device__ __forceinline__ uint32_t e4m3_finite_only(uint32_t w) { return w & ~((e4m3_nan_bits(w) >> 7) * 0xffu); }

}  // namespace spectre
