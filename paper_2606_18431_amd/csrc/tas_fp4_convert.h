// tas_fp4_convert.h - between four bits and 16 (device code).
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "tas_step_matrix.h"

namespace tas_step_impl {
namespace {

// A scale's byte as the float 2^e that the conversions take (of its exponent bits: 255
// makes every element NaN, 0 is 2^-127; checked over all 256 bytes).
__device__ float scale_of(uint32_t byte) { return __builtin_bit_cast(float, byte << 23); }

template <int SEL>
__device__ vec2<__bf16> pair_of(uint32_t codes, float scale, __bf16) {
    return __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, SEL);
}
template <int SEL>
__device__ vec2<_Float16> pair_of(uint32_t codes, float scale, _Float16) {
    return __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(codes, scale, SEL);
}
// The eight elements of four bytes of codes.
template <typename T>
__device__ vec8<T> values_of(uint32_t codes, float scale) {
    const vec2<T> a = pair_of<0>(codes, scale, T()), b = pair_of<1>(codes, scale, T());
    const vec2<T> c = pair_of<2>(codes, scale, T()), d = pair_of<3>(codes, scale, T());
    return vec8<T>{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// The largest magnitude, as bits: they order as the values do, infinity and NaN last.
__device__ uint32_t magnitude(float x) { return __builtin_bit_cast(uint32_t, x) & 0x7fffffffu; }
__device__ uint32_t largest(const float (&x)[8]) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; e++) m = max(m, magnitude(x[e]));
    return m;
}
// The scale's byte for a block's largest magnitude, given as bits (of a number that is not
// negative). 7 * 2^e is 1.75 * 2^(e + 2), so adding
// a quarter to the mantissa carries into the exponent where it is reached.
template <typename T>
__device__ uint32_t scale_byte(uint32_t most) {
    constexpr bool F16 = __is_same(T, _Float16);
    constexpr int lo = 127 + (F16 ? -23 : -125), hi = 127 + (F16 ? 13 : 125);
    if (most >= 0x7f800000u) return 255;  // (a NaN's sign too)
    return (uint32_t)min(max((int)((most + 0x200000u) >> 23) - 2, lo), hi);
}
// Eight elements' codes. The conversion rounds to nearest, halves to the even code, and
// stops at the largest; what it does with NaN does not matter, whose blocks have codes of 0.
__device__ uint32_t codes_of(const float (&x)[8], uint32_t byte) {
    const float s = scale_of(byte);
    uint32_t c = 0;
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[0], x[1], s, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[2], x[3], s, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[4], x[5], s, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c, x[6], x[7], s, 3);
    return byte == 255 ? 0 : c;
}
// A double as a float on the same side of every border between two codes, and of every
// power of two times 7: rounded to odd (those have even mantissas).
__device__ float odd_float(double x) {
    const float f = (float)x;
    const double d = (double)f;
    uint32_t u = __builtin_bit_cast(uint32_t, f);
    if (d != x && x == x) {
        if (fabs(d) > fabs(x)) u--;
        u |= 1;
    }
    return __builtin_bit_cast(float, u);
}

}  // namespace
}  // namespace tas_step_impl
