// 8-bit rows with scales: groups of 32 consecutive channels share a scale
// 2^e; the codes are e4m3 (OCP, no infinities, largest 448) of value / 2^e.
//
// e is the smallest exponent >= -117 with max |v| / 2^e <= 448 over the
// group's finite values, so that no finite value saturates.  A power of two
// costs up to one bit of the 8-bit type's range (which has 18 octaves to
// spare) and makes the division and its inverse exact: the only rounding is
// the code's, half a step of 2^-3, and a value read back has four significant
// bits, which bf16 holds exactly.  -117 keeps the smallest code (2^-9) at
// f32's and bf16's smallest normal, 2^-126.  Infinities and NaN become NaN
// codes and do not touch their group's scale.
#pragma once

#include "common.h"

namespace pcpp {

constexpr int EIGHT_GROUP = 32;
constexpr int EIGHT_BIAS = 127;      // a scale byte holds e + 127
constexpr int EIGHT_MIN_EXP = -117;

__device__ __forceinline__ bool is_finite(float v) { return (__float_as_uint(v) & 0x7fffffffu) < 0x7f800000u; }

__device__ __forceinline__ float finite_abs(float v) { return is_finite(v) ? fabsf(v) : 0.f; }

// The scale byte of a group whose largest finite magnitude is `top`: 448 is
// 1.75 * 2^8, so the exponent is that of `top` less 8, one more when its
// mantissa is above 1.75.
__device__ __forceinline__ int eight_scale(float top) {
    const uint32_t b = __float_as_uint(top);
    const int e = (int)(b >> 23) - EIGHT_BIAS - 8 + ((b & 0x7fffffu) > 0x600000u);
    return max(e, EIGHT_MIN_EXP) + EIGHT_BIAS;
}

// 2^-e and 2^e of a scale byte.  Every byte of eight_scale, 10 .. 247, gives
// normal numbers.
__device__ __forceinline__ float eight_inverse(int scale) { return __uint_as_float((uint32_t)(254 - scale) << 23); }
__device__ __forceinline__ float eight_value(int scale) { return __uint_as_float((uint32_t)scale << 23); }

// v, a signalling NaN as a quiet one.
__device__ __forceinline__ float quieted(float v) { return __builtin_canonicalizef(v); }

// Four values, already divided by the scale, as four codes.
__device__ __forceinline__ uint32_t to_e4m3(float a, float b, float c, float d) {
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}

// v / 2^e, NaN for what is not finite.
__device__ __forceinline__ float eight_scaled(float v, float inverse) {
    return is_finite(v) ? v * inverse : __uint_as_float(0x7fc00000u);
}

__device__ __forceinline__ f32x4 from_e4m3(uint32_t w) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
    return f32x4{lo[0], lo[1], hi[0], hi[1]};
}

// The largest magnitude of eight values; quiet NaN among them may be passed over
// or come through.  (A signalling NaN, which no arithmetic leaves, would come
// through as a quiet one and hide a larger value: quieted() before.)
__device__ __forceinline__ float max_abs8(const float (&v)[8]) {
    float a, b;
    asm("v_max_f32 %0, |%1|, |%2|" : "=v"(a) : "v"(v[0]), "v"(v[1]));
    asm("v_max_f32 %0, |%1|, |%2|" : "=v"(b) : "v"(v[2]), "v"(v[3]));
    asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(a) : "v"(a), "v"(v[4]), "v"(v[5]));
    asm("v_max3_f32 %0, %1, |%2|, |%3|" : "=v"(b) : "v"(b), "v"(v[6]), "v"(v[7]));
    asm("v_max_f32 %0, %1, %2" : "=v"(a) : "v"(a), "v"(b));
    return a;
}

// The largest of the four neighbouring lanes' (4k .. 4k + 3), by quad
// permutations (lanes 1 0 3 2, then 2 3 0 1).
__device__ __forceinline__ float max_of_quad(float top) {
    top = fmaxf(top, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(top), 0xB1, 0xF, 0xF, true)));
    return fmaxf(top, __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(top), 0x4E, 0xF, 0xF, true)));
}

// Eight consecutive channels of a lane, its group being four neighbouring
// lanes (all of them here together): the codes, and the scale byte that all
// four share.  A group whose largest magnitude is finite has no infinities, and
// what NaN it has become NaN codes by themselves.
__device__ __forceinline__ u32x2 to_eight_bits(const float (&v)[8], int& scale) {
    float top = max_of_quad(max_abs8(v));
    if (is_finite(top)) {
        scale = eight_scale(top);
        const float inv = eight_inverse(scale);
        return u32x2{to_e4m3(v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv),
                     to_e4m3(v[4] * inv, v[5] * inv, v[6] * inv, v[7] * inv)};
    }
    top = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) top = fmaxf(top, finite_abs(v[i]));
    scale = eight_scale(max_of_quad(top));
    const float inv = eight_inverse(scale);
    float t[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = eight_scaled(v[i], inv);
    return u32x2{to_e4m3(t[0], t[1], t[2], t[3]), to_e4m3(t[4], t[5], t[6], t[7])};
}

}  // namespace pcpp
