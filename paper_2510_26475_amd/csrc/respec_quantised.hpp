// The cache of 8 bits: e4m3 numbers with one power of two for each token and KV head.
//
// With top = max |x| of a token's head the scale is the least power of two s = 2^e with top <= 448 s (448 is the largest e4m3 number), kept
// as the byte e + 127, and the codes are x / s rounded to nearest even.  A division by a power of two is exact, so the codes depend on
// the bits of x alone.  What a code stands for has four significant bits and is a multiple of 2^(byte - 136): a bf16 number exactly under bytes from 3
// on (the least bf16 number is 2^-133), a float under all of them; but codes past 240 under byte 247 (numbers from 31/32 of 2^128 on) are read as infinite.
// Against top / 448 itself the power of two costs nothing but range at the low end: e4m3 is a floating-point format, its relative step is the same
// everywhere above 2^-6.
#pragma once

#include <hip/hip_runtime.h>

#include <cstdint>

namespace respec {

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float floatx2_t __attribute__((ext_vector_type(2)));
typedef float floatx4_t __attribute__((ext_vector_type(4)));

// The byte of the scale of a head whose largest finite magnitude is `top`: the exponent of top less 8, one more where top's significand
// is past 1.75 = 448 / 256.
__device__ inline int scale_byte(float top) {
    const uint32_t bits = __float_as_uint(top);
    return max(1, (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0));
}
__device__ inline float scale_of(int byte) { return __uint_as_float((uint32_t)byte << 23); }
__device__ inline float inverse_of(int byte) { return __uint_as_float((uint32_t)(254 - byte) << 23); }  // (bytes 1 .. 247: never past a float)

// Four numbers, already divided by the scale, as codes.  What is not finite becomes NaN, which e4m3 has; infinities it has none.
__device__ inline uint32_t codes_of(const float (&x)[4]) {
    float y[4];
    for (int i = 0; i < 4; ++i) y[i] = fabsf(x[i]) < INFINITY ? x[i] : NAN;
    int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], w, true);
}

// What four codes stand for, as four bf16 numbers: exact for bytes from 3 on, rounded to nearest even under 1 and 2.
__device__ inline void values_of(uint32_t codes, float scale, uint32_t &lo, uint32_t &hi) {
    lo = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, false));
    hi = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(codes, scale, true));
}
// The same as four floats: exact under every byte.
__device__ inline floatx4_t floats_of(uint32_t codes, float scale) {
    const floatx2_t lo = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, false), hi = __builtin_amdgcn_cvt_scalef32_pk_f32_fp8(codes, scale, true);
    return floatx4_t{lo[0], lo[1], hi[0], hi[1]};
}

}  // namespace respec
