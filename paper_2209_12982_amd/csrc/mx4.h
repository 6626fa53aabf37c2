// The 4-bit format of the decoder operators, on the device: 32 neighbours
// share a power of two 2^(s - 127), s one byte (255: not a number); a code is
// a sign bit over the magnitudes 0, 1/2, 1, 3/2, 2, 3, 4, 6.  A value has two
// significant bits, so it is exact in bf16, and a product of two bf16 numbers
// is exact in the fp32 accumulator of the matrix cores.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>
#include "winof4.h"

namespace mx4 {

typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(2))) _Float16 f16x2;
typedef __attribute__((ext_vector_type(8))) _Float16 f16x8;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(2))) uint32_t u32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int kGroup = 32;

// 2^(s - 127) as fp32; a quiet NaN for s = 255.
__device__ inline float scale_value(uint32_t s) {
    const uint32_t bits = s << 23;
    return __builtin_bit_cast(float, s == 255u ? 0x7fc00000u : (s == 0u ? 0x00400000u : bits));
}

// The value of the code in the low 4 bits, without its scale: x 2 is an integer.
__device__ inline float code_value(uint32_t c) {
    const uint32_t m = c & 7u;
    const float a = m < 4u ? 0.5f * (float)m : (m < 6u ? (float)(m - 2u) : (float)(2u * m - 8u));
    return (c & 8u) ? -a : a;
}

// Smallest e with amax <= 6 2^e, as the scale byte e + 127: amax = f 2^x with
// f in [1/2, 1), and 6 2^e = 3/4 2^(e + 3), so e = x - 3, or x - 2 if f > 3/4.
// 127 for amax = 0, 255 where amax is not finite.  Exponents that a byte does
// not hold (below 2^-127) give 0.
__device__ inline uint32_t scale_byte(float amax) {
    const uint32_t b = __builtin_bit_cast(uint32_t, amax) & 0x7fffffffu;
    if (b >= 0x7f800000u) return 255u;
    if (b == 0u) return 127u;
    // fp32: value = 1.m 2^(E - 127), so x = E - 126 and f > 3/4 is 1.m > 1.5
    const int e = (int)(b >> 23) - 126 - 3 + ((b & 0x7fffffu) > 0x400000u ? 1 : 0);
    return e < -127 ? 0u : (uint32_t)(e + 127);      // subnormals (E = 0) end here too
}

// The code of x 2^-e, nearest value, ties to the even code.
__device__ inline uint32_t encode(float x, float inv_scale) {
    const float v = x * inv_scale;
    const float a = __builtin_fabsf(v);
    const uint32_t m = (a > 0.25f) + (a >= 0.75f) + (a > 1.25f) + (a >= 1.75f) + (a > 2.5f) + (a >= 3.5f) + (a > 5.0f);
    return m | ((__builtin_bit_cast(uint32_t, x) >> 28) & 8u);
}

// 2^-(s - 127) for a scale byte below 255 (2^127 for s = 0).
__device__ inline float inverse_scale(uint32_t s) {
    return s >= 254u ? __builtin_bit_cast(float, s == 254u ? 0x00400000u : 0u)
                     : __builtin_bit_cast(float, (254u - s) << 23);
}

// Eight codes (one word) to bf16 with their scale, exactly: the converter reads
// only the exponent bits of its scale operand, so the byte shifted into place
// is 2^(s - 127) down to s = 0, and s = 255 gives NaN.
__device__ inline bf16x8 decode8(uint32_t word, float scale_bits) {
    const bf16x2 a = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale_bits, 0));
    const bf16x2 b = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale_bits, 1));
    const bf16x2 c = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale_bits, 2));
    const bf16x2 d = __builtin_bit_cast(bf16x2, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(word, scale_bits, 3));
    return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
// The same to fp16, exact while 2^(s - 127) lies between 2^-23 and 2^13.
__device__ inline f16x8 decode8_f16(uint32_t word, float scale_bits) {
    const f16x2 a = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale_bits, 0));
    const f16x2 b = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale_bits, 1));
    const f16x2 c = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale_bits, 2));
    const f16x2 d = __builtin_bit_cast(f16x2, __builtin_amdgcn_cvt_scalef32_pk_f16_fp4(word, scale_bits, 3));
    return f16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}
__device__ inline float scale_bits(uint32_t s) { return __builtin_bit_cast(float, s << 23); }

// Both halves (rows) of a wave beside each other: x of this lane's half-wave
// (row) and of the other one, in some order.
template <int ROWS> __device__ inline f32x2 swap_rows(float x) {
    const uint32_t a = __builtin_bit_cast(uint32_t, x);
    const auto s = ROWS == 2 ? __builtin_amdgcn_permlane32_swap(a, a, false, false)
                             : __builtin_amdgcn_permlane16_swap(a, a, false, false);
    const uint32_t u = s[0], v = s[1];      // scalars: a bit cast of a vector's element reads element 0
    return f32x2{__builtin_bit_cast(float, u), __builtin_bit_cast(float, v)};
}
// The largest of three; the compiler's own maximum first quiets operands that
// it does not know to be numbers, an instruction each.  A NaN loses.
__device__ inline float max3(float a, float b, float c) {
    float r;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(r) : "v"(a), "v"(b), "v"(c));
    return r;
}
// Maximum and sum over the four 16-lane rows of a wave, lane by lane.
__device__ inline float max_rows(float x) {
    const f32x2 a = swap_rows<2>(x);
    const f32x2 b = swap_rows<1>(max3(a[0], a[1], a[1]));
    return max3(b[0], b[1], b[1]);
}
__device__ inline float sum_rows(float x) {
    const f32x2 a = swap_rows<2>(x);
    const f32x2 b = swap_rows<1>(a[0] + a[1]);
    return b[0] + b[1];
}

// 16-bit floating types at the edges of a kernel.
template <int TYPE> struct Half;
template <> struct Half<WINO_BF16> {
    typedef __bf16 type;
};
template <> struct Half<WINO_FP16> {
    typedef _Float16 type;
};

}  // namespace mx4
