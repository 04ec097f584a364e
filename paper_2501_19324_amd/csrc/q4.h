// The 4-bit format of weights and cache entries, and the moves between it and bf16 that its kernels share.
//
// A group of 32 values along the contracted axis has one scale 2^(s - 127), a byte s; a value is a sign and one of 0, .5, 1, 1.5, 2,
// 3, 4, 6 (two exponent bits, one fraction bit).  The scale is the least power of two with max|x| <= 7 * 2^e: a maximum between
// 6 and 7 units saturates to 6, an error of at most half the top step, as everywhere else on the grid.  Scaling by a power of two is exact, so a
// code does not depend on the precision it is computed in, and a value has two significant bits: exact in bf16, an operand
// of the matrix instructions as it is.  s is kept within 2 .. 252: nothing that the grid holds then overflows or is subnormal.
// A group with a NaN or an infinity has s = 255 and codes 0; it reads as NaN.
#pragma once
#include "common.h"

#define Q4_NAN 255
typedef short s16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
// the same at any address of a bf16 or an fp32 value: the memory serves such loads and stores, across lines too
typedef u32x4_t u32x4_any_t __attribute__((aligned(2)));
typedef u32x2_t u32x2_any_t __attribute__((aligned(2)));
typedef f32x4_t f32x4_any_t __attribute__((aligned(4)));
template <int N> struct u32vec;
template <> struct u32vec<1> { typedef uint32_t type __attribute__((ext_vector_type(1))); };
template <> struct u32vec<2> { typedef u32x2_t type; };
template <> struct u32vec<4> { typedef u32x4_t type; };

// scale byte of a group whose largest magnitude is amax (amax finite): the fraction field of 1.75 is 0x600000, and adding 0x1FFFFF
// carries into the exponent exactly where the fraction is larger
__device__ __forceinline__ int q4_scale_byte(float amax) {
    const int s = (int)((__float_as_uint(amax) + 0x1FFFFFu) >> 23) - 2;
    return s < 2 ? 2 : s > 252 ? 252 : s;
}
__device__ __forceinline__ bool q4_finite(float x) { return (__float_as_uint(x) & 0x7F800000u) != 0x7F800000u; }

// Two values -> a byte, the first in the low half.  The conversion instruction rounds to nearest, ties to the even code, and saturates
// at 6 (a test compares it with the definition value by value).
__device__ __forceinline__ uint32_t q4_encode2(float a, float b, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(0u, a, b, scale, 0) & 0xFFu;
}

// Byte BYTE of `codes` -> its two values times the scale, as a pair of bf16 (exact).  The instruction takes nothing but the exponent
// field of `scale`; an exponent of 255 gives NaN.
template <int BYTE> __device__ __forceinline__ uint32_t q4_decode2(uint32_t codes, uint32_t scale_bits) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, __uint_as_float(scale_bits), BYTE));
}
// eight values of one dword, one scale
__device__ __forceinline__ u32x4_t q4_decode8(uint32_t codes, uint32_t scale_bits) {
    return u32x4_t{q4_decode2<0>(codes, scale_bits), q4_decode2<1>(codes, scale_bits), q4_decode2<2>(codes, scale_bits), q4_decode2<3>(codes, scale_bits)};
}
// byte t of a dword of scale bytes, at the exponent's place (the bits around it are not looked at)
template <int T> __device__ __forceinline__ uint32_t q4_scale_at(uint32_t bytes) {
    if constexpr (T == 3) return bytes >> 1;
    else return bytes << (23 - 8 * T);
}

__device__ __forceinline__ f32x4_t q4_mfma(u32x4_t a, u32x4_t b, f32x4_t c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0, 0, 0);
}

// An fp32 value as the sum of three bf16 numbers, exactly: 24 significant bits cut into 8 + 8 + 8 (cutting, not rounding, so that nothing
// overflows and the rest is exact).  An infinity or NaN is its first part.
__device__ __forceinline__ void q4_cut3(float x, uint32_t& a, uint32_t& b, uint32_t& c) {
    const uint32_t u = __float_as_uint(x);
    if (!q4_finite(x)) { a = (u & 0x007FFFFFu) ? 0x7FC0u : u >> 16; b = c = 0; return; }
    a = u >> 16;
    const float r = x - __uint_as_float(u & 0xFFFF0000u);
    const uint32_t v = __float_as_uint(r);
    b = v >> 16;
    c = __float_as_uint(r - __uint_as_float(v & 0xFFFF0000u)) >> 16;
}
// PLANES = 1: bf16 values as they are; 3: fp32 values in three parts.  Eight values to an operand per plane.
template <int PLANES> __device__ __forceinline__ void q4_operand(const float x[8], u32x4_t o[PLANES]) {
    if constexpr (PLANES == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) o[0][i] = (__float_as_uint(x[2 * i]) >> 16) | (__float_as_uint(x[2 * i + 1]) & 0xFFFF0000u);
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            uint32_t a0, b0, c0, a1, b1, c1;
            q4_cut3(x[2 * i], a0, b0, c0);
            q4_cut3(x[2 * i + 1], a1, b1, c1);
            o[0][i] = a0 | (a1 << 16);
            o[1][i] = b0 | (b1 << 16);
            o[2][i] = c0 | (c1 << 16);
        }
    }
}
// Where lanes of one wave exchange through LDS: its operations stay in the order of the program, whose order this keeps the compiler from
// changing (no instruction).
__device__ __forceinline__ void wave_order() {
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
}
// maximum over the 16 lanes of a row
__device__ __forceinline__ float row16_max(float v) {
    row16_moves([&](auto c) { v = fmaxf(v, __uint_as_float(dpp_move<decltype(c)::value>(__float_as_uint(v)))); });
    return v;
}
__device__ __forceinline__ float row16_sum(float v) {
    row16_moves([&](auto c) { v += __uint_as_float(dpp_move<decltype(c)::value>(__float_as_uint(v))); });
    return v;
}
__device__ __forceinline__ int row16_or(int v) {
    row16_moves([&](auto c) { v |= (int)dpp_move<decltype(c)::value>((uint32_t)v); });
    return v;
}
