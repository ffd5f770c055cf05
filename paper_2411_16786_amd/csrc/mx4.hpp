// 4-bit weights (OCP MXFP4): element codes E2M1, two per byte with the even column in the low half, and one power-of-two scale
// byte (E8M0, 2^(byte - 127), 255 = NaN) per 32 columns of a row.  One instruction of gfx950 turns a byte of codes and a scale
// into two values; a code has two significant bits and the scale is a power of two, so the values are exact in bf16 as in
// float, and products on the matrix cores see the weights as they are.  (From 2^128 on they are infinite: codes of 4 and 6 under scale byte
// 253, of 2 and more under 254, which the quantisation here never writes.)
#pragma once
#include "common.hpp"

namespace dicemoe {

constexpr int kMxGroup = 32;                         // columns that share a scale

typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));
typedef float f32x2_t __attribute__((ext_vector_type(2)));

// The scale as the conversions take it: they read the exponent field alone, 0 as 2^-127 and 255 as NaN (checked for all 256 bytes).
__device__ __forceinline__ float mx4_scale(uint32_t byte) { return __uint_as_float(byte << 23); }

// the two values of byte B of `codes`: bf16 pair (even column in the low half) or two floats
template <int B>
__device__ __forceinline__ uint32_t mx4_bf16(uint32_t codes, float scale) {
    const bf16x2_t r = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, B);
    return __builtin_bit_cast(uint32_t, r);
}
template <int B>
__device__ __forceinline__ f32x2_t mx4_f32(uint32_t codes, float scale) {
    return __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, scale, B);
}

}  // namespace dicemoe
