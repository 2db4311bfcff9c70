// Device arithmetic of microscaled 4-bit floating point.
#ifndef IOLB_MX4_MATH_H
#define IOLB_MX4_MATH_H

#include "block.h"
#include "dense_math.h"

namespace iolb {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

constexpr int MX4_NAN = 255;                        // a block's scale where a value is not finite

// 2^(s - 127) for s from 0 to 254 (2^-127 is below the normal range).
__device__ __forceinline__ float mx4_unit(int s) { return __uint_as_float(s > 0 ? (unsigned)s << 23 : 0x400000u); }

// The scale of a block whose largest magnitude has these bits: the least s with magnitude <= 7 2^(s - 127), 7 = 1.75 2^2.  From a
// magnitude of 1.75 2^2 up the exponent field less 2, one more above it; fields below 2 and 3 end at 0.
__device__ __forceinline__ int mx4_scale(unsigned bits)
{
    if (bits >= 0x7f800000u) return MX4_NAN;
    const int s = (int)(bits >> 23) - 2 + ((bits & 0x7fffffu) > 0x600000u ? 1 : 0);
    return s < 0 ? 0 : s;
}

// Eight values in codes, the first in the lowest bits; nearest, ties to even, beyond 6 it is 6.
__device__ __forceinline__ unsigned mx4_codes(const float (&v)[8], float unit)
{
    unsigned w = 0;
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[0], v[1], unit, 0);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[2], v[3], unit, 1);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[4], v[5], unit, 2);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, v[6], v[7], unit, 3);
    return w;
}

__device__ __forceinline__ unsigned magnitude_bits(float v) { return __float_as_uint(v) & 0x7fffffffu; }

// The largest of four neighbouring lanes'.
__device__ __forceinline__ unsigned most_of_four(unsigned v)
{
    const unsigned a = (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0xb1, 0xf, 0xf, true);        // quad_perm [1,0,3,2]
    v = a > v ? a : v;
    const unsigned b = (unsigned)__builtin_amdgcn_mov_dpp((int)v, 0x4e, 0xf, 0xf, true);        // quad_perm [2,3,0,1]
    return b > v ? b : v;
}

// c += (rows of a) (rows of b)^T; a lane holds the 32 codes of one row in one block, and that block's scale in byte BYTE of its word.
// 16 rows, 128 k: row lane % 16, block lane / 16; element i of c is a's row 4 (lane / 16) + i, b's row lane % 16.
// 32 rows, 64 k: row lane % 32, block lane / 32; element i of c is a's row 8 (i / 4) + 4 (lane / 32) + i % 4, b's row lane % 32.
// Measured on registers alone, two waves to a SIMD, operands of zeros / of random bits: 16 rows 6.7 / 4.9 PFLOP/s (23 cycles an instruction: taking up the
// scales costs some seven beside 16 of product, 13 with one wave), 32 rows 9.5 / 6.4 (33 cycles, the product's 32; at random bits the card's power binds).
__device__ __forceinline__ i32x8 mx4_operand(const u32x4& a) { return i32x8{(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}; }

template <int BYTE>
__device__ __forceinline__ f32x4 mx4_multiply_16(const u32x4& a, unsigned a_scale, const u32x4& b, unsigned b_scale, const f32x4& c)
{
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(mx4_operand(a), mx4_operand(b), c, 4, 4, BYTE, (int)a_scale, BYTE, (int)b_scale);
}

template <int BYTE>
__device__ __forceinline__ f32x16 mx4_multiply_32(const u32x4& a, unsigned a_scale, const u32x4& b, unsigned b_scale, const f32x16& c)
{
    return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx4_operand(a), mx4_operand(b), c, 4, 4, BYTE, (int)a_scale, BYTE, (int)b_scale);
}

}  // namespace iolb

#endif
