// Device arithmetic of microscaled 4-bit floating point.
#ifndef IOLB_MX4_MATH_H
#define IOLB_MX4_MATH_H

#include "block.h"
#include "dense_math.h"

namespace iolb {

typedef float f32x2 __attribute__((ext_vector_type(2)));
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

// c += (16 rows of a) (16 rows of b)^T over 128 k; a lane holds the 32 codes of row lane % 16 in block lane / 16, and that block's scale in byte
// A_BYTE / B_BYTE of its word.  Element i of c: a's row 4 (lane / 16) + i, b's row lane % 16.
template <int A_BYTE, int B_BYTE>
__device__ __forceinline__ f32x4 mx4_multiply(const u32x4& a, unsigned a_scale, const u32x4& b, unsigned b_scale, const f32x4& c)
{
    const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0}, y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], 0, 0, 0, 0};
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, A_BYTE, (int)a_scale, B_BYTE, (int)b_scale);
}

}  // namespace iolb

#endif
