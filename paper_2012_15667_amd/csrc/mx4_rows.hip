// Products of two operands in microscaled 4-bit floating point on the matrix cores.
#include "mx4_math.h"

namespace iolb {

namespace {

// A wave takes 16 x 16 sums and reads both operands from the caches, 16 bytes a lane: a block of 32 codes.  The columns' operand comes first, so that a
// lane holds four neighbouring columns of one row.
template <int DT>
__global__ void __launch_bounds__(256)
mx4_wave_kernel(Mx4Product p, int tiles_m)
{
    const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4;
    const long long tile = (long long)blockIdx.x * 4 + (threadIdx.x >> 6);
    const int m0 = (int)(tile % tiles_m) * 16;
    const long long n0 = tile / tiles_m * 16;
    if (n0 >= p.N) return;
    // (rows beyond the operand are read from its last row: their sums are never stored)
    const int m = m0 + l16 < p.M ? m0 + l16 : p.M - 1;
    const long long n = n0 + l16 < p.N ? n0 + l16 : p.N - 1;
    const int steps = (p.K + MX4_WIDE - 1) / MX4_WIDE;
    const uint8_t *const a = p.a + m * (steps * 64LL) + grp * 16, *const b = p.b + n * (steps * 64LL) + grp * 16;
    const uint8_t *const sa = p.a_scales + m * (steps * 4LL), *const sb = p.b_scales + n * (steps * 4LL);
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int t = 0; t < steps; ++t) {
        const u32x4 u = *reinterpret_cast<const u32x4*>(a + t * 64LL), v = *reinterpret_cast<const u32x4*>(b + t * 64LL);
        const unsigned x = *reinterpret_cast<const unsigned*>(sa + t * 4LL) >> 8 * grp, y = *reinterpret_cast<const unsigned*>(sb + t * 4LL) >> 8 * grp;
        sum = mx4_multiply_16<0>(v, y, u, x, sum);
    }
    float bias[4];
    const int first = (int)n0 + 4 * grp;
    load_bias<DT>(p.f, first, bias);
    finish_four<DT>(p.f, m0 + l16, first, bias, sum);
}

}  // namespace

hipError_t launch_mx4_few(const Mx4Product& p, int dtype, hipStream_t st)
{
    const int tiles_m = (p.M + 15) / 16;
    const long long groups = ((long long)tiles_m * ((p.N + 15) / 16) + 3) / 4;
    if (groups * 256 > 0xffffffffLL) return hipErrorInvalidValue;
    if (dtype == IOLB_F32) mx4_wave_kernel<IOLB_F32><<<(unsigned)groups, 256, 0, st>>>(p, tiles_m);
    else if (dtype == IOLB_F16) mx4_wave_kernel<IOLB_F16><<<(unsigned)groups, 256, 0, st>>>(p, tiles_m);
    else mx4_wave_kernel<IOLB_BF16><<<(unsigned)groups, 256, 0, st>>>(p, tiles_m);
    return hipGetLastError();
}

}  // namespace iolb
