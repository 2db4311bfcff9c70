// Products of few rows with weights in microscaled 4-bit floating point: bound by reading the weights, or by the latency of the call.
#include "mx4_math.h"

namespace iolb {

namespace {

constexpr int WAVES = 8;

// The 32 values of a block as codes and scale, as mx4_pack has them; those from `have` on are zeros.
template <class T>
__device__ __forceinline__ unsigned block_codes(const T* x, int have, u32x4& codes)
{
    typedef typename Piece<T, 8>::type Eight;
    Eight v[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        if (have >= 8 * q + 8) {
            v[q] = *reinterpret_cast<const Eight*>(x + 8 * q);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[q][i] = 8 * q + i < have ? x[8 * q + i] : (T)0.f;
        }
    }
    if constexpr (sizeof(T) == 4) {
        unsigned most = 0;
#pragma unroll
        for (int i = 0; i < 32; ++i) {
            const unsigned b = magnitude_bits(v[i / 8][i % 8]);
            most = b > most ? b : most;
        }
        const int s = mx4_scale(most);
        const float unit = mx4_unit(s);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            float f[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) f[i] = v[q][i];
            codes[q] = s == MX4_NAN ? 0u : mx4_codes(f, unit);
        }
        return (unsigned)s;
    } else {
        // 16 bits: the largest magnitude by whole numbers, two at a time, and codes from the type itself
        typedef unsigned short Two __attribute__((ext_vector_type(2)));
        typedef T TwoT __attribute__((ext_vector_type(2)));
        Two most = {0, 0};
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const Two b = __builtin_bit_cast(Two, __builtin_bit_cast(u32x4, v[i / 4])[i % 4] & 0x7fff7fffu);
            most = __builtin_elementwise_max(most, b);
        }
        const unsigned short one = most[0] > most[1] ? most[0] : most[1];
        const int s = mx4_scale(magnitude_bits((float)__builtin_bit_cast(T, one)));
        const float unit = mx4_unit(s);
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            // (two values as a vector of the type: of an element of a vector a cast of bits would take the first)
            const TwoT t[4] = {{v[q][0], v[q][1]}, {v[q][2], v[q][3]}, {v[q][4], v[q][5]}, {v[q][6], v[q][7]}};
            unsigned w = 0;
            if constexpr (std::is_same<T, __bf16>::value) {
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, t[0], unit, 0);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, t[1], unit, 1);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, t[2], unit, 2);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(w, t[3], unit, 3);
            } else {
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, t[0], unit, 0);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, t[1], unit, 1);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, t[2], unit, 2);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f16(w, t[3], unit, 3);
            }
            codes[q] = s == MX4_NAN ? 0u : w;
        }
        return (unsigned)s;
    }
}

// A workgroup takes sixteen columns, its waves a share of the summed axis each, in turn steps of 128 k: the weights go from memory to the registers of
// the wave that multiplies them, four steps ahead, with MR times sixteen rows of x.  A lane holds a block of 32 of row lane % 16 of either operand.
// PACKED: x is in 4 bits already; a tensor's blocks are brought into them where they are multiplied, by every workgroup again, which a launch of its own
// would cost more than.  The columns' operand comes first, so that a lane holds four neighbouring columns of one row.
// A row's time is a trip to memory, x into 4 bits and the waves' exchange: 1 x 4096 -> 4096 bf16 6.9 us on the GPU, of which 1.6 for W's bytes.
// (x's next blocks on their way meanwhile: 64 x 4096 -> 4096 19.1 -> 20.4 us, and more registers.  What counts there is the lanes' 64 bytes each, far apart.)
template <int DT, bool PACKED, int MR>
__global__ void __launch_bounds__(64 * WAVES)
mx4_few_kernel(Mx4Product p)
{
    typedef typename DenseType<DT>::type T;
    __shared__ f32x4 part[MR][WAVES][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4, wave = threadIdx.x >> 6;
    // (rows beyond the operand are read from its last row: their sums are never stored)
    const int m0 = (int)blockIdx.y * (16 * MR);
    const long long n0 = (long long)blockIdx.x * 16, n = n0 + l16 < p.N ? n0 + l16 : p.N - 1;
    const int steps = (p.K + MX4_WIDE - 1) / MX4_WIDE;
    const uint8_t *const b = p.b + n * (steps * 64LL) + grp * 16, *const sb = p.b_scales + n * (steps * 4LL) + grp;
    const uint8_t *a[MR], *sa[MR];
    const T* x[MR];
#pragma unroll
    for (int r = 0; r < MR; ++r) {
        const int m = m0 + 16 * r + l16 < p.M ? m0 + 16 * r + l16 : p.M - 1;
        a[r] = p.a + m * (steps * 64LL) + grp * 16;
        sa[r] = p.a_scales + m * (steps * 4LL) + grp;
        x[r] = static_cast<const T*>(p.x) + m * p.ldx + grp * MX4_BLOCK;
    }
    f32x4 sum[MR];
#pragma unroll
    for (int r = 0; r < MR; ++r) sum[r] = f32x4{0.f, 0.f, 0.f, 0.f};
    constexpr int AHEAD = 4;
    u32x4 w[AHEAD];
    unsigned ws[AHEAD];
    const auto load = [&](int t, int i) {
        if (t < steps) {
            w[i] = *reinterpret_cast<const u32x4*>(b + t * 64LL);
            ws[i] = sb[t * 4LL];
        }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load(wave + i * WAVES, i);
    for (int t0 = wave; t0 < steps; t0 += AHEAD * WAVES) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int t = t0 + i * WAVES;
            if (t < steps) {
#pragma unroll
                for (int r = 0; r < MR; ++r) {
                    u32x4 v;
                    unsigned s;
                    if constexpr (PACKED) {
                        v = *reinterpret_cast<const u32x4*>(a[r] + t * 64LL);
                        s = sa[r][t * 4LL];
                    } else {
                        s = block_codes(x[r] + (long long)t * MX4_WIDE, p.K - t * MX4_WIDE - grp * MX4_BLOCK, v);
                    }
                    sum[r] = mx4_multiply_16<0>(w[i], ws[i], v, s, sum[r]);
                }
            }
            load(t + AHEAD * WAVES, i);
        }
    }
#pragma unroll
    for (int r = 0; r < MR; ++r) part[r][wave][lane] = sum[r];
    __syncthreads();
    // a wave joins and finishes sixteen rows
    if (wave >= MR) return;
    f32x4 all = part[wave][0][lane];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) all += part[wave][i][lane];
    float bias[4];
    const int first = (int)n0 + 4 * grp;
    load_bias<DT>(p.f, first, bias);
    finish_four<DT>(p.f, m0 + 16 * wave + l16, first, bias, all);
}

template <int DT, int MR>
void launch(const Mx4Product& p, hipStream_t st)
{
    const dim3 groups((unsigned)(((long long)p.N + 15) / 16), (unsigned)((p.M + 16 * MR - 1) / (16 * MR)));
    if (p.x) mx4_few_kernel<DT, false, MR><<<groups, 64 * WAVES, 0, st>>>(p);
    else mx4_few_kernel<DT, true, MR><<<groups, 64 * WAVES, 0, st>>>(p);
}

template <int DT>
void launch_rows(const Mx4Product& p, hipStream_t st)
{
    if (p.M <= 16) launch<DT, 1>(p, st);
    else if (p.M <= 32) launch<DT, 2>(p, st);
    else launch<DT, 4>(p, st);
}

}  // namespace

bool mx4_few_launchable(int N) { return ((long long)N + 15) / 16 * (64 * WAVES) <= 0xffffffffLL; }

hipError_t launch_mx4_few(const Mx4Product& p, int dtype, hipStream_t st)
{
    if (dtype == IOLB_F32) launch_rows<IOLB_F32>(p, st);
    else if (dtype == IOLB_F16) launch_rows<IOLB_F16>(p, st);
    else launch_rows<IOLB_BF16>(p, st);
    return hipGetLastError();
}

}  // namespace iolb
