// fp32 operands of large products in two fp16 parts, half the matrix work of three bf16 parts.
//
// A row (the summed axis lies along it) is scaled by the power of two that brings its largest finite value into [2^14, 2^15), and a
// scaled value is h + l, both fp16 rounded to nearest: held to 2^-22 of itself or, below 2^-17 of its row's largest value, to 2^-40 of that.  Three
// products are taken, l h, h l and h h; l l is below 2^-22 of the product.  Where every value is held to 2^-22 of itself that is a sum within 2^-20.4 of
// its sum of magnitudes, beside what fp32 sums are off by; so it is made everywhere:
//   A row of whose non-zero values more than one in 64 is below 2^-20 of its largest (of normal values, 3 in a million are) is uneven, and an operand
// with one sends the whole product to three bf16 parts.
//   What other rows' parts leave out of values beyond that is added up, `lost`, scaled, for each row.  A sum is off by at most a row's loss times the
// other row's largest value, below 2^15; the kernels that finish sums judge them by that, and take those that may be off by more than 2^-20 of themselves again as
// fp32 products (least_sum, dense_math.h).  Of sums of 9216 normal values that is one in ten million; where they are many, as in rows of W that read only
// such columns, a block of sums is left to three parts.
// Infinities and NaN as in dense.h: h is the value, l zero, h h comes last.
//
// One workgroup (or wave) reads a row twice, the second time from L2: bound by memory: 4096 x 9216 twice 136 us, of 128 for
// what it reads and writes.
#include "dense_math.h"
#include "kernels.h"

namespace iolb {

namespace {

__global__ void __launch_bounds__(64) dense_even_kernel(int* uneven) { if (threadIdx.x < 2) uneven[threadIdx.x] = 0; }

// THREADS (64 or 256) to a row.
template <int THREADS>
__global__ void __launch_bounds__(256)
dense_halves_kernel(DenseHalves first, DenseHalves second, int cols, long long pitch, int groups_first, int* uneven)
{
    constexpr int AT_ONCE = 256 / THREADS;
    __shared__ float most_of[4], lost_of[4];
    __shared__ int small_of[4], count_of[4];
    const bool is_second = (int)blockIdx.x >= groups_first;
    const DenseHalves g = is_second ? second : first;
    const int tid = threadIdx.x % THREADS, wave = threadIdx.x >> 6;
    const long long r = (long long)(blockIdx.x - (is_second ? groups_first : 0)) * AT_ONCE + threadIdx.x / THREADS;
    const bool live = r < g.rows;
    const float* const row = g.x + (live ? r : 0) * g.ld;
    float most = 0.f;
    if (live) {
        for (int c = tid * 8; c < cols; c += THREADS * 8) {
            float v[8];
            load_columns(row + c, cols - c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) most = fmaxf(most, finite_magnitude(v[i]));
        }
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
    if constexpr (THREADS == 256) {
        if ((threadIdx.x & 63) == 0) most_of[wave] = most;
        __syncthreads();
        most = fmaxf(fmaxf(most_of[0], most_of[1]), fmaxf(most_of[2], most_of[3]));
    }
    int top;                                        // most = f 2^top, f in [0.5, 1)
    (void)frexpf(most, &top);
    const int shift = most > 0.f ? 15 - top : 0;
    const float line = 0x1p-20f * ldexpf(most, shift);
    int small = 0, count = 0;
    float lost = 0.f;
    for (int c = live ? tid * 8 : (int)pitch; c < (int)pitch; c += THREADS * 8) {
        float v[8];
        load_columns(row + c, cols - c, v);
        u32x4 h, l;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unsigned hb[2], lb[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float x = v[2 * i + j], s = ldexpf(x, shift);
                const bool finite = fabsf(x) < __builtin_inff();
                const _Float16 hv = finite ? (_Float16)s : (_Float16)x;
                const float rest = s - (float)hv;
                const _Float16 lv = finite ? (_Float16)rest : (_Float16)0.f;
                const float left_out = fabsf(s) >= 0x1p-100f ? fabsf(rest - (float)lv) : 0x1p-100f;       // (below, s itself may be cut)
                lost += finite && x != 0.f && left_out > 0x1p-22f * fabsf(s) ? left_out : 0.f;
                count += x != 0.f;
                small += x != 0.f && fabsf(s) < line;
                hb[j] = __builtin_bit_cast(unsigned short, hv);
                lb[j] = __builtin_bit_cast(unsigned short, lv);
            }
            h[i] = hb[0] | hb[1] << 16;
            l[i] = lb[0] | lb[1] << 16;
        }
        *reinterpret_cast<u32x4*>(g.planes + r * pitch + c) = h;
        *reinterpret_cast<u32x4*>(g.planes + ((long long)g.rows + r) * pitch + c) = l;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) {
        small += __shfl_xor(small, d);
        count += __shfl_xor(count, d);
        lost += __shfl_xor(lost, d);
    }
    if constexpr (THREADS == 256) {
        if ((threadIdx.x & 63) == 0) { small_of[wave] = small; count_of[wave] = count; lost_of[wave] = lost; }
        __syncthreads();
        small = small_of[0] + small_of[1] + small_of[2] + small_of[3];
        count = count_of[0] + count_of[1] + count_of[2] + count_of[3];
        lost = (lost_of[0] + lost_of[1]) + (lost_of[2] + lost_of[3]);
    }
    if (live && tid == 0) {
        g.scales[r] = {-shift, count ? lost : -1.f};
        if (small > count / 64) *uneven = 1;                // (whoever writes it writes the same)
    }
}

}  // namespace

hipError_t launch_dense_halves(const DenseHalves& a, const DenseHalves& b, int cols, long long pitch, int* uneven, hipStream_t st)
{
    const bool workgroup = dense_halves_by_workgroup(a.rows, b.rows, cols);
    const int groups_a = workgroup ? a.rows : (a.rows + 3) / 4;
    const unsigned groups = (unsigned)dense_halves_groups(a.rows, b.rows, cols);
    dense_even_kernel<<<1, 64, 0, st>>>(uneven);
    if (workgroup) dense_halves_kernel<256><<<groups, 256, 0, st>>>(a, b, cols, pitch, groups_a, uneven);
    else dense_halves_kernel<64><<<groups, 256, 0, st>>>(a, b, cols, pitch, groups_a, uneven);
    return hipGetLastError();
}

}  // namespace iolb
