// What stands around the dense layers of a residual block: norms with gate and residual scale and their gradients, dropout, and
// microscaled 4-bit floating point with its product.  What the kernels and the entry points share.
#ifndef IOLB_BLOCK_H
#define IOLB_BLOCK_H

#include "dense.h"

namespace iolb {

// Whether a streaming call goes past the caches (non-temporal loads and stores): where its tensors together, `bytes`, are more than half of the 256 MB
// before memory.  Smaller ones are faster through them, and so is whoever reads the result next.
inline bool past_caches(double bytes) { return bytes > 128e6; }

// ---- norms -----------------------------------------------------------------------------------------
// Rows are N values.  p = post(h);  x' = a x + g p, rounded to the type;  y = pre(x').
struct BlockNorm {
    const void *x, *h, *gate;               // h null: y = pre(x) alone
    const void *post_weight, *post_bias, *pre_weight, *pre_bias;
    void *out, *y;                          // x', y; either may be null
    long long ldx, ldh, ldo, ldy;
    int M, N;
    int post, pre;                          // IOLB_NORM_...
    int rows_per_group;                     // rows that share a row of the gate
    float scale, eps;
};
hipError_t launch_block_norm(const BlockNorm& p, int dtype, hipStream_t st);

// Gradients.  d = dout + (gradient of pre at x', of dy);  dx = a d;  dh = (gradient of post at h, of g d).
// Column sums over the rows of a gate's group, S1 = sum of d hat(h), S0 = sum of d, and over all rows T1 = sum of dy hat(x'),
// T0 = sum of dy, give what the weights and the gate get: dgate = wp S1 + bp S0, dwp = sum of g S1 over the groups,
// dbp = sum of g S0, dw = T1, db = T0.
struct BlockNormBackward {
    const void *dy, *dout, *x, *h, *gate;   // dy, dout: either may be null
    const void *post_weight, *post_bias, *pre_weight;
    void *dx, *dh;                          // dense; null: not wanted
    void *dgate, *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;
    long long lddy, lddout, ldx, ldh;
    int M, N;
    int post, pre;
    int rows_per_group, groups;
    float scale, eps;
    float* rows;                            // [M][NORM_ROW_SUMS]: what the rows' pass leaves for the columns' pass
    float* columns;                         // [pieces][NORM_COLUMN_SUMS][N rounded up to 8]
};
constexpr int NORM_ROW_SUMS = 8, NORM_COLUMN_SUMS = 4;
// How the column sums are shared: `per` rows to a piece, no piece across two groups.
struct NormPieces { int per, in_group; };
struct NormBackwardPlan { NormPieces pieces; size_t row_bytes, column_bytes; bool launchable = true; };
NormBackwardPlan block_norm_backward_plan(const BlockNormBackward& p, int dtype);
hipError_t launch_block_norm_backward(const BlockNormBackward& p, const NormBackwardPlan& plan, int dtype, hipStream_t st);

// ---- dropout ---------------------------------------------------------------------------------------
struct Dropout {
    const void *x, *residual;               // residual may be null
    void* y;
    int8_t* zq;                             // checkpoint of y, or null
    uint8_t* ze;
    long long ldx, ldr, ldy;
    int rows, cols;
    unsigned least;                         // a value stays where its 16 random bits are at least this
    float scale;
    unsigned long long seed, offset;
    const unsigned long long* counter;      // on the device: [0] is added to the seed, [1] to the offset; may be null
};
hipError_t launch_dropout(const Dropout& p, int dtype, hipStream_t st);

// ---- microscaled 4-bit floating point ----------------------------------------------------------------
constexpr int MX4_BLOCK = 32, MX4_WIDE = 128;       // values that share a scale; columns that rows are padded to
inline long long mx4_pitch(long long cols) { return (cols + MX4_WIDE - 1) / MX4_WIDE * (MX4_WIDE / 2); }            // bytes of a row's codes
inline long long mx4_scale_pitch(long long cols) { return (cols + MX4_WIDE - 1) / MX4_WIDE * (MX4_WIDE / MX4_BLOCK); }
hipError_t launch_mx4_pack(const void* x, long long ldx, int rows, int cols, int dtype, uint8_t* codes, uint8_t* scales, hipStream_t st);
hipError_t launch_mx4_unpack(const uint8_t* codes, const uint8_t* scales, int rows, int cols, int dtype, void* y, long long ldy, hipStream_t st);

// sums[m][n] = sum over k of a[m][k] b[n][k], both in 4 bits as mx4_pack lays them out, finished by p.f.
struct Mx4Product {
    const uint8_t *a, *a_scales, *b, *b_scales;
    int M, N, K;
    const void* x;                          // few rows: a as a tensor of the type, rows ldx apart, in place of its codes; else null
    long long ldx;
    int splits;                             // workgroups that share a tile's K; their sums go to `partial` if > 1
    float* partial;                         // [splits][M][N rounded up to 4]
    DenseFinish f;
};
// The kernel for few rows reads weights once for up to 64 rows of a, and can bring those into 4 bits itself.  It takes up to sixteen rows always, and more, in
// groups of 64, where the summed axis is short and there is little to do.  Every sixteen columns bring x into 4 bits again, some 0.13 us of a SIMD for
// sixteen rows and 128 k, against a launch of 2 to 4 us.  Calls, us, x in the kernel / packed before it (beyond sixteen rows by the other kernel): 1 x 4096 -> 4096
// bf16 8.1 / 12.4, 1 x 512 -> 1000 7.6 / 11.7, 1 x 4096 -> 16384 15.5 / 13.4, 1 x 16384 -> 4096 17.6 / 14.0; 17 x 4096 -> 4096 10.3 / 14.0, 32 x 4096 -> 4096 11.6 / 14.5,
// 64 x 512 -> 1000 8.5 / 10.8, 64 x 4096 -> 1024 18.3 / 13.3, 256 x 1000 -> 1000 7.9 / 11.1, 512 x 1000 -> 1000 9.8 / 11.1 (on the GPU alone 10.0 / 7.7),
// 2048 x 512 -> 512 11.9 / 10.9.  Packed already, this kernel / the other: 32 x 4096 -> 4096 8.1 / 12.2, 64 x 4096 -> 4096 11.4 / 9.6, 32 x 16384 -> 4096 24.7 / 15.2.
inline bool mx4_short(long long M, long long N, long long K)
{
    const long long at_once = M <= 16 ? 1 : M <= 32 ? 2 : 4, blocks = ((M + 15) / 16) * ((N + 15) / 16);
    return M <= 1 << 15 && at_once * K <= 8192 && blocks * K <= (M <= 32 ? 1 << 21 : 1 << 20);
}
inline bool mx4_few_wanted(long long M, long long N, long long K) { return M <= 16 || mx4_short(M, N, K); }
bool mx4_few_launchable(int N);
hipError_t launch_mx4_few(const Mx4Product& p, int dtype, hipStream_t st);
DenseTilePlan mx4_tile_plan(int M, int N, int K);
hipError_t launch_mx4_tile(const Mx4Product& p, int tile, int dtype, hipStream_t st);

}  // namespace iolb

#endif
