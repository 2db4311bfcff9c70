// Dense layers (y = act(x W^T + b) + r), 8-bit activation checkpoints and the layers' gradients: what the kernels share.
//
// Products run on the 16-bit matrix cores with sums in fp32.  bf16 and fp16 tensors go there as they are; an fp32 tensor as
// the sum of three bf16 parts, x = h + m + l, eight significant bits each, of whose nine products the six that reach fp32
// precision are taken (the other three are below 2^-24 of the product), smallest first; in large forward products as two fp16 parts
// scaled by rows, of which three products are taken (dense_halves.hip).  A part is a "plane" of its own in memory, and a product of
// two planes a "segment" of the sum.
//
// Not finite: h of an infinity or NaN is that value, m and l are zero.  h h then gives what fp32 arithmetic gives, while
// the other products may turn 0 x inf into NaN or add infinities of the wrong sign; so h h comes last, and sums that are not
// finite before it are cleared.  Likewise a value whose h would round up to infinity is cut off instead of rounded.
#ifndef IOLB_DENSE_H
#define IOLB_DENSE_H

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "iolbconv.h"

namespace iolb {

constexpr int CKPT_BLOCK = 32;              // values of a row that share a scale
constexpr int MAX_SEGMENTS = 6;

// ---- what is done to a sum before it is written --------------------------------------------------
struct DenseFinish {
    const void* bias;                       // may be null
    const void* residual;                   // may be null
    void* y;
    int8_t* zq;                             // checkpoint of what the activation is applied to; may be null
    uint8_t* ze;
    long long ldr, ldy;
    int M, N;
    int act, first;                         // first: the residual is added before the activation
};

// A row in two fp16 parts: its values are those of the parts times 2^exponent; what the parts leave out, scaled like them (dense_halves.hip).
struct DenseScale { int exponent; float lost; };

// C[m][n] = sum over segments and k of A[m][k] B[n][k]; both operands contiguous along k, 16-byte aligned rows.
struct DenseProduct {
    const void* a;
    const void* b;
    long long lda, ldb;                     // elements
    int M, N, K;                            // K: a multiple of 8
    int segments;
    long long a_plane[MAX_SEGMENTS], b_plane[MAX_SEGMENTS];   // where the segment's planes start, in elements
    int splits;                             // workgroups that share a tile's K; their sums go to `partial` if > 1
    float* partial;                         // [splits][M][N rounded up to 4]
    int block_columns, per;                 // kernels for few rows: workgroups take runs of `per` steps, block after block of columns,
                                            // and a block's pieces are as many as runs meet it (block_columns 0: `splits`)
    // fp32 operands in two fp16 parts: their rows' scales (null otherwise), and the operands themselves, `values_k` long, for sums that are taken again
    const DenseScale *scales_a, *scales_b;
    const float *values_a, *values_b;
    long long ld_values_a, ld_values_b;
    int values_k;
    // not null: [0] operands that two parts do not hold, [1] blocks of sums that were left out.  `when` 0: the launch in two parts, nothing if [0];
    // 1: in three, nothing unless [0] or [1], and where not [0] only the blocks marked in `left`.
    int *uneven, *left;
    int when;
    DenseFinish f;
};

// Blocks of the tile kernel.
enum { DENSE_TILE_256, DENSE_TILE_128, DENSE_TILE_64x128, DENSE_TILE_64, DENSE_TILES };
struct DenseTilePlan { int tile, splits; };
DenseTilePlan dense_tile_plan(int M, int N, int K, int segments);
bool dense_tile_launchable(const DenseTilePlan& plan, int M, int N);           // whether a launch can count its threads
inline size_t dense_partial_bytes(int splits, long long M, long long N) { return (size_t)splits * M * ((N + 3) / 4 * 4) * 4; }
// dtype: of y, bias and residual.  Operands are of the type; for fp32 they are in two fp16 parts where scales_a is given, else in three bf16 parts.
hipError_t launch_dense_product(const DenseProduct& p, int tile, int dtype, hipStream_t st);
// Blocks of sums that are finished together, marks in `left`.
long long dense_finish_blocks(const DenseTilePlan& plan, int M, int N);

// The same for few rows of A: both operands as the caller holds them (fp32 too: taken apart in the kernels), K at least 8,
// bound by reading B.  across: B is [K][N], summed along its rows, N at least 2.  K is shared by workgroups, at most `splits` to a sum.  Sums go to `partial` if join is
// set (always with splits > 1 or a checkpoint).
constexpr int DENSE_FEW = 16;               // rows of the kernel for the fewest
// Whether a product with M rows and an N x K weight runs on them, or on the product kernel with its operands laid out.  fp32: the layout of the
// weights in parts costs more than all of the product up to some hundred rows (4096 x 4096, us: 64 rows 24 against 69, 128 33 / 77, 256 54 / 84, 512 93 / 110;
// 512 x 512, 256 rows 12 / 16).  Their rows are read in pieces of eight values, or two across: shorter ones are left to the product kernel.  16-bit types: the product kernel reads weights in place (4096 x 4096, 20 rows 15.7 against 12.6), but across
// they would be transposed: 4096 x 4096, 64 rows 15.5 against 28, 128 24.8 / 31, 256 40 / 37; 1000 x 2048, 20 rows 13.1 / 13.2, 64 17.9 / 14.2.
inline bool dense_rows_wanted(long long M, long long N, long long K, int dtype, bool across)
{
    if (across ? N < 8 || K < 2 : K < 8) return false;
    if (dtype == IOLB_F32) return M <= 512;
    if (!across) return M <= DENSE_FEW;
    return M <= 32 || (M <= 128 && N * K >= (1 << 22));
}
constexpr int DENSE_OUTER_MOST = 64;
constexpr int DENSE_ROWS_STEP = 64;         // k of a step
struct DenseRowsPlan { int splits, per; bool join; int block_columns; };
DenseRowsPlan dense_rows_plan(int M, int N, int K, int dtype, bool across, bool checkpoint);
bool dense_rows_launchable(const DenseRowsPlan& plan, int M, int N, int K, bool across);
hipError_t launch_dense_rows(const DenseProduct& p, bool across, bool join, int dtype, hipStream_t st);
hipError_t launch_dense_join(const DenseProduct& p, int dtype, hipStream_t st);
// The same for a short summed axis, 0 < K <= DENSE_OUTER_MOST: operands in planes, `plane_a` and `plane_b` elements apart; no bias, activation,
// residual or checkpoint.  At most DENSE_OUTER_ROWS rows of A.
constexpr long long DENSE_OUTER_ROWS = 65535 * 128LL;
hipError_t launch_dense_outer(const DenseProduct& p, int planes_b, long long plane_a, long long plane_b, int dtype, hipStream_t st);

// ---- operands laid out for the product --------------------------------------------------------------
// Values v[r][c], rows x cols, from one of three sources:
enum { DENSE_FROM_TENSOR, DENSE_FROM_CHECKPOINT, DENSE_FROM_GRADIENT };
struct DenseLayout {
    int source;
    int planes;                             // 1 or 3 (fp32: bf16 parts; 1 where the values are exact in bf16)
    int rows, cols;
    const void* src;                        // tensor: v = src;  gradient: v = src * act'(checkpoint), or src where q is null
    long long ld;
    const int8_t* q;                        // checkpoint: v = act(value)
    const uint8_t* e;
    int act;
    void* rowmajor;                         // [planes][rows][ld_rm], or null; columns up to the next multiple of 8 are zero
    long long ld_rm;
    void* transposed;                       // [planes][cols][ld_tr], or null; likewise
    long long ld_tr;
    void* copy;                             // v in the tensor's own type, [rows][cols], or null
    float* colsum;                          // [ceil(rows / 64)][cols]: sums over 64 rows each, or null
    void* total;                            // up to 64 rows: the sums in the tensor's type instead, or null
    int odd;                                // set by the launcher: 16-bit values of src may start at odd addresses
};
// Up to three of them in one launch.
constexpr int MAX_LAYOUTS = 3;
struct DenseLayouts {
    int count;
    const int* uneven;                      // not null: the launch does nothing unless one of the two is set
    DenseLayout of[MAX_LAYOUTS];
};
// dtype: of src, copy and (16-bit types) the planes.
hipError_t launch_dense_layouts(int dtype, const DenseLayouts& l, hipStream_t st);
// out[c] = sum of colsum over its `blocks` rows, in `dtype`.
hipError_t launch_dense_colsum(const float* colsum, int blocks, int cols, void* out, int dtype, hipStream_t st);

// Rows of a tensor, `cols` long, in two fp16 parts, planes [2][rows][pitch] (pitch: cols rounded up to 8), their scales;
// uneven[0] becomes 1 if two parts do not hold a row well, else 0, and uneven[1] 0.
struct DenseHalves {
    const float* x;
    long long ld;
    int rows;
    unsigned short* planes;
    DenseScale* scales;
};
// Workgroups of 256: a wave to a row, or all of it where there are few rows or they are long.
inline bool dense_halves_by_workgroup(long long rows_a, long long rows_b, long long cols) { return rows_a + rows_b < 4096 || cols > 4096; }
inline long long dense_halves_groups(long long rows_a, long long rows_b, long long cols)
{
    return dense_halves_by_workgroup(rows_a, rows_b, cols) ? rows_a + rows_b : (rows_a + 3) / 4 + (rows_b + 3) / 4;
}
hipError_t launch_dense_halves(const DenseHalves& a, const DenseHalves& b, int cols, long long pitch, int* uneven, hipStream_t st);

hipError_t launch_checkpoint_pack(const void* x, long long ldx, int rows, int cols, int dtype, int8_t* q, uint8_t* e, hipStream_t st);
hipError_t launch_checkpoint_unpack(const int8_t* q, const uint8_t* e, int rows, int cols, int act, int dtype, void* y, long long ldy,
                                    hipStream_t st);

// The calling thread's stream, and its record of the last HIP error (IOLB_EHIP is returned).
hipStream_t call_stream();
int note_hip_error(hipError_t e);

}  // namespace iolb

#endif
