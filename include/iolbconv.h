/*
 * iolbconv -- forward 2-D convolution for AMD MI355X (gfx950), tiled by the red-blue-pebble
 * I/O lower bound of "I/O Lower Bounds for Auto-tuning of Convolutions in CNNs".
 *
 * C ABI.  Every tensor pointer is a DEVICE pointer to dense fp32 data owned by the caller; the
 * library never frees or keeps them.  All entry points return 0 on success or a negative
 * IOLB_E* code; no exception crosses this boundary and nothing aborts.  Arguments are checked
 * before anything is launched, so a call that fails validation writes nothing.
 *
 * Work is enqueued on the stream given to iolb_set_stream (the null stream by default; the setting is per host
 * thread) and the calls return without waiting for it.  Thread-compatible with one stream per host thread: the
 * library keeps one workspace per (GPU, stream), so calls on different streams do not share scratch memory;
 * calls on one stream are ordered by the stream.  A call that does not have to grow its stream's workspace
 * enqueues kernels only (no allocation, no memset, no synchronisation), so after one eager call for the same
 * layer on the same stream it can be recorded by a stream capture and replayed as a graph.  One that has to grow it
 * while the stream is captured allocates there and then; the graph holds its kernels only.  A workspace that
 * has to grow is replaced, never freed before iolb_release_workspace, so kernels in flight and graphs captured
 * earlier keep valid addresses; iolb_release_workspace invalidates such graphs.
 *
 * Symbols (paper -> here): W_in,H_in,C_in -> W,H,C;  C_out -> K;  W_ker,H_ker -> S,R;
 * W_out,H_out -> Q,P;  mu -> stride;  e -> m.  A batch of N images shares the K kernels.
 */
#ifndef IOLBCONV_H
#define IOLBCONV_H

#include <stddef.h>
#include <stdint.h>

#ifdef __cplusplus
extern "C" {
#endif

#define IOLB_OK            0
#define IOLB_EINVAL       -1   /* null pointer, non-positive extent, stride < 1, pad < 0, empty output */
#define IOLB_EUNSUPPORTED -2   /* Winograd m outside {2,3,4,6}; algo, layout, type, activation or norm outside its enum; dense layer or tensor too large */
#define IOLB_ENOTILE      -3   /* no tile fits the LDS / register budgets */
#define IOLB_EWORKSPACE   -4   /* workspace missing or too small */
#define IOLB_EHIP         -5   /* a HIP runtime call or launch failed; see iolb_last_hip_error */

enum { IOLB_DIRECT = 0, IOLB_WINO_F2 = 1, IOLB_WINO_F4 = 2, IOLB_WINO_F3 = 3, IOLB_WINO_F6 = 4 };
enum { IOLB_PATH_FMA = 0, IOLB_PATH_MFMA = 1, IOLB_PATH_FUSED = 2, IOLB_PATH_POINT = 3 };
/* FUSED: Winograd only, all four steps in one matrix-core kernel (Sec. 5.3).  POINT: direct convolution with
 * R = S = 1, no padding, channels-outermost tensors only: the dataflow of Sec. 5.2 on the output plane taken as
 * one row of P * Q pixels (without a kernel window the pixels do not interact). */
enum { IOLB_LAYOUT_CHW = 0, IOLB_LAYOUT_HWC = 1, IOLB_LAYOUT_CWH = 2 };   /* per image: channels outermost, channels
                                                                           innermost, channels outermost with W before H */

/* A convolution layer (Sec. 2.2).  Output extents are P = floor((H+2 pad-R)/stride)+1 and
 * Q = floor((W+2 pad-S)/stride)+1.  For the Winograd algos R = S = 3 and stride = 1. */
typedef struct iolb_shape {
    int32_t N, C, H, W, K, R, S, stride, pad;
    int32_t algo;               /* IOLB_DIRECT or IOLB_WINO_F2 / _F3 / _F4 / _F6 (m = 2, 3, 4, 6) */
} iolb_shape;

/* A tile configuration: the output sub-block x * y * z of Sec. 5.2 (x along W_out, y along
 * H_out, z along C_out) taken over b images, the channels per stage alpha, and the thread
 * decomposition (Table 1 of Sec. 6.2: tile sizes and thread numbers).
 * For the Winograd algos the block is a strip of x/m sub-domains of m x m outputs (b = 1,
 * y = m) of one transformed plane.  For IOLB_PATH_POINT the block is x consecutive pixels of the image
 * taken as one row of P * Q pixels (b = 1, y = 1; a block may run on into the next image) by z output
 * channels.  All fields are exact integers. */
typedef struct iolb_tile_config {
    int32_t b, x, y, z;
    int32_t alpha;               /* input channels staged per step of the channel loop */
    int32_t threads;             /* workgroup size */
    int32_t waves_m, waves_n;    /* MFMA path: wave grid over (z, pixels); FMA path: channel groups, 1 */
    int32_t path;                /* IOLB_PATH_FMA, _MFMA, _FUSED or _POINT */
    int32_t wt_mode;             /* 0: raw R*S weights staged; 1: pre-transformed (m+2)^2 weights; 2: thin direct
                                    layers (3 x 3, stride 1, C <= 4, channels-outermost tensors): one lane per x / 256
                                    neighbouring pixels of a row and all z = K channels, kernels through the scalar unit */
    int32_t lds_bytes_used;      /* staging bytes the tile needs */
    int32_t acc_regs_per_thread; /* partial sums held per lane */
    int64_t q_read_elems;        /* modelled elements read by all workgroups (exact form of the
                                    reading volume of Sec. 5.2 / 5.3 for this tile) */
    int64_t q_write_elems;       /* N*K*P*Q: every output written once */
} iolb_tile_config;

/* Figures of the lower-bound theory for one layer at fast-memory size S_f (in elements). */
typedef struct iolb_bounds_out {
    int32_t P, Q;
    int64_t vertices;            /* internal+output vertices of the DAG: Sec. 4.2 second lemma
                                    (direct); per-step counts of the Sec. 4.3 lemma (Winograd) */
    int64_t compulsory_elems;    /* N*C*H*W + K*C*R*S + N*K*P*Q (Sec. 3.1: each input loaded and
                                    each output stored at least once) */
    int64_t q_write_elems;
    double  t_bound_2s;          /* T(2 S_f): Sec. 4.2 third lemma / Sec. 4.3 T lemma */
    double  q_lower_lead;        /* leading term printed in the theorems of Sec. 4.2 / 4.3 */
    double  q_lower_explicit;    /* S_f (|V|/T(2 S_f) - 1), the general theorem of Sec. 4.1 */
    double  q_dataflow;          /* total volume of the near-optimal dataflow, Sec. 5.2 / 5.3, N_p = 1 */
} iolb_bounds_out;

/* Direct convolution (Sec. 2.2, dataflow of Sec. 5.2).
 *   y[n,k,p,q] = sum_{c,r,s} xpad[n,c,p*stride+r-pad,q*stride+s-pad] * w[k,c,r,s]
 * x: [N][C][H][W], w: [K][C][R][S], y: [N][K][P][Q]; cross-correlation, zero padding.
 * y is fully overwritten; x and y must not overlap.  The tile comes from iolb_tune with the
 * default budgets.  May grow the stream's workspace in the library (one allocation, kept).
 * Without a caller-supplied tile, layers that are bound by the fp32 matrix instructions run on the 16-bit ones instead
 * (this call, conv_direct_layout with cfg NULL, conv_direct_pad2, conv_direct_noalloc; the products of conv_winograd,
 * conv_winograd_pad, and conv_winograd_ws / _pre with cfg NULL): every operand as the sum of two fp16 parts under a
 * scale taken from the data, three products of parts, or, for few channels and small layers, as the sum of three bf16 parts,
 * six products; fp32 sums.  Their blocks are not tiles of the enumeration; a caller-supplied tile always runs on the fp32 kernels.
 * Precision.  Three parts: no less than fp32 products.  Two parts, n = C R S: to the rounding of fp32 sums two errors add.  Parts hold an
 * operand to 2^-23 of it and their smallest product is left out: 2^-21 |x| |w| per product at most.  And operands below 2^-10 (Winograd F(4x4): 2^-4) of a
 * sample's largest value lose more; that is at most 2^-21 in the root mean square, sqrt(n) 2^-20 at worst, of the largest of the sums of the
 * same kernel that are judged together: those of a few neighbouring output pixels of one image (Winograd: of the sums of a plane, and
 * 2^-18).  Where no sum of them is large enough for that, they are computed again in fp32, as are outputs that the parts cannot hold
 * (infinities, NaN, operands or sums near the end of the range).  So a single output is less precise than an fp32 sum only where it is
 * far smaller than its neighbours of the same kernel and its window holds values far below the largest of theirs.  What is computed
 * again costs time: 1.1 - 1.5 times the layer's where few outputs are, up to twelve times where most are (one huge value in every image,
 * channels and kernels scaled by 1e3 and 1e-3 against each other). */
int conv_direct(const float* x, const float* w, float* y,
                int N, int C, int H, int W, int K, int R, int S, int stride, int pad);

/* Same, with the tile given by the caller (for sweeps).  cfg must be one that iolb_tune or
 * iolb_enumerate produced for this shape; IOLB_EINVAL otherwise. */
int conv_direct_cfg(const float* x, const float* w, float* y,
                    int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                    const iolb_tile_config* cfg);

/* Direct convolution with the tensor layout as a parameter (the layout entry of the searching
 * domain, Table 1 of Sec. 6.2).  IOLB_LAYOUT_CHW: as conv_direct.  IOLB_LAYOUT_HWC:
 * x: [N][H][W][C], y: [N][P][Q][K].  IOLB_LAYOUT_CWH: x: [N][C][W][H], y: [N][K][Q][P] (the
 * transposed image: computed as the CHW convolution of the W x H image with the kernels
 * transposed, so tiles are those of that transposed layer).  w is [K][C][R][S] for all.  cfg may be NULL (the tuned
 * tile is used; tiles do not depend on the layout, except that IOLB_PATH_POINT tiles and the thin-layer tiles
 * (wt_mode 2) exist for IOLB_LAYOUT_CHW only: IOLB_EINVAL with another layout; with cfg NULL the best other tile is used).  Other layout values: IOLB_EUNSUPPORTED. */
int conv_direct_layout(const float* x, const float* w, float* y,
                       int N, int C, int H, int W, int K, int R, int S, int stride, int pad,
                       int layout, const iolb_tile_config* cfg);

/* conv_direct for callers that cannot allocate device memory: code under HIP graph capture, tight serving
 * loops, harnesses that forbid hipMalloc.  Same arguments, layouts and result (bit for bit) as conv_direct, but
 * the re-laid-out weights go into a fixed array inside the library instead of the grown workspace: the call
 * makes no hipMalloc / hipFree and no allocating library call, and enqueues kernels only.
 * Limit: K rounded up to 32, times C rounded up to whole stages (at most 16 extra channels), times R * S must
 * not exceed conv_direct_noalloc_max_weight_floats() = 4194304 floats (the array has room for them in three bf16
 * parts: 24 MiB, held by every GPU the library has run this call on until the process ends); beyond it the call returns IOLB_EWORKSPACE and launches
 * nothing.  All calls on one GPU share that array: calls that overlap on one GPU (two streams) race, and a
 * captured graph must not replay concurrently with another call of this entry point on the same GPU. */
int conv_direct_noalloc(const float* x, const float* w, float* y,
                        int N, int C, int H, int W, int K, int R, int S, int stride, int pad);
size_t conv_direct_noalloc_max_weight_floats(void);

/* conv_direct with its own padding per axis: pad_h rows of zeros above and below, pad_w columns left and
 * right (the 1 x 7 / 7 x 1 factorised kernels of Inception-v3 pad one axis only); P and Q follow from
 * pad_h and pad_w.  NCHW tensors, tuned tile. */
int conv_direct_pad2(const float* x, const float* w, float* y,
                     int N, int C, int H, int W, int K, int R, int S, int stride, int pad_h, int pad_w);

/* Winograd F(m x m, 3 x 3) convolution (Sec. 2.3; four steps of Sec. 4.3), R = S = 3,
 * stride 1, pad 1 (P = H, Q = W), m in {2, 3, 4, 6} (Sec. 2.3 names e = 2 and e = 3; larger m
 * trades more rounding error for fewer multiplications).  Same layouts as conv_direct.  The transformed
 * kernels, inputs and products live in the library's device workspace, grown on demand.
 * Thin layers (C <= 4 and C * (m+2)^2 <= 128; the tuned tile then has path == IOLB_PATH_FMA) run the
 * fused dataflow of Sec. 5.3 as one kernel: transformed inputs and channel sums stay in registers, the
 * workspace holds the transformed kernels only. */
int conv_winograd(const float* x, const float* w, float* y,
                  int N, int C, int H, int W, int K, int m);

/* conv_winograd with `pad` zeros on every side instead of one (pad >= 0, H + 2 pad >= 3, W + 2 pad >= 3):
 * y is [N][K][H + 2 pad - 2][W + 2 pad - 2].  Sub-domain (i, j) reads the (m+2) x (m+2) window whose corner is
 * (i m - pad, j m - pad).  Library workspace, tuned tile. */
int conv_winograd_pad(const float* x, const float* w, float* y,
                      int N, int C, int H, int W, int K, int m, int pad);

/* Bytes of workspace conv_winograd_ws needs for this layer (0 on invalid arguments). */
size_t conv_winograd_workspace_bytes(int N, int C, int H, int W, int K, int m);

/* conv_winograd with a caller-owned device workspace of at least that many bytes, 256-byte
 * aligned.  cfg may be NULL (the tuned tile is used). */
int conv_winograd_ws(const float* x, const float* w, float* y,
                     int N, int C, int H, int W, int K, int m,
                     void* workspace, size_t workspace_bytes, const iolb_tile_config* cfg);

/* Kernels transformed once, used by many calls (inference: the weights do not change).
 * conv_winograd_kernel_bytes: size of the transformed-kernel buffer for C x K kernels of
 * F(m x m, 3 x 3) (0 on invalid arguments).  conv_winograd_transform_kernels: writes
 * U = L g L^T (first step of Sec. 4.3) for w [K][C][3][3] into that caller-owned, 256-byte
 * aligned device buffer, laid out [(m+2)^2][C rounded up to 16][K rounded up to 32] with zeros
 * in the padding.  conv_winograd_pre: conv_winograd_ws with U in place of w; the workspace
 * size is the one conv_winograd_workspace_bytes reports. */
size_t conv_winograd_kernel_bytes(int C, int K, int m);
int conv_winograd_transform_kernels(const float* w, float* U, int C, int K, int m);
int conv_winograd_pre(const float* x, const float* U, float* y,
                      int N, int C, int H, int W, int K, int m,
                      void* workspace, size_t workspace_bytes, const iolb_tile_config* cfg);

/* The analytical tuner.  Searching domain: Table 1 of Sec. 6.2 read for this machine (tile extents from the
 * factors of the output extents, blocks that fit the accumulator registers and the LDS).  Order: a modelled
 * run time -- THIS LIBRARY'S HEURISTIC, fitted to tile sweeps on an MI355X -- whose memory term and tie-break
 * are the reading volume of the dataflow of Sec. 5.2 / 5.3.  Host only; shape and out are host pointers.
 * lds_bytes: LDS available to one workgroup; 0 = automatic: 81920 (half a compute unit's LDS, the
 * "two blocks per multiprocessor" rule of Sec. 6.2), or the whole LDS for tiles whose registers
 * allow only one workgroup per compute unit anyway.  vgpr_budget: accumulator registers per
 * lane (0 = default 128; the fused Winograd blocks, which hold up to 96, are exempt from the default).
 * IOLB_ENOTILE when nothing fits. */
int iolb_tune(const iolb_shape* shape, size_t lds_bytes, int vgpr_budget, iolb_tile_config* out);

/* The bound-only pick: the same domain restricted to the optimality box of Table 1 (z <= sqrt(S_b/rho),
 * x y <= sqrt(S_b rho); the whole domain if the box is empty), ordered by the paper's objective alone -- the
 * reading volume Q_read of Sec. 5.2 / 5.3 evaluated exactly for the tile, ties by |b x y mu^2 - W_ker H_ker z|
 * (distance from the optimality condition x y = R z), then the fuller block.  For the Winograd algos the fused
 * dataflow of Sec. 5.3 comes before the unfused tiles.  Same arguments and errors as iolb_tune. */
int iolb_tune_bound(const iolb_shape* shape, size_t lds_bytes, int vgpr_budget, iolb_tile_config* out);

/* Every feasible tile for the shape, best first (the domain the exhaustive sweep times).
 * use_box != 0 applies the optimality-condition box z <= sqrt(S_b/rho), xy <= sqrt(S_b rho).
 * Writes at most `capacity` entries to out (may be NULL) and returns the total count, or a
 * negative code. */
int64_t iolb_enumerate(const iolb_shape* shape, size_t lds_bytes, int vgpr_budget, int use_box,
                       iolb_tile_config* out, int64_t capacity);

/* What a call without a caller-supplied tile runs on: IOLB_ROUTE_TILE, the fp32 kernels with the tuned tile, or
 * IOLB_ROUTE_SPLIT, the 16-bit matrix cores (see conv_direct); or a negative code.  It depends on the layer and the layout
 * alone.  layout: as for conv_direct_layout (IOLB_LAYOUT_CHW for the Winograd algos).  *bytes (may be NULL): on the split
 * route the bytes of the re-laid-out kernels (direct) or the least workspace that takes it (Winograd), else 0.
 * conv_direct_noalloc takes the route of conv_direct, within its limit.  Host only. */
enum { IOLB_ROUTE_TILE = 0, IOLB_ROUTE_SPLIT = 1 };
int iolb_route(const iolb_shape* shape, int layout, size_t* bytes);

/* Lower-bound figures for a layer at fast-memory size S_f elements.  Host only. */
int iolb_bounds(const iolb_shape* shape, int64_t S_f_elems, iolb_bounds_out* out);

/* The constant transform matrices the Winograd kernels use for F(m x m, 3 x 3) (Sec. 2.3: input
 * transform B d B^T, kernel transform L g L^T, output transform A M A^T), row-major into host
 * arrays A[m][m+2], L[m+2][3], B[m+2][m+2].  Host only.  IOLB_EUNSUPPORTED for other m. */
int iolb_winograd_matrices(int m, float* A, float* L, float* B);

/* ---- Dense layers and 8-bit activation checkpoints -----------------------------------------------------
 * What follows a network's convolutions: y = act(x W^T + b) with a residual, its gradients, and the activations that the
 * backward pass needs held in 8 bits.  Tensors are fp32, fp16 or bf16, all of a call of one type, and hold rows of
 * contiguous values whose starts are ld... values apart (at least the row's length; any alignment of the type's own size).  Sums are
 * held in fp32 and rounded once to the tensor's type.  fp32 operands go to the matrix cores as the sum of three bf16 parts, which
 * hold them to the last bit from 2^-110 up; below that the absolute error stays under 2^-133.  Large fp32 products of iolb_linear (M above
 * 512 or K below 8, M N K at least 3e9) take two fp16 parts instead, which hold a value to 2^-22 of itself unless it is far below its row's
 * largest.  Every sum is within 2^-19 of its sum of magnitudes beside the rounding of fp32 sums: where an operand has rows with many such
 * values, or sums are too small for what was cut, the call finds that on the device and takes the product, or those sums, in full.  Infinities and NaN give what fp32 arithmetic gives.  Extents may be zero: no output then, or (a sum over nothing) bias and residual alone.
 * These calls allocate nothing: scratch is the caller's, 256-byte aligned, at least as large as the ..._workspace_bytes
 * call of the same arguments says (it may be 0: NULL then).  It depends on addresses too: tensors whose rows
 * do not start on 16 bytes are copied.  They enqueue kernels only, on the stream of iolb_set_stream, and can be captured. */
enum { IOLB_F32 = 0, IOLB_F16 = 1, IOLB_BF16 = 2 };
/* silu: z / (1 + e^-z);  gelu: z Phi(z);  gelu_tanh: z (1 + tanh(sqrt(2 / pi) (z + 0.044715 z^3))) / 2.  All three are 0 at
 * -infinity; a NaN stays one.  In fp32 they hold to 1e-6 |z| + 1e-7 (gelu's tail from a published formula: 5e-5 of the result at z = -3, 5e-4 at -4),
 * their slopes to 4e-6. */
enum { IOLB_ACT_NONE = 0, IOLB_ACT_RELU = 1, IOLB_ACT_SILU = 2, IOLB_ACT_GELU = 3, IOLB_ACT_GELU_TANH = 4 };

/* z = x w^T + bias (+ residual if residual_first);  y = act(z) (+ residual otherwise).
 * x [M][K], w [N][K], bias [N] or NULL, residual [M][N] or NULL, y [M][N]; y may be the residual itself, and overlaps nothing
 * else.  zq, ze (both or neither): the checkpoint of z, from the fp32 sums, as iolb_checkpoint_pack lays it out.
 * M, N up to 2^30, K up to 2^22, and no launch of 2^32 threads or more, as 2^27 columns for up to 16 rows would take (IOLB_EUNSUPPORTED beyond). */
typedef struct iolb_linear_args {
    int64_t M, N, K;
    int32_t dtype, act, residual_first;
    const void *x, *w, *bias, *residual;
    void* y;
    int64_t ldx, ldw, ldr, ldy;
    int8_t* zq;
    uint8_t* ze;
} iolb_linear_args;
int iolb_linear_workspace_bytes(const iolb_linear_args* args, size_t* bytes);
int iolb_linear(const iolb_linear_args* args, void* workspace, size_t workspace_bytes);

/* The 8-bit checkpoint of x [rows][cols]: q [rows][cols] and one byte for each 32 values of a row, e [rows][ceil(cols / 32)].
 * A value is q 2^(e - 127), q from -127 to 127, with the least exponent that brings the block's finite values within
 * that (at least 2^-126, for fp16 2^-24; at most 2^122, for fp16 2^10, where q stops at 63), rounded to nearest even.  The error is at most
 * half of 2^(e - 127): 1/127 of the block's largest value, 1/254 at best, with an exponent between the two ends; at the least one it may be all
 * of a value up to 2^-127 (fp16 2^-25); at the largest one, where q stops, up to 2^(e - 127) (fp16: 65504 is held as 64512), and finite sums beyond
 * the type, in iolb_linear's checkpoint, are held as 63 2^10 or 63 2^122 while y is infinite.  Values that are not finite become q = -128 and read back as NaN.
 * Every value is one of the tensor's type, and of bf16.  A checkpoint does not say what type it was packed from: read as another one, its values are
 * rounded to that, and as fp16 they are infinite from 65520 on. */
int iolb_checkpoint_pack(const void* x, int64_t ldx, int64_t rows, int64_t cols, int dtype, int8_t* q, uint8_t* e);
/* y [rows][cols] = act(values of the checkpoint). */
int iolb_checkpoint_unpack(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, int act, int dtype, void* y, int64_t ldy);

/* Gradients of iolb_linear from dy [M][N], w [N][K] and checkpoints: xq, xe of the layer's input, [M][K] (x = act_x of its values:
 * an input that is another layer's activation is recomputed from that layer's checkpoint); zq, ze of what the activation
 * was applied to, [M][N] (NULL with IOLB_ACT_NONE).
 *   dz = dy act'(z);  dx [M][K] = dz w;  dw [N][K] = dz^T x;  db [N] = sum of dz over its rows
 * dz [M][N] is the residual's gradient where that came before the activation.  Outputs are dense; each may be NULL, and w, xq
 * with it.  The slope of relu at 0 is 0, and a dy that it stops is not looked at.  16-bit types: dz, and an input
 * that is recomputed through silu, gelu or gelu_tanh, are rounded to the type once, before the products (as fp16 a dz below 2^-25 is 0: scale dy); db is summed
 * before that.  Sums are added in a fixed order: equal calls give equal bits.
 * M, N up to 2^22, K up to 2^30, and no launch of 2^32 threads or more (IOLB_EUNSUPPORTED beyond). */
typedef struct iolb_linear_backward_args {
    int64_t M, N, K;
    int32_t dtype, act, x_act;
    const void *dy, *w;
    int64_t ldy, ldw;
    const int8_t* xq;
    const uint8_t* xe;
    const int8_t* zq;
    const uint8_t* ze;
    void *dx, *dw, *db, *dz;
} iolb_linear_backward_args;
int iolb_linear_backward_workspace_bytes(const iolb_linear_backward_args* args, size_t* bytes);
int iolb_linear_backward(const iolb_linear_backward_args* args, void* workspace, size_t workspace_bytes);

/* ---- Around the dense layers of a residual block --------------------------------------------------------
 * Norms with gate and residual scale and their gradients, dropout, and dense layers in microscaled 4-bit floating point.  Types, rows, strides,
 * extents of zero, workspaces, streams and capture: as above.  M, N, rows, cols up to 2^30 if not said otherwise. */
enum { IOLB_NORM_NONE = 0, IOLB_NORM_RMS = 1, IOLB_NORM_LAYER = 2 };

/* The end of a block and the start of the next, row by row of N values:
 *   p = post(h) post_weight + post_bias;   x' = scale x + gate p;   y = pre(x') pre_weight + pre_bias
 * IOLB_NORM_RMS: v / sqrt(mean of v^2 + eps);  IOLB_NORM_LAYER: (v - mean) / sqrt(variance + eps);  IOLB_NORM_NONE: v itself, without weight
 * and bias (pre: there is no y).  x, h [M][N]; weights and biases [N], each may be NULL; gate [groups][N] or NULL: groups divides M, and
 * row m takes the gate's row m / (M / groups).  x' is rounded to the type, and y is of x' as rounded: what a backward pass reads is what was normalised.
 * x_out [M][N] may be x itself, and y and x_out overlap nothing else.  h NULL: y = pre(x) alone; post, gate, x_out are none then, and scale is 1.
 * Sums in fp32, of squares too, before they are divided by N: rows of fp32 and bf16 (what h, x' hold) are normalised as said while their values stay below
 * 2^63 / sqrt(N) (N = 4096: 2^57), and become 0 where the sum of squares reaches 2^128.  With eps 0 a row needs a value, with the mean taken off, of 2^-60
 * or more; one of equal values is NaN then.  A row with a NaN becomes NaN. */
typedef struct iolb_block_norm_args {
    int64_t M, N, groups;
    int32_t dtype, post, pre;
    float scale, eps;
    const void *x, *h, *post_weight, *post_bias, *gate, *pre_weight, *pre_bias;
    void *x_out, *y;
    int64_t ldx, ldh, ldo, ldy;
} iolb_block_norm_args;
int iolb_block_norm(const iolb_block_norm_args* args);

/* Gradients of iolb_block_norm from dy [M][N] (of y; NULL with pre IOLB_NORM_NONE, or none), dx_out [M][N] (of x' from elsewhere, or NULL),
 * x [M][N]: the x' that the forward call left (the x it was given, where h was NULL), and h [M][N] or NULL.  Statistics are taken again from these.
 *   d = dx_out + (gradient of pre at x', of dy);  dx = scale d;  dh = (gradient of post at h, of gate d)
 * and of weights, biases and gate the sums of their factors over the rows that share them.  Outputs are dense, dx, dh [M][N], dgate [groups][N], the
 * others [N]; each may be NULL.  dh needs h, dgate the gate (and post_bias, where p had one), dpost_... a norm of h, dpre_... dy.
 * For rows within the limits above.  Their sums are fp32's too: with T, D, X the largest |dy pre_weight|, |d gate post_weight| and |x'| of a row, N T X, N^1.5 T
 * and N^1.5 D must stay below 2^126.
 * Sums are added in a fixed order: equal calls give equal bits.  M, N and groups up to 2^22, and with
 * gradients of weights, biases or gate groups x ceil(N / 16) below 2^32 (the workspace, 16 bytes a column and group and more, would be 2^40).  Outputs overlap nothing. */
typedef struct iolb_block_norm_backward_args {
    int64_t M, N, groups;
    int32_t dtype, post, pre;
    float scale, eps;
    const void *dy, *dx_out, *x, *h, *post_weight, *post_bias, *gate, *pre_weight;
    int64_t lddy, lddx, ldx, ldh;
    void *dx, *dh, *dgate, *dpost_weight, *dpost_bias, *dpre_weight, *dpre_bias;
} iolb_block_norm_backward_args;
int iolb_block_norm_backward_workspace_bytes(const iolb_block_norm_backward_args* args, size_t* bytes);
int iolb_block_norm_backward(const iolb_block_norm_backward_args* args, void* workspace, size_t workspace_bytes);

/* y = residual + (x scaled by 1 / (1 - p) where it stays, 0 where it is dropped); residual [rows][cols] or NULL.  The mask is not stored: the call with
 * the same seed and offset on dy, without the residual, is the backward pass.
 * Each value has 16 bits of Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, 2011) and stays where they are at least t = p 2^16, rounded; the scale is
 * 2^16 / (2^16 - t), so that the mean is kept for the p that holds.  p of 1 drops all, of less at most 65535 of 65536.  Key: seed; counter: the offset in its upper
 * 64 bits, in its lower ones r ceil(cols / 8) + c / 8 for the value in row r, column c, whose bits are the c % 8 th of eight, each word's lower half first.  So other
 * offsets give other masks, and no stride matters.  counter: two 64-bit words on the device, read when the kernel runs, added to seed and offset (a graph
 * that is replayed takes its masks from there); or NULL.
 * A dropped x is not looked at (a NaN leaves 0).  y may be x or the residual, and overlaps nothing else.  zq, ze (both or neither): the checkpoint
 * of y as rounded, as iolb_checkpoint_pack gives it. */
typedef struct iolb_dropout_args {
    int64_t rows, cols;
    int32_t dtype;
    double p;
    uint64_t seed, offset;
    const uint64_t* counter;
    const void *x, *residual;
    void* y;
    int64_t ldx, ldr, ldy;
    int8_t* zq;
    uint8_t* ze;
} iolb_dropout_args;
int iolb_dropout(const iolb_dropout_args* args);

/* Microscaled 4-bit floating point: 32 values of a row share a power of two 2^(s - 127), and each has a sign and a magnitude of 0, 0.5, 1, 1.5, 2, 3, 4 or 6 of it
 * (codes 0 to 7, the sign is bit 3).  s is the least that brings the block within 7 (so nothing is off by more than half a step there either: 6 is
 * the nearest of up to 7), values are rounded to nearest, ties to the even code.  A block with a value that is not finite has s = 255 and is NaN as a whole.  A block's
 * largest value is off by 1/6 of itself at most; what lies below 1/28 of it may become 0.
 * codes [rows][64 ceil(cols / 128)] bytes: column c in byte c / 2, the even one in the lower half; scales [rows][4 ceil(cols / 128)] bytes.  Rows
 * are padded to 128 columns of zeros, which the products read: pack writes them.  codes 16-byte aligned, scales 4-byte. */
int iolb_mx4_pack(const void* x, int64_t ldx, int64_t rows, int64_t cols, int dtype, uint8_t* codes, uint8_t* scales);
/* y [rows][cols]: the values.  What the type does not reach (6 2^126, or 2^16 in fp16) becomes its largest value. */
int iolb_mx4_unpack(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, int dtype, void* y, int64_t ldy);

/* iolb_linear with both operands in that form: w_codes, w_scales as iolb_mx4_pack lays w [N][K] out, and x either likewise (x_codes, x_scales; x NULL) or
 * a tensor [M][K] of the type, which the call brings into it first.  Products are exact, sums in fp32; bias, activation and residual
 * as there; y may be the residual.  No gradients: weights in 4 bits are for answering.  M, N up to 2^30, K up to 2^22, and no launch of 2^32 threads. */
typedef struct iolb_linear_mx4_args {
    int64_t M, N, K;
    int32_t dtype, act, residual_first;
    const void* x;
    int64_t ldx;
    const uint8_t *x_codes, *x_scales, *w_codes, *w_scales;
    const void *bias, *residual;
    void* y;
    int64_t ldr, ldy;
} iolb_linear_mx4_args;
int iolb_linear_mx4_workspace_bytes(const iolb_linear_mx4_args* args, size_t* bytes);
int iolb_linear_mx4(const iolb_linear_mx4_args* args, void* workspace, size_t workspace_bytes);

/* Stream (a hipStream_t) later calls enqueue on; NULL selects the null stream. */
int iolb_set_stream(void* hip_stream);

/* Timing hook for benchmarks: when enabled, the main kernel of each conv call is bracketed by
 * HIP events on the call's stream.  Kinds: the direct-convolution kernel (IOLB_TIME_DIRECT), the
 * Winograd batched product (IOLB_TIME_WINO_PRODUCT) and the fused Winograd matrix-core kernel
 * (IOLB_TIME_WINO_FUSED).  iolb_timing_read waits for the recorded
 * events of one kind, returns how many launches were timed since the last read of that kind and
 * their total duration in milliseconds, and forgets them. */
enum { IOLB_TIME_DIRECT = 0, IOLB_TIME_WINO_PRODUCT = 1, IOLB_TIME_WINO_FUSED = 2 };
int iolb_timing_enable(int on);
int iolb_timing_read(int kind, int* launches, float* total_ms);

/* Ceiling probes for roofline reports (the experimental set-up of Sec. 7 quotes peak rates; these measure
 * what the device at hand delivers).  Both run `reps` launches on the set stream after one untimed launch,
 * wait for them, and return the average duration of a launch in milliseconds.
 *   iolb_probe_hbm_copy: a streaming copy of `bytes` (a multiple of 16) from src to dst, device buffers
 *     that do not overlap; the traffic of a launch is 2 * bytes.
 *   iolb_probe_mfma_f32: a loop of independent v_mfma_f32_32x32x2_f32 with operands in registers; `sink`
 *     is a device buffer of at least iolb_probe_mfma_sink_bytes() bytes that receives the accumulators'
 *     sums; *flop_per_launch gets the floating-point operations of one launch.
 * IOLB_EINVAL for null pointers, bytes == 0 or not a multiple of 16, iters < 1, reps < 1. */
int iolb_probe_hbm_copy(const void* src, void* dst, size_t bytes, int reps, float* ms_per_launch);
size_t iolb_probe_mfma_sink_bytes(void);
int iolb_probe_mfma_f32(void* sink, int iters, int reps, float* ms_per_launch, double* flop_per_launch);

/* Probe of how the waves of one SIMD share its fp32 pipeline (the fused Winograd kernels of Sec. 5.3 mix matrix
 * and plain vector arithmetic in one workgroup; this measures what that costs).  One launch of 256 workgroups of
 * 4 * slots waves, so that every SIMD holds `slots` waves (1..4); the waves of slot s run roles[s] (a host array):
 * IOLB_PROBE_ROLE_MFMA = `iters` rounds of 8 v_mfma_f32_32x32x2_f32 (512 matrix cycles per round),
 * IOLB_PROBE_ROLE_VALU = `iters` rounds of 64 v_fma_f32.  `scratch` is a device buffer of at least
 * iolb_probe_share_scratch_bytes() bytes.  *ms gets the duration of the launch, ticks_per_slot[s] (host, `slots`
 * doubles) the average clock ticks a wave of slot s spent in its loop.  Runs on the set stream and waits for it.
 * IOLB_EINVAL for null pointers, slots outside 1..4, an unknown role, iters < 1. */
enum { IOLB_PROBE_ROLE_MFMA = 0, IOLB_PROBE_ROLE_VALU = 1 };
size_t iolb_probe_share_scratch_bytes(void);
int iolb_probe_pipeline_share(void* scratch, int slots, const int* roles, int iters, float* ms, double* ticks_per_slot);

/* Waits for the current GPU and frees the library's workspaces on it (all streams, and the buffers larger ones
 * have replaced); they are otherwise kept until the process ends.  Graphs captured from calls that used them
 * must not be replayed afterwards. */
int iolb_release_workspace(void);

const char* iolb_strerror(int code);
/* Text of the last HIP error seen by this thread's calls ("" if none). */
const char* iolb_last_hip_error(void);

#ifdef __cplusplus
}
#endif
#endif /* IOLBCONV_H */
