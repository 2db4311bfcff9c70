// Operands of dense layers laid out for the product kernel, and 8-bit checkpoints.  Streaming kernels: bound by memory.
#include "dense_math.h"
#include "kernels.h"

namespace iolb {

namespace {

// ---- layout -----------------------------------------------------------------------------------------
// A workgroup takes 64 x 64 values: a thread reads eight neighbouring columns of two rows, forms the values (a tensor's, a
// checkpoint's through an activation, or a gradient's through the activation's slope), and writes them as planes along the
// rows; the transposed planes go through LDS, and the column sums (the bias gradient's first stage) too.  The three layouts of a bf16
// gradient, M 8192, N 8192, K 4096 (dz both ways, the input and the weights transposed): 158 us in one launch, 587 MB, 3.7 TB/s.
constexpr int PITCH = 72;                          // 16-bit values of a transposed row in LDS: 144 bytes

template <class T>
__device__ __forceinline__ void store_eight(T* p, int have, const float (&v)[8])
{
    typename Piece<T, 8>::type t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (T)v[i];
    if (have >= 8) {
        *reinterpret_cast<typename Piece<T, 8>::type*>(p) = t;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) p[i] = t[i];
    }
}

typedef unsigned Codes __attribute__((ext_vector_type(2), aligned(1)));          // eight 8-bit codes, at any address

__device__ __forceinline__ void load_checkpoint(const int8_t* p, float unit, int have, float (&v)[8])
{
    if (have >= 8) {
        const Codes t = *reinterpret_cast<const Codes*>(p);
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = ckpt_value((int)(t[i / 4] << (24 - 8 * (i % 4))) >> 24, unit);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = i < have ? ckpt_value(p[i], unit) : 0.f;
    }
}

// 16-bit types: one part of the type, as a tensor of dz or of the layer's input would hold it in memory.  That is a second rounding beside the result's own, chosen
// because two parts would double the matrix work (8192 x 4096 -> 8192 bf16: some 830 of 987 us).  Error of the gradients against 64 bits, relative 2-norm, with
// unrounded operands / this: bf16 dx and dW through gelu 1.66e-3 / 2.33e-3, fp16 dW with the input through silu 2.07e-4 / 2.54e-4.  (A checkpoint's values
// are exact in either type they were packed from, also through relu; db is summed from the unrounded values.)
template <int DT>
__device__ __forceinline__ void plane_bits(float v, unsigned short (&bits)[DT == IOLB_F32 ? 3 : 1])
{
    if constexpr (DT == IOLB_F32) dense_parts(v, bits[0], bits[1], bits[2]);
    else if constexpr (DT == IOLB_F16) bits[0] = __builtin_bit_cast(unsigned short, (_Float16)v);
    else bits[0] = __builtin_bit_cast(unsigned short, (__bf16)v);
}

struct LayoutLaunch {
    DenseLayouts all;
    unsigned first[MAX_LAYOUTS];                   // workgroup at which each starts
};

template <int DT>
__global__ void __launch_bounds__(256)
dense_layout_kernel(LayoutLaunch launch)
{
    if (launch.all.uneven && !(launch.all.uneven[0] | launch.all.uneven[1])) return;
    typedef typename DenseType<DT>::type T;
    constexpr int PLANES = DT == IOLB_F32 ? 3 : 1;
    __shared__ __align__(16) unsigned short turned[PLANES][64][PITCH];
    __shared__ float sums[32][64 + 1];
    int which = 0;
#pragma unroll
    for (int i = 1; i < MAX_LAYOUTS; ++i) which = i < launch.all.count && blockIdx.x >= launch.first[i] ? i : which;
    const DenseLayout& g = launch.all.of[which];
    const unsigned block = blockIdx.x - launch.first[which], blocks_c = (unsigned)((g.cols + 63) / 64);
    const int tid = threadIdx.x, c8 = (tid & 7) * 8, r_in = tid >> 3;
    const int c0 = (int)(block % blocks_c) * 64, r0 = (int)(block / blocks_c) * 64;
    const int c = c0 + c8, have = g.cols - c;                      // may be negative
    const long long blocks_q = (g.cols + CKPT_BLOCK - 1) / CKPT_BLOCK;
    float column[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int half = 0; half < 2; ++half) {
        const int in = r_in + 32 * half, r = r0 + in;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        const bool live = r < g.rows && have > 0;
        if (live) {
            if (g.source != DENSE_FROM_CHECKPOINT) {
                const T* const from = static_cast<const T*>(g.src) + r * g.ld + c;
                if (sizeof(T) == 2 && g.odd && have >= 8) {
                    typedef T T8 __attribute__((ext_vector_type(8)));
                    if constexpr (sizeof(T) == 2) {
                        const T8 t = __builtin_bit_cast(T8, words_at_odd(from));
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = (float)t[i];
                    }
                } else {
                    load_columns(from, have, v);
                }
            }
            if (g.q) {
                float z[8];
                const float unit = two_to((int)g.e[r * blocks_q + c / CKPT_BLOCK] - 127);
                load_checkpoint(g.q + (long long)r * g.cols + c, unit, have, z);
                by_activation(g.act, [&](auto act) __attribute__((always_inline)) {
                    constexpr int ACT = decltype(act)::value;
                    if (g.source == DENSE_FROM_CHECKPOINT) {
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = activate<ACT>(z[i]);
                    } else {
#pragma unroll
                        for (int i = 0; i < 8; ++i) v[i] = i < have ? through_activation<ACT>(v[i], z[i]) : 0.f;
                    }
                });
            }
        }
        unsigned short bits[8][PLANES];
#pragma unroll
        for (int i = 0; i < 8; ++i) plane_bits<DT>(v[i], bits[i]);
        if (live && g.rowmajor) {
#pragma unroll
            for (int p = 0; p < PLANES; ++p) {
                u32x4 w;
#pragma unroll
                for (int i = 0; i < 4; ++i) w[i] = bits[2 * i][p] | (unsigned)bits[2 * i + 1][p] << 16;
                if (p < g.planes)
                    *reinterpret_cast<u32x4*>(static_cast<unsigned short*>(g.rowmajor) + (p * (long long)g.rows + r) * g.ld_rm + c) = w;
            }
        }
        if (live && g.copy) {
            store_eight(static_cast<T*>(g.copy) + (long long)r * g.cols + c, have, v);
        }
        if (g.transposed) {
#pragma unroll
            for (int p = 0; p < PLANES; ++p)
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (p < g.planes) turned[p][c8 + i][in] = bits[i][p];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) column[i] += v[i];
    }
    if (g.colsum || g.total) {
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[r_in][c8 + i] = column[i];
    }
    __syncthreads();
    if (g.transposed) {
        // 64 rows of 64 values: eight threads a row, two rows a thread
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int tc = r_in + 32 * half;
            if (c0 + tc < g.cols && r0 + c8 < g.rows) {
#pragma unroll
                for (int p = 0; p < PLANES; ++p)
                    if (p < g.planes)
                        *reinterpret_cast<u32x4*>(static_cast<unsigned short*>(g.transposed) + (p * (long long)g.cols + c0 + tc) * g.ld_tr + r0 + c8) =
                            *reinterpret_cast<const u32x4*>(&turned[p][tc][c8]);
            }
        }
    }
    if ((g.colsum || g.total) && tid < 64 && c0 + tid < g.cols) {
        float s = 0.f;
        for (int i = 0; i < 32; ++i) s += sums[i][tid];
        if (g.total) static_cast<T*>(g.total)[c0 + tid] = (T)s;
        else g.colsum[(long long)(r0 / 64) * g.cols + c0 + tid] = s;
    }
}

// Sixteen threads a group of 16 columns, in a fixed order.
template <int DT>
__global__ void __launch_bounds__(256)
dense_colsum_kernel(const float* colsum, int blocks, int cols, void* out)
{
    __shared__ float part[16][17];
    const int cx = threadIdx.x & 15, by = threadIdx.x >> 4, c = blockIdx.x * 16 + cx;
    float s = 0.f;
    if (c < cols)
        for (long long b = by; b < blocks; b += 16) s += colsum[b * cols + c];
    part[by][cx] = s;
    __syncthreads();
    if (by == 0 && c < cols) {
        s = 0.f;
        for (int i = 0; i < 16; ++i) s += part[i][cx];
        static_cast<typename DenseType<DT>::type*>(out)[c] = (typename DenseType<DT>::type)s;
    }
}

// ---- checkpoints -------------------------------------------------------------------------------------
// Four lanes share a block of 32, eight values each.  A workgroup covers `wide` threads of a row and 256 / wide rows.  Bound by memory:
// 16384 x 8192 bf16 81 us, 5.0 TB/s.
template <int DT>
__global__ void __launch_bounds__(256)
checkpoint_pack_kernel(const void* x, long long ldx, int rows, int cols, int8_t* q, uint8_t* e, int wide_log)
{
    typedef typename DenseType<DT>::type T;
    const int wide = 1 << wide_log, tx = threadIdx.x & (wide - 1), ty = threadIdx.x >> wide_log;
    const int c = (int)((blockIdx.x * (unsigned)wide + tx) * 8);
    const long long blocks = (cols + CKPT_BLOCK - 1) / CKPT_BLOCK;
    for (long long r = (long long)blockIdx.y * (256 >> wide_log) + ty; r - ty < rows; r += (long long)gridDim.y * (256 >> wide_log)) {
        const int have = r < rows ? cols - c : 0;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (have > 0) load_columns(static_cast<const T*>(x) + r * ldx + c, have, v);
        unsigned words[2];
        int ex;
        ckpt_codes<DT, 8, 4>(v, have, words, ex);
        if (have <= 0) continue;
        const Codes code = {words[0], words[1]};
        int8_t* const to = q + r * cols + c;
        if (have >= 8) {
            *reinterpret_cast<Codes*>(to) = code;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) to[i] = (int8_t)(code[i / 4] >> 8 * (i % 4));
        }
        if ((tx & 3) == 0) e[r * blocks + c / CKPT_BLOCK] = (uint8_t)(ex + 127);
    }
}

// Two lanes share a block, sixteen codes each, so that a lane's load is 16 bytes too.  16384 x 8192 to bf16: 84 us, 4.8 TB/s; through gelu 101, where
// the vector instructions count too.  (Eight codes a lane 107 without an activation, four rows of a lane at a time 156.)
template <int DT>
__global__ void __launch_bounds__(256)
checkpoint_unpack_kernel(const int8_t* q, const uint8_t* e, int rows, int cols, int act, void* y, long long ldy, int wide_log)
{
    typedef typename DenseType<DT>::type T;
    const int wide = 1 << wide_log, tx = threadIdx.x & (wide - 1), ty = threadIdx.x >> wide_log;
    const int c = (int)((blockIdx.x * (unsigned)wide + tx) * 16), have = cols - c;
    const long long blocks = (cols + CKPT_BLOCK - 1) / CKPT_BLOCK;
    if (have <= 0) return;
    for (long long r = (long long)blockIdx.y * (256 >> wide_log) + ty; r < rows; r += (long long)gridDim.y * (256 >> wide_log)) {
        const float unit = two_to((int)e[r * blocks + c / CKPT_BLOCK] - 127);
        const int8_t* const from = q + r * cols + c;
        float v[2][8];
        if (have >= 16) {
            const u32x4 t = words_at<4>(from);
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i / 8][i % 8] = ckpt_value((int)(t[i / 4] << (24 - 8 * (i % 4))) >> 24, unit);
        } else {
            load_checkpoint(from, unit, have, v[0]);
            load_checkpoint(from + 8, unit, have - 8, v[1]);
        }
        by_activation(act, [&](auto a) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < 16; ++i) v[i / 8][i % 8] = activate<decltype(a)::value>(v[i / 8][i % 8]);
        });
        T* const to = static_cast<T*>(y) + r * ldy + c;
        store_eight(to, have, v[0]);
        store_eight(to + 8, have - 8, v[1]);
    }
}

struct RowGrid { dim3 grid; int wide_log; };
// each: columns of a thread
RowGrid row_grid(int rows, int cols, long long each)
{
    int wide_log = 2;                               // whole blocks of 32
    while (wide_log < 8 && (each << wide_log) < cols) ++wide_log;
    const long long gx = (cols + (each << wide_log) - 1) / (each << wide_log), per = 256 >> wide_log;
    const long long gy = (rows + per - 1) / per;
    return {dim3((unsigned)gx, (unsigned)(gy < 65535 ? gy : 65535)), wide_log};
}

}  // namespace

hipError_t launch_dense_layouts(int dtype, const DenseLayouts& l, hipStream_t st)
{
    LayoutLaunch a{l, {}};
    long long n = 0;
    for (int i = 0; i < l.count; ++i) {
        a.all.of[i].odd = reinterpret_cast<uintptr_t>(l.of[i].src) % 4 || l.of[i].ld % 2;
        a.first[i] = (unsigned)n;
        n += ((l.of[i].cols + 63LL) / 64) * ((l.of[i].rows + 63LL) / 64);
        if (n > 0x7fffffffLL) return hipErrorInvalidValue;
    }
    if (n == 0) return hipSuccess;
    if (dtype == IOLB_F32) dense_layout_kernel<IOLB_F32><<<(unsigned)n, 256, 0, st>>>(a);
    else if (dtype == IOLB_F16) dense_layout_kernel<IOLB_F16><<<(unsigned)n, 256, 0, st>>>(a);
    else dense_layout_kernel<IOLB_BF16><<<(unsigned)n, 256, 0, st>>>(a);
    return hipGetLastError();
}

hipError_t launch_dense_colsum(const float* colsum, int blocks, int cols, void* out, int dtype, hipStream_t st)
{
    const unsigned n = (unsigned)((cols + 15) / 16);
    if (dtype == IOLB_F32) dense_colsum_kernel<IOLB_F32><<<n, 256, 0, st>>>(colsum, blocks, cols, out);
    else if (dtype == IOLB_F16) dense_colsum_kernel<IOLB_F16><<<n, 256, 0, st>>>(colsum, blocks, cols, out);
    else dense_colsum_kernel<IOLB_BF16><<<n, 256, 0, st>>>(colsum, blocks, cols, out);
    return hipGetLastError();
}

hipError_t launch_checkpoint_pack(const void* x, long long ldx, int rows, int cols, int dtype, int8_t* q, uint8_t* e, hipStream_t st)
{
    const RowGrid g = row_grid(rows, cols, 8);
    if (dtype == IOLB_F32) checkpoint_pack_kernel<IOLB_F32><<<g.grid, 256, 0, st>>>(x, ldx, rows, cols, q, e, g.wide_log);
    else if (dtype == IOLB_F16) checkpoint_pack_kernel<IOLB_F16><<<g.grid, 256, 0, st>>>(x, ldx, rows, cols, q, e, g.wide_log);
    else checkpoint_pack_kernel<IOLB_BF16><<<g.grid, 256, 0, st>>>(x, ldx, rows, cols, q, e, g.wide_log);
    return hipGetLastError();
}

hipError_t launch_checkpoint_unpack(const int8_t* q, const uint8_t* e, int rows, int cols, int act, int dtype, void* y, long long ldy,
                                    hipStream_t st)
{
    const RowGrid g = row_grid(rows, cols, 16);
    if (dtype == IOLB_F32) checkpoint_unpack_kernel<IOLB_F32><<<g.grid, 256, 0, st>>>(q, e, rows, cols, act, y, ldy, g.wide_log);
    else if (dtype == IOLB_F16) checkpoint_unpack_kernel<IOLB_F16><<<g.grid, 256, 0, st>>>(q, e, rows, cols, act, y, ldy, g.wide_log);
    else checkpoint_unpack_kernel<IOLB_BF16><<<g.grid, 256, 0, st>>>(q, e, rows, cols, act, y, ldy, g.wide_log);
    return hipGetLastError();
}

}  // namespace iolb
