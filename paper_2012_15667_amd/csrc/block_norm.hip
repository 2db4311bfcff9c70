// Norms before and after a block with its gate and residual scale, and their gradients.  Streaming kernels: bound by memory.
#include "block.h"
#include "dense_math.h"

namespace iolb {

namespace {

// v added over the lane's sixteen neighbours (DPP), then over the wave.  All lanes get the sum, in an order that does not depend on anything.
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v)
{
    return v + __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), CTRL, 0xf, 0xf, true));
}

__device__ __forceinline__ float sum_16(float v)
{
    v = dpp_add<0xb1>(v);                           // quad_perm [1,0,3,2]
    v = dpp_add<0x4e>(v);                           // quad_perm [2,3,0,1]
    v = dpp_add<0x141>(v);                          // row_half_mirror
    return dpp_add<0x140>(v);                       // row_mirror
}

__device__ __forceinline__ float lane_value(float v, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); }

__device__ __forceinline__ float sum_64(float v)
{
    v = sum_16(v);
    return (lane_value(v, 0) + lane_value(v, 16)) + (lane_value(v, 32) + lane_value(v, 48));
}

// K values added over the TR threads of a row: sixteen lanes, a wave, or a workgroup of TR threads.
template <int K, int TR>
struct RowSum {
    static constexpr int WAVES = TR / 64;
    typedef float Part[2][K][WAVES > 1 ? WAVES : 1];
    Part& part;
    int turn = 0;
    // (two buffers in turn: who writes one again has passed the barrier behind all reads of it)
    template <int N>
    __device__ __forceinline__ void operator()(float (&v)[N])
    {
        static_assert(N <= K, "room for as many");
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = TR == 16 ? sum_16(v[k]) : sum_64(v[k]);
        if constexpr (WAVES > 1) {
            if ((threadIdx.x & 63) == 0) {
#pragma unroll
                for (int k = 0; k < N; ++k) part[turn][k][threadIdx.x >> 6] = v[k];
            }
            __syncthreads();
#pragma unroll
            for (int k = 0; k < N; ++k) {
                v[k] = 0.f;
#pragma unroll
                for (int i = 0; i < WAVES; ++i) v[k] += part[turn][k][i];
            }
            turn ^= 1;
        }
    }
};

struct RowStats { float mean, r; };

// v normalised is (v - mean) r.
template <int DT, class F>
__device__ __forceinline__ RowStats stats_of(const typename DenseType<DT>::type* row, int N, int kind, float eps, F sum)
{
    if (kind == IOLB_NORM_NONE) return {0.f, 1.f};
    float mean = 0.f;
    if (kind == IOLB_NORM_LAYER) {
        float s = 0.f;
        for (int c = threadIdx.x * 8; c < N; c += blockDim.x * 8) {
            float v[8];
            load_columns(row + c, N - c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) s += v[i];
        }
        mean = sum(s) / (float)N;
    }
    float s = 0.f;
    for (int c = threadIdx.x * 8; c < N; c += blockDim.x * 8) {
        float v[8];
        load_columns(row + c, N - c, v);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = c + i < N ? v[i] - mean : 0.f;
            s = __builtin_fmaf(d, d, s);
        }
    }
    return {mean, 1.f / sqrtf(sum(s) / (float)N + eps)};
}

// Eight columns of a weight, a bias or a gate; `or_else` where there is none.
template <class T>
__device__ __forceinline__ void load_or(const T* p, int c, int N, float or_else, float (&v)[8])
{
    if (p) {
        load_columns(p + c, N - c, v);
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = or_else;
    }
}

// PAST: past the caches, where the tensors of a call are more than those hold.
template <bool PAST = false, class T>
__device__ __forceinline__ void store_eight_of(T* p, int have, const typename Piece<T, 8>::type& t)
{
    if (have >= 8) {
        if constexpr (PAST) __builtin_nontemporal_store(t, reinterpret_cast<typename Piece<T, 8>::type*>(p));
        else *reinterpret_cast<typename Piece<T, 8>::type*>(p) = t;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < have) p[i] = t[i];
    }
}

template <class T>
__device__ __forceinline__ void store_columns_of(T* p, int have, const float (&v)[8])
{
    typename Piece<T, 8>::type t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = (T)v[i];
    store_eight_of(p, have, t);
}

// ---- rows in registers ------------------------------------------------------------------------------------
// How rows end: after a whole piece of eight values; within one; or within the first.
enum RowEnd { WHOLE, CUT, SHORT };

// Eight neighbouring values as they are in memory; zeros beyond the row's end.  A last piece that is cut is read in one access that ends with the row, and
// settle_eight moves its values to their places, once other loads are on their way.  16-bit rows of 4094 values, 8192 of them: value by value 64 us, gradients
// 116, so 54 / 99; of 1001, 20000 of them, 39 / 72 and 35 / 62.  (With this in the kernel of whole rows those would hold twice the registers.)
template <class T> using Eight = typename Piece<T, 8>::type;

template <int ENDS, class T>
__device__ __forceinline__ Eight<T> load_eight(const T* row, int at, int N)
{
    Eight<T> t = {};
    if constexpr (ENDS == SHORT) {
#pragma unroll
        for (int i = 0; i < 8; ++i) t[i] = at + i < N ? row[at + i] : (T)0.f;
    } else if (at < N) {
        t = *reinterpret_cast<const Eight<T>*>(row + (ENDS == WHOLE || at < N - 8 ? at : N - 8));
    }
    return t;
}

// The values moved down by BY places, with zeros behind them.
template <int BY, class T>
__device__ __forceinline__ void move_down(Eight<T>& t)
{
    constexpr int W = 2 * sizeof(T), STEP = BY * (int)sizeof(T) / 4;    // words; words to move by, or half a word
    typedef unsigned Words __attribute__((ext_vector_type(W)));
    const Words w = __builtin_bit_cast(Words, t);
    Words to;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        if constexpr (STEP == 0) to[i] = __builtin_amdgcn_alignbyte(i + 1 < W ? w[i + 1 < W ? i + 1 : 0] : 0, w[i], 2);
        else to[i] = i + STEP < W ? w[i + STEP < W ? i + STEP : 0] : 0;
    }
    t = __builtin_bit_cast(Eight<T>, to);
}

template <int ENDS, class T>
__device__ __forceinline__ void settle_eight(Eight<T>& t, int at, int N)
{
    if constexpr (ENDS == CUT) {
        if (at == N - (N & 7)) {
            const int by = 8 - (N & 7);
            if (by & 4) move_down<4, T>(t);
            if (by & 2) move_down<2, T>(t);
            if (by & 1) move_down<1, T>(t);
        }
    }
}

// A row's values, TR threads to a row, C times eight a thread: c-th piece at column 8 (c TR + thread).
template <class T, int C> struct Row { Eight<T> of[C]; };

template <int TR, int C, int ENDS, class T>
__device__ __forceinline__ void load_row(const T* p, int N, int thread, Row<T, C>& row)
{
#pragma unroll
    for (int c = 0; c < C; ++c) {
        const int at = 8 * (c * TR + thread);
        row.of[c] = load_eight<ENDS>(p, at, N);
    }
}

template <int TR, int C, int ENDS, class T>
__device__ __forceinline__ void settle(Row<T, C>& row, int N, int thread)
{
#pragma unroll
    for (int c = 0; c < C; ++c) settle_eight<ENDS, T>(row.of[c], 8 * (c * TR + thread), N);
}

// A weight's, a bias's or a gate's values; `or_else` where there is none.
template <int TR, int C, int ENDS, class T>
__device__ __forceinline__ void load_row_or(const T* p, int N, int thread, float or_else, Row<T, C>& row)
{
    if (p) {
        load_row<TR, C, ENDS>(p, N, thread, row);
    } else {
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) row.of[c][i] = (T)or_else;
    }
}

// Keeps the compiler from holding the values in 32 bits across a step: they are taken from what is in memory's form again, for half the registers.
template <class T, int C>
__device__ __forceinline__ void hold(Row<T, C>& row)
{
    if constexpr (sizeof(T) == 2) {
#pragma unroll
        for (int c = 0; c < C; ++c) {
            u32x4 w = __builtin_bit_cast(u32x4, row.of[c]);
            asm volatile("" : "+v"(w));
            row.of[c] = __builtin_bit_cast(Eight<T>, w);
        }
    }
}

// (v - mean) r is the row normalised; v [C][8] in 32 bits, zeros beyond the end.
template <int TR, int C, class S>
__device__ __forceinline__ RowStats stats_of_row(float (&v)[C][8], int N, int thread, int kind, float eps, S& sum)
{
    float one[1];
    float mean = 0.f;
    if (kind == IOLB_NORM_LAYER) {
        one[0] = 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) one[0] += v[c][i];
        sum(one);
        mean = one[0] / (float)N;
    }
    one[0] = 0.f;
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float d = 8 * (c * TR + thread) + i < N ? v[c][i] - mean : 0.f;
            one[0] = __builtin_fmaf(d, d, one[0]);
        }
    sum(one);
    return {mean, 1.f / sqrtf(one[0] / (float)N + eps)};
}

// One pass: the row stays in registers from its loads to its stores, and the threads of a row join two sums (four with the mean taken off).  Bound by memory:
// 8192 x 4096 bf16 51 us, 5.3 TB/s; 1 x 4096 4.0 us, two trips to memory and the exchanges.
template <int DT, int TR, int C, int ENDS, bool PAST>
__global__ void __launch_bounds__(TR > 256 ? TR : 256)
block_norm_rows_kernel(BlockNorm p)
{
    typedef typename DenseType<DT>::type T;
    constexpr int ROWS = TR > 256 ? 1 : 256 / TR;
    __shared__ typename RowSum<1, TR>::Part part;
    RowSum<1, TR> sum{part};
    const int thread = threadIdx.x % TR;
    // (more than a wave to a row: all threads of the workgroup alike)
    for (long long m = (long long)blockIdx.x * ROWS + threadIdx.x / TR; m < p.M; m += (long long)gridDim.x * ROWS) {
        Row<T, C> x, w, b;
        load_row<TR, C, ENDS>(static_cast<const T*>(p.x) + m * p.ldx, p.N, thread, x);
        float v[C][8];
        if (p.h) {
            Row<T, C> h, g;
            load_row<TR, C, ENDS>(static_cast<const T*>(p.h) + m * p.ldh, p.N, thread, h);
            load_row_or<TR, C, ENDS>(static_cast<const T*>(p.post_weight), p.N, thread, 1.f, w);
            load_row_or<TR, C, ENDS>(p.gate ? static_cast<const T*>(p.gate) + m / p.rows_per_group * p.N : nullptr, p.N, thread, 1.f, g);
            settle<TR, C, ENDS>(x, p.N, thread);
            settle<TR, C, ENDS>(h, p.N, thread);
            settle<TR, C, ENDS>(w, p.N, thread);
            settle<TR, C, ENDS>(g, p.N, thread);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = (float)h.of[c][i];
            RowStats s{0.f, 1.f};
            if (p.post != IOLB_NORM_NONE) s = stats_of_row<TR, C>(v, p.N, thread, p.post, p.eps, sum);
#pragma unroll
            for (int c = 0; c < C; ++c) {
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = (v[c][i] - s.mean) * s.r * (float)w.of[c][i];
                const int at = 8 * (c * TR + thread);
                if (p.post_bias) {
                    Eight<T> bias = load_eight<ENDS>(static_cast<const T*>(p.post_bias), at, p.N);
                    settle_eight<ENDS, T>(bias, at, p.N);
#pragma unroll
                    for (int i = 0; i < 8; ++i) v[c][i] += (float)bias[i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[c][i] = p.scale * (float)x.of[c][i] + (float)g.of[c][i] * v[c][i];
                    x.of[c][i] = (T)v[c][i];
                    v[c][i] = at + i < p.N ? (float)x.of[c][i] : 0.f;       // (as rounded: what a backward pass reads is what is normalised)
                }
                store_eight_of<PAST>(static_cast<T*>(p.out) + m * p.ldo + at, p.N - at, x.of[c]);
            }
        } else {
            settle<TR, C, ENDS>(x, p.N, thread);
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[c][i] = (float)x.of[c][i];
        }
        if (!p.y) continue;
        load_row_or<TR, C, ENDS>(static_cast<const T*>(p.pre_weight), p.N, thread, 1.f, w);
        load_row_or<TR, C, ENDS>(static_cast<const T*>(p.pre_bias), p.N, thread, 0.f, b);
        settle<TR, C, ENDS>(w, p.N, thread);
        settle<TR, C, ENDS>(b, p.N, thread);
        const RowStats s = stats_of_row<TR, C>(v, p.N, thread, p.pre, p.eps, sum);
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = 8 * (c * TR + thread);
#pragma unroll
            for (int i = 0; i < 8; ++i) x.of[c][i] = (T)((v[c][i] - s.mean) * s.r * (float)w.of[c][i] + (float)b.of[c][i]);
            store_eight_of<PAST>(static_cast<T*>(p.y) + m * p.ldy + at, p.N - at, x.of[c]);
        }
    }
}

// ---- rows of any length ------------------------------------------------------------------------------------
// A workgroup to a row, which it reads again from the caches for each step: 2048 x 20000 bf16 114 us (2.9 TB/s), gradients with the columns' pass 320.
template <int DT>
__global__ void __launch_bounds__(256)
block_norm_long_kernel(BlockNorm p)
{
    typedef typename DenseType<DT>::type T;
    __shared__ RowSum<1, 256>::Part part;
    RowSum<1, 256> sums{part};
    const auto sum = [&](float v) {
        float one[1] = {v};
        sums(one);
        return one[0];
    };
    for (long long m = blockIdx.x; m < p.M; m += gridDim.x) {
        const T* from = static_cast<const T*>(p.x) + m * p.ldx;
        if (p.h) {
            const T* const h = static_cast<const T*>(p.h) + m * p.ldh;
            T* const out = static_cast<T*>(p.out) + m * p.ldo;
            const T* const gate = p.gate ? static_cast<const T*>(p.gate) + m / p.rows_per_group * p.N : nullptr;
            const RowStats s = stats_of<DT>(h, p.N, p.post, p.eps, sum);
            for (int c = threadIdx.x * 8; c < p.N; c += 256 * 8) {
                float x[8], v[8], w[8], b[8], g[8];
                load_columns(from + c, p.N - c, x);
                load_columns(h + c, p.N - c, v);
                load_or(static_cast<const T*>(p.post_weight), c, p.N, 1.f, w);
                load_or(static_cast<const T*>(p.post_bias), c, p.N, 0.f, b);
                load_or(gate, c, p.N, 1.f, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = p.scale * x[i] + g[i] * ((v[i] - s.mean) * s.r * w[i] + b[i]);
                store_columns_of(out + c, p.N - c, x);
            }
            from = out;                                 // (a thread reads what it wrote itself)
        }
        if (p.y) {
            const RowStats s = stats_of<DT>(from, p.N, p.pre, p.eps, sum);
            for (int c = threadIdx.x * 8; c < p.N; c += 256 * 8) {
                float v[8], w[8], b[8];
                load_columns(from + c, p.N - c, v);
                load_or(static_cast<const T*>(p.pre_weight), c, p.N, 1.f, w);
                load_or(static_cast<const T*>(p.pre_bias), c, p.N, 0.f, b);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = (v[i] - s.mean) * s.r * w[i] + b[i];
                store_columns_of(static_cast<T*>(p.y) + m * p.ldy + c, p.N - c, v);
            }
        }
    }
}

// ---- gradients -----------------------------------------------------------------------------------------
// With hat = (v - mean) r and its gradient t, v gets r (t - hat mean(t hat) - mean(t)), the last for IOLB_NORM_LAYER alone.
struct RowSums { float mean_x, r_x, along_x, mean_d, mean_h, r_h, along_h, mean_p; };
static_assert(sizeof(RowSums) == 4 * NORM_ROW_SUMS, "as the workspace counts them");

template <int DT>
__device__ __forceinline__ void gradient_of_out(const BlockNormBackward& p, long long m, int c, const RowSums& s, float (&d)[8], float (&hat)[8], float (&dy)[8])
{
    typedef typename DenseType<DT>::type T;
    const int have = p.N - c;
    if (p.dout) load_columns(static_cast<const T*>(p.dout) + m * p.lddout + c, have, d);
    else {
#pragma unroll
        for (int i = 0; i < 8; ++i) d[i] = 0.f;
    }
    if (!p.dy) return;
    float w[8];
    load_columns(static_cast<const T*>(p.x) + m * p.ldx + c, have, hat);
    load_columns(static_cast<const T*>(p.dy) + m * p.lddy + c, have, dy);
    load_or(static_cast<const T*>(p.pre_weight), c, p.N, 1.f, w);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        hat[i] = (hat[i] - s.mean_x) * s.r_x;
        d[i] += s.r_x * (dy[i] * w[i] - hat[i] * s.along_x - s.mean_d);
    }
}

template <int DT>
__global__ void __launch_bounds__(256)
norm_backward_long_kernel(BlockNormBackward p)
{
    typedef typename DenseType<DT>::type T;
    __shared__ RowSum<1, 256>::Part part;
    RowSum<1, 256> sums{part};
    const auto sum = [&](float v) {
        float one[1] = {v};
        sums(one);
        return one[0];
    };
    const float per = 1.f / (float)p.N;
    for (long long m = blockIdx.x; m < p.M; m += gridDim.x) {
        RowSums s{0.f, 1.f, 0.f, 0.f, 0.f, 1.f, 0.f, 0.f};
        if (p.dy) {
            const T* const x = static_cast<const T*>(p.x) + m * p.ldx;
            const T* const dys = static_cast<const T*>(p.dy) + m * p.lddy;
            const RowStats t = stats_of<DT>(x, p.N, p.pre, p.eps, sum);
            s.mean_x = t.mean; s.r_x = t.r;
            float along = 0.f, all = 0.f;
            for (int c = threadIdx.x * 8; c < p.N; c += 256 * 8) {
                float v[8], dy[8], w[8];
                load_columns(x + c, p.N - c, v);
                load_columns(dys + c, p.N - c, dy);             // (0 beyond the row)
                load_or(static_cast<const T*>(p.pre_weight), c, p.N, 1.f, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    along += dy[i] * w[i] * ((v[i] - t.mean) * t.r);
                    all += dy[i] * w[i];
                }
            }
            s.along_x = sum(along) * per;
            if (p.pre == IOLB_NORM_LAYER) s.mean_d = sum(all) * per;
        }
        const T* const gate = p.gate ? static_cast<const T*>(p.gate) + m / p.rows_per_group * p.N : nullptr;
        const T* const h = static_cast<const T*>(p.h) + m * p.ldh;
        if (p.h && p.post != IOLB_NORM_NONE) {
            const RowStats t = stats_of<DT>(h, p.N, p.post, p.eps, sum);
            s.mean_h = t.mean; s.r_h = t.r;
            float along = 0.f, all = 0.f;
            for (int c = threadIdx.x * 8; c < p.N; c += 256 * 8) {
                float d[8], hat[8], dy[8], v[8], w[8], g[8];
                gradient_of_out<DT>(p, m, c, s, d, hat, dy);
                load_columns(h + c, p.N - c, v);
                load_or(static_cast<const T*>(p.post_weight), c, p.N, 1.f, w);
                load_or(gate, c, p.N, 1.f, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float t1 = c + i < p.N ? d[i] * g[i] * w[i] : 0.f;
                    along += t1 * ((v[i] - t.mean) * t.r);
                    all += t1;
                }
            }
            s.along_h = sum(along) * per;
            if (p.post == IOLB_NORM_LAYER) s.mean_p = sum(all) * per;
        }
        for (int c = threadIdx.x * 8; c < p.N && (p.dx || p.dh); c += 256 * 8) {
            float d[8], hat[8], dy[8];
            gradient_of_out<DT>(p, m, c, s, d, hat, dy);
            if (p.dh) {
                float v[8], w[8], g[8], to[8];
                load_columns(h + c, p.N - c, v);
                load_or(static_cast<const T*>(p.post_weight), c, p.N, 1.f, w);
                load_or(gate, c, p.N, 1.f, g);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float t1 = d[i] * g[i] * w[i];
                    to[i] = p.post == IOLB_NORM_NONE ? t1 : s.r_h * (t1 - (v[i] - s.mean_h) * s.r_h * s.along_h - s.mean_p);
                }
                store_columns_of(static_cast<T*>(p.dh) + m * p.N + c, p.N - c, to);
            }
            if (p.dx) {
#pragma unroll
                for (int i = 0; i < 8; ++i) d[i] *= p.scale;
                store_columns_of(static_cast<T*>(p.dx) + m * p.N + c, p.N - c, d);
            }
        }
        if (p.rows && threadIdx.x == 0) reinterpret_cast<RowSums*>(p.rows)[m] = s;
    }
}

enum { S1, S0, T1, T0 };

// A workgroup takes 64 columns of a piece's rows: eight threads across, 32 along.
template <int DT>
__global__ void __launch_bounds__(256)
norm_backward_columns_kernel(BlockNormBackward p, NormPieces pieces)
{
    typedef typename DenseType<DT>::type T;
    __shared__ float part[32][64 + 1];
    const unsigned across = (unsigned)(p.N + 63) / 64, row = blockIdx.x / across, c0 = blockIdx.x % across * 64;
    const int tx = threadIdx.x & 7, ty = threadIdx.x >> 3, c = (int)c0 + tx * 8;
    const long long ld = (p.N + 7) / 8 * 8;
    const int group = (int)(row / pieces.in_group), piece = (int)(row % pieces.in_group);
    const long long first = (long long)group * p.rows_per_group, r0 = first + (long long)piece * pieces.per;
    const long long r1 = r0 + pieces.per < first + p.rows_per_group ? r0 + pieces.per : first + p.rows_per_group;
    float sums[NORM_COLUMN_SUMS][8];
#pragma unroll
    for (int k = 0; k < NORM_COLUMN_SUMS; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) sums[k][i] = 0.f;
    if (c < p.N)
        for (long long m = r0 + ty; m < r1; m += 32) {
            const RowSums s = reinterpret_cast<const RowSums*>(p.rows)[m];
            float d[8], hat[8], dy[8];
            gradient_of_out<DT>(p, m, c, s, d, hat, dy);
            if (p.h) {
                float v[8];
                load_columns(static_cast<const T*>(p.h) + m * p.ldh + c, p.N - c, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sums[S1][i] += d[i] * ((v[i] - s.mean_h) * s.r_h);
                    sums[S0][i] += d[i];
                }
            }
            if (p.dy) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sums[T1][i] += dy[i] * hat[i];
                    sums[T0][i] += dy[i];
                }
            }
        }
#pragma unroll
    for (int k = 0; k < NORM_COLUMN_SUMS; ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 8; ++i) part[ty][tx * 8 + i] = sums[k][i];
        __syncthreads();
        const int n = (int)c0 + threadIdx.x;
        if (threadIdx.x < 64 && n < p.N) {
            float t = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) t += part[i][threadIdx.x];
            p.columns[((long long)row * NORM_COLUMN_SUMS + k) * ld + n] = t;
        }
    }
}

// The same for rows that are held in registers: a workgroup takes a piece's rows, TR threads to a row, reads everything once, and holds its columns' sums
// meanwhile; the next row's values are asked for where this row's have been used last.  BIASES: whether S0 and T0 are wanted.
// Memory and a row's two exchanges bind it: 8192 x 4096 bf16 86 to 95 us (4.2 to 4.7 TB/s), and 8 to join the pieces' sums.  fp32 (a call): 8192 x 4096 176 us,
// with means off and biases 191; of 4097 to 8192 values some of a row's do not fit the registers, 38 to 41 of a lane's, with biases 116 to 129: 4096 x 8192 189 / 257.
template <int DT, int TR, int C, bool BIASES, int ENDS, bool PAST>
__global__ void __launch_bounds__(TR > 256 ? TR : 256)
norm_backward_rows_kernel(BlockNormBackward p, NormPieces pieces, unsigned wanted)
{
    typedef typename DenseType<DT>::type T;
    constexpr int ROWS = TR > 256 ? 1 : 256 / TR;
    __shared__ typename RowSum<4, TR>::Part part;
    RowSum<4, TR> sum{part};
    const int thread = threadIdx.x % TR, slot = threadIdx.x / TR;
    const int group = (int)(blockIdx.x / (unsigned)pieces.in_group), piece = (int)(blockIdx.x % (unsigned)pieces.in_group);
    const long long first = (long long)group * p.rows_per_group, r0 = first + (long long)piece * pieces.per;
    const long long r1 = r0 + pieces.per < first + p.rows_per_group ? r0 + pieces.per : first + p.rows_per_group;
    const float per = 1.f / (float)p.N;

    Row<T, C> w, wp, g;
    load_row_or<TR, C, ENDS>(static_cast<const T*>(p.pre_weight), p.N, thread, 1.f, w);
    load_row_or<TR, C, ENDS>(static_cast<const T*>(p.post_weight), p.N, thread, 1.f, wp);
    load_row_or<TR, C, ENDS>(p.gate ? static_cast<const T*>(p.gate) + (long long)group * p.N : nullptr, p.N, thread, 1.f, g);
    settle<TR, C, ENDS>(w, p.N, thread);
    settle<TR, C, ENDS>(wp, p.N, thread);
    settle<TR, C, ENDS>(g, p.N, thread);
    float s1[C][8], t1[C][8], s0[BIASES ? C : 1][8], t0[BIASES ? C : 1][8];
#pragma unroll
    for (int c = 0; c < C; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            s1[c][i] = t1[c][i] = 0.f;
            if constexpr (BIASES) s0[c][i] = t0[c][i] = 0.f;
        }
    struct Rows { Row<T, C> x, h, dy, dout; };
    Rows r{};
    const auto load_x = [&](long long m) {
        if (m >= r1) return;
        if (p.dy) {
            load_row<TR, C, ENDS>(static_cast<const T*>(p.x) + m * p.ldx, p.N, thread, r.x);
            load_row<TR, C, ENDS>(static_cast<const T*>(p.dy) + m * p.lddy, p.N, thread, r.dy);
        }
        if (p.dout) load_row<TR, C, ENDS>(static_cast<const T*>(p.dout) + m * p.lddout, p.N, thread, r.dout);
    };
    const auto load_h = [&](long long m) {
        if (m < r1 && p.h) load_row<TR, C, ENDS>(static_cast<const T*>(p.h) + m * p.ldh, p.N, thread, r.h);
    };
    load_x(r0 + slot);
    load_h(r0 + slot);
    for (long long m = r0 + slot; m < r1; m += ROWS) {
        settle<TR, C, ENDS>(r.x, p.N, thread);
        settle<TR, C, ENDS>(r.h, p.N, thread);
        settle<TR, C, ENDS>(r.dy, p.N, thread);
        settle<TR, C, ENDS>(r.dout, p.N, thread);
        hold(w);
        hold(wp);
        hold(g);
        float mean_x = 0.f, mean_h = 0.f;
        if (p.pre == IOLB_NORM_LAYER || p.post == IOLB_NORM_LAYER) {
            float v[2] = {0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[0] += (float)r.x.of[c][i];
                    v[1] += (float)r.h.of[c][i];
                }
            sum(v);
            if (p.pre == IOLB_NORM_LAYER) mean_x = v[0] * per;
            if (p.post == IOLB_NORM_LAYER) mean_h = v[1] * per;
        }
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool live = 8 * (c * TR + thread) + i < p.N;
                const float x = live ? (float)r.x.of[c][i] - mean_x : 0.f, h = live ? (float)r.h.of[c][i] - mean_h : 0.f;
                const float t = (float)r.dy.of[c][i] * (float)w.of[c][i];
                v[0] = __builtin_fmaf(x, x, v[0]);
                v[1] = __builtin_fmaf(t, x, v[1]);
                v[2] += t;
                v[3] = __builtin_fmaf(h, h, v[3]);
            }
        sum(v);
        const float r_x = p.dy ? 1.f / sqrtf(v[0] * per + p.eps) : 0.f, along_x = v[1] * r_x * per, mean_d = p.pre == IOLB_NORM_LAYER ? v[2] * per : 0.f;
        const float r_h = p.post != IOLB_NORM_NONE ? 1.f / sqrtf(v[3] * per + p.eps) : 1.f;
        hold(r.x);
        hold(r.h);
        hold(r.dy);
        float d[C][8], u[2] = {0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool live = 8 * (c * TR + thread) + i < p.N;
                const float dy = (float)r.dy.of[c][i], hat_x = ((float)r.x.of[c][i] - mean_x) * r_x, hat_h = ((float)r.h.of[c][i] - mean_h) * r_h;
                d[c][i] = live ? (float)r.dout.of[c][i] + r_x * (dy * (float)w.of[c][i] - hat_x * along_x - mean_d) : 0.f;
                s1[c][i] = __builtin_fmaf(d[c][i], hat_h, s1[c][i]);
                t1[c][i] = __builtin_fmaf(dy, hat_x, t1[c][i]);
                if constexpr (BIASES) {
                    s0[c][i] += d[c][i];
                    t0[c][i] += dy;
                }
                const float t = d[c][i] * (float)g.of[c][i] * (float)wp.of[c][i];
                u[0] = __builtin_fmaf(t, hat_h, u[0]);
                u[1] += t;
            }
        load_x(m + ROWS);
        if (p.post != IOLB_NORM_NONE) sum(u);
        hold(r.h);
        hold(g);
        hold(wp);
        const float along_h = p.post != IOLB_NORM_NONE ? u[0] * per : 0.f, mean_p = p.post == IOLB_NORM_LAYER ? u[1] * per : 0.f;
#pragma unroll
        for (int c = 0; c < C; ++c) {
            const int at = 8 * (c * TR + thread);
            Eight<T> to;
            if (p.dh) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float hat_h = ((float)r.h.of[c][i] - mean_h) * r_h, t = d[c][i] * (float)g.of[c][i] * (float)wp.of[c][i];
                    to[i] = (T)(r_h * (t - hat_h * along_h - mean_p));
                }
                store_eight_of<PAST>(static_cast<T*>(p.dh) + m * p.N + at, p.N - at, to);
            }
            if (p.dx) {
#pragma unroll
                for (int i = 0; i < 8; ++i) to[i] = (T)(p.scale * d[c][i]);
                store_eight_of<PAST>(static_cast<T*>(p.dx) + m * p.N + at, p.N - at, to);
            }
        }
        load_h(m + ROWS);
    }
    if (!wanted) return;
    // the rows' sums joined where several rows were taken at a time, and written
    const long long ld = (p.N + 7) / 8 * 8;
    float* const out = p.columns + (long long)blockIdx.x * NORM_COLUMN_SUMS * ld;
    const auto put = [&](int k, const float (&v)[C][8]) {
        if (!(wanted >> k & 1)) return;
        if constexpr (ROWS == 1) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = 8 * (c * TR + thread);
                if (at < p.N) {
                    *reinterpret_cast<f32x4*>(out + k * ld + at) = f32x4{v[c][0], v[c][1], v[c][2], v[c][3]};
                    *reinterpret_cast<f32x4*>(out + k * ld + at + 4) = f32x4{v[c][4], v[c][5], v[c][6], v[c][7]};
                }
            }
        } else {
            __shared__ float all[ROWS][8 * TR * C];
            __syncthreads();
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) all[slot][8 * (c * TR + thread) + i] = v[c][i];
            __syncthreads();
            for (int n = threadIdx.x; n < 8 * TR * C && n < p.N; n += 256) {
                float t = 0.f;
#pragma unroll
                for (int i = 0; i < ROWS; ++i) t += all[i][n];
                out[k * ld + n] = t;
            }
        }
    };
    put(S1, s1);
    put(T1, t1);
    if constexpr (BIASES) {
        put(S0, s0);
        put(T0, t0);
    }
}

// Rows whose columns' sums do not fit beside them: a workgroup of 1024 to a row, which it reads once.  The sums are another pass, which reads all again.
// 16-bit rows leave registers for the next row to be asked for meanwhile; 32-bit ones do not.  2048 x 16384 bf16 162 us (both passes; a row read again
// for each step 240), 1640 x 14640 fp32 222 (317), 64 x 10000 bf16 22 (37).
template <int DT, int C, int ENDS>
__global__ void __launch_bounds__(1024)
norm_backward_wide_kernel(BlockNormBackward p)
{
    typedef typename DenseType<DT>::type T;
    constexpr int TR = 1024;
    constexpr bool AHEAD = sizeof(T) == 2;
    __shared__ typename RowSum<4, TR>::Part part;
    RowSum<4, TR> sum{part};
    const int thread = threadIdx.x;
    const float per = 1.f / (float)p.N;
    Row<T, C> x{}, h{}, dy{}, dout{}, w, g;
    const auto load_x = [&](long long m) {
        if (m >= p.M) return;
        if (p.dy) {
            load_row<TR, C, ENDS>(static_cast<const T*>(p.x) + m * p.ldx, p.N, thread, x);
            load_row<TR, C, ENDS>(static_cast<const T*>(p.dy) + m * p.lddy, p.N, thread, dy);
        }
        if (p.dout) load_row<TR, C, ENDS>(static_cast<const T*>(p.dout) + m * p.lddout, p.N, thread, dout);
    };
    const auto load_h = [&](long long m) {
        if (m < p.M && p.h) load_row<TR, C, ENDS>(static_cast<const T*>(p.h) + m * p.ldh, p.N, thread, h);
    };
    if (AHEAD) {
        load_x(blockIdx.x);
        load_h(blockIdx.x);
    }
    for (long long m = blockIdx.x; m < p.M; m += gridDim.x) {
        if (!AHEAD) {
            x = h = dy = dout = Row<T, C>{};
            load_x(m);
            load_h(m);
        }
        load_row_or<TR, C, ENDS>(static_cast<const T*>(p.pre_weight), p.N, thread, 1.f, w);
        settle<TR, C, ENDS>(x, p.N, thread);
        settle<TR, C, ENDS>(dy, p.N, thread);
        settle<TR, C, ENDS>(h, p.N, thread);
        settle<TR, C, ENDS>(w, p.N, thread);
        settle<TR, C, ENDS>(dout, p.N, thread);
        RowSums s{0.f, 1.f, 0.f, 0.f, 0.f, 1.f, 0.f, 0.f};
        if (p.pre == IOLB_NORM_LAYER || p.post == IOLB_NORM_LAYER) {
            float v[2] = {0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    v[0] += (float)x.of[c][i];
                    v[1] += (float)h.of[c][i];
                }
            sum(v);
            if (p.pre == IOLB_NORM_LAYER) s.mean_x = v[0] * per;
            if (p.post == IOLB_NORM_LAYER) s.mean_h = v[1] * per;
        }
        hold(x);
        hold(h);
        hold(dy);
        hold(w);
        float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool live = 8 * (c * TR + thread) + i < p.N;
                const float vx = live ? (float)x.of[c][i] - s.mean_x : 0.f, vh = live ? (float)h.of[c][i] - s.mean_h : 0.f;
                const float t = (float)dy.of[c][i] * (float)w.of[c][i];
                v[0] = __builtin_fmaf(vx, vx, v[0]);
                v[1] = __builtin_fmaf(t, vx, v[1]);
                v[2] += t;
                v[3] = __builtin_fmaf(vh, vh, v[3]);
            }
        sum(v);
        if (p.dy) {
            s.r_x = 1.f / sqrtf(v[0] * per + p.eps);
            s.along_x = v[1] * s.r_x * per;
            if (p.pre == IOLB_NORM_LAYER) s.mean_d = v[2] * per;
        }
        if (p.post != IOLB_NORM_NONE) s.r_h = 1.f / sqrtf(v[3] * per + p.eps);
        hold(x);
        hold(h);
        hold(dy);
        hold(w);
        hold(dout);
        float d[C][8];
#pragma unroll
        for (int c = 0; c < C; ++c)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool live = 8 * (c * TR + thread) + i < p.N;
                const float along = ((float)x.of[c][i] - s.mean_x) * s.r_x * s.along_x;
                d[c][i] = (float)dout.of[c][i];
                if (p.dy) d[c][i] += s.r_x * ((float)dy.of[c][i] * (float)w.of[c][i] - along - s.mean_d);
                if (!live) d[c][i] = 0.f;
            }
        if (AHEAD) load_x(m + gridDim.x);
        if (p.dx) {
#pragma unroll
            for (int c = 0; c < C; ++c) {
                const int at = 8 * (c * TR + thread);
                Eight<T> to;
#pragma unroll
                for (int i = 0; i < 8; ++i) to[i] = (T)(p.scale * d[c][i]);
                store_eight_of(static_cast<T*>(p.dx) + m * p.N + at, p.N - at, to);
            }
        }
        if (p.h && (p.dh || p.rows)) {
            load_row_or<TR, C, ENDS>(static_cast<const T*>(p.post_weight), p.N, thread, 1.f, w);
            load_row_or<TR, C, ENDS>(p.gate ? static_cast<const T*>(p.gate) + m / p.rows_per_group * p.N : nullptr, p.N, thread, 1.f, g);
            settle<TR, C, ENDS>(w, p.N, thread);
            settle<TR, C, ENDS>(g, p.N, thread);
            float u[2] = {0.f, 0.f};
#pragma unroll
            for (int c = 0; c < C; ++c)
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    d[c][i] *= (float)g.of[c][i] * (float)w.of[c][i];
                    u[0] = __builtin_fmaf(d[c][i], ((float)h.of[c][i] - s.mean_h) * s.r_h, u[0]);
                    u[1] += d[c][i];
                }
            if (p.post != IOLB_NORM_NONE) {
                sum(u);
                s.along_h = u[0] * per;
                if (p.post == IOLB_NORM_LAYER) s.mean_p = u[1] * per;
            }
            hold(h);
            if (p.dh) {
#pragma unroll
                for (int c = 0; c < C; ++c) {
                    const int at = 8 * (c * TR + thread);
                    Eight<T> to;
#pragma unroll
                    for (int i = 0; i < 8; ++i) to[i] = (T)(s.r_h * (d[c][i] - ((float)h.of[c][i] - s.mean_h) * s.r_h * s.along_h - s.mean_p));
                    store_eight_of(static_cast<T*>(p.dh) + m * p.N + at, p.N - at, to);
                }
            }
        }
        if (AHEAD) load_h(m + gridDim.x);
        if (p.rows && threadIdx.x == 0) reinterpret_cast<RowSums*>(p.rows)[m] = s;
    }
}

// What weights, biases and gate get.  First the pieces of a group (its rows of the gate are done then, and all of it where there is one group); then
// (`across`) the groups, whose sums lie in the place of their first piece.  A workgroup takes 16 columns, 64 threads to each.  BIASES: whether S0 and T0
// are there; of a pair one may have been left out, and what stands in its place is then read but goes nowhere.
template <int DT, bool BIASES>
__global__ void __launch_bounds__(1024)
norm_backward_weights_kernel(BlockNormBackward p, int in_group, bool across)
{
    typedef typename DenseType<DT>::type T;
    __shared__ float part[NORM_COLUMN_SUMS][64][16 + 1];
    const unsigned blocks = (unsigned)(p.N + 15) / 16;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, n = (int)(blockIdx.x % blocks * 16) + tx;
    const long long ld = (p.N + 7) / 8 * 8;
    const int group = (int)(blockIdx.x / blocks), count = across ? p.groups : in_group;
    const T* const gates = static_cast<const T*>(p.gate);
    float sums[NORM_COLUMN_SUMS] = {0.f, 0.f, 0.f, 0.f};
    float* const at = p.columns + (long long)group * in_group * NORM_COLUMN_SUMS * ld + n;
    if (n < p.N) {
#pragma unroll 4
        for (int i = ty; i < count; i += 64) {
            const float* const from = at + (long long)(across ? i * (long long)in_group : i) * NORM_COLUMN_SUMS * ld;
            const float g = across && gates ? (float)gates[(long long)i * p.N + n] : 1.f;
#pragma unroll
            for (int k = 0; k < NORM_COLUMN_SUMS; ++k)
                if (BIASES || k == S1 || k == T1) sums[k] += (k == S1 || k == S0 ? g : 1.f) * from[k * ld];
        }
    }
#pragma unroll
    for (int k = 0; k < NORM_COLUMN_SUMS; ++k) part[k][ty][tx] = sums[k];
    __syncthreads();
    // a wave adds one of the four, four threads to a column
    const int k = threadIdx.x >> 6;
    if (k < NORM_COLUMN_SUMS) {
        const int col = threadIdx.x & 15, row = threadIdx.x >> 4 & 3;
        float t = 0.f;
#pragma unroll
        for (int i = 0; i < 16; ++i) t += part[k][4 * i + row][col];
        t += __shfl_xor(t, 16);
        t += __shfl_xor(t, 32);
        __builtin_amdgcn_wave_barrier();
        if (row == 0) part[k][0][col] = t;
    }
    __syncthreads();
    if (ty != 0 || n >= p.N) return;
#pragma unroll
    for (int j = 0; j < NORM_COLUMN_SUMS; ++j) sums[j] = part[j][0][tx];
    const T *const wp = static_cast<const T*>(p.post_weight), *const bp = static_cast<const T*>(p.post_bias);
    if (!across && p.dgate)
        static_cast<T*>(p.dgate)[(long long)group * p.N + n] = (T)((wp ? (float)wp[n] : 1.f) * sums[S1] + (bp ? (float)bp[n] * sums[S0] : 0.f));
    if (!across && p.groups > 1) {
#pragma unroll
        for (int j = 0; j < NORM_COLUMN_SUMS; ++j) at[j * ld] = sums[j];
        return;
    }
    const float g = !across && gates ? (float)gates[n] : 1.f;
    if (p.dpost_weight) static_cast<T*>(p.dpost_weight)[n] = (T)(g * sums[S1]);
    if (p.dpost_bias) static_cast<T*>(p.dpost_bias)[n] = (T)(g * sums[S0]);
    if (p.dpre_weight) static_cast<T*>(p.dpre_weight)[n] = (T)sums[T1];
    if (p.dpre_bias) static_cast<T*>(p.dpre_bias)[n] = (T)sums[T0];
}

// The same in one launch for some groups: a wave takes a group after the other, four threads to a column, and what it has summed over them is joined.
template <int DT, bool BIASES>
__global__ void __launch_bounds__(1024)
norm_backward_groups_kernel(BlockNormBackward p, int in_group)
{
    typedef typename DenseType<DT>::type T;
    __shared__ float part[NORM_COLUMN_SUMS][16][16 + 1];
    const int tx = threadIdx.x & 15, row = threadIdx.x >> 4 & 3, wave = threadIdx.x >> 6, n = (int)(blockIdx.x * 16) + tx;
    const long long ld = (p.N + 7) / 8 * 8;
    const bool live = n < p.N;
    const T* const gates = static_cast<const T*>(p.gate);
    const float wp = p.post_weight && live ? (float)static_cast<const T*>(p.post_weight)[n] : 1.f;
    const float bp = p.post_bias && live ? (float)static_cast<const T*>(p.post_bias)[n] : 0.f;
    float all[NORM_COLUMN_SUMS] = {0.f, 0.f, 0.f, 0.f};
    for (int group = wave; group < p.groups; group += 16) {
        float sums[NORM_COLUMN_SUMS] = {0.f, 0.f, 0.f, 0.f};
        const float* from = p.columns + ((long long)group * in_group + row) * NORM_COLUMN_SUMS * ld + n;
        const float g = live && gates ? (float)gates[(long long)group * p.N + n] : 1.f;
        if (live) {
#pragma unroll 4
            for (int i = row; i < in_group; i += 4, from += 4 * NORM_COLUMN_SUMS * ld)
#pragma unroll
                for (int k = 0; k < NORM_COLUMN_SUMS; ++k)
                    if (BIASES || k == S1 || k == T1) sums[k] += from[k * ld];
        }
#pragma unroll
        for (int k = 0; k < NORM_COLUMN_SUMS; ++k) {
            sums[k] += __shfl_xor(sums[k], 16);
            sums[k] += __shfl_xor(sums[k], 32);
            all[k] += (k == S1 || k == S0 ? g : 1.f) * sums[k];
        }
        if (p.dgate && live && row == 0) static_cast<T*>(p.dgate)[(long long)group * p.N + n] = (T)(wp * sums[S1] + (p.post_bias ? bp * sums[S0] : 0.f));
    }
    if (row == 0) {
#pragma unroll
        for (int k = 0; k < NORM_COLUMN_SUMS; ++k) part[k][wave][tx] = all[k];
    }
    __syncthreads();
    if (threadIdx.x >= 16 || !live) return;
#pragma unroll
    for (int k = 0; k < NORM_COLUMN_SUMS; ++k) {
        all[k] = 0.f;
        for (int i = 0; i < 16; ++i) all[k] += part[k][i][tx];
    }
    if (p.dpost_weight) static_cast<T*>(p.dpost_weight)[n] = (T)all[S1];
    if (p.dpost_bias) static_cast<T*>(p.dpost_bias)[n] = (T)all[S0];
    if (p.dpre_weight) static_cast<T*>(p.dpre_weight)[n] = (T)all[T1];
    if (p.dpre_bias) static_cast<T*>(p.dpre_bias)[n] = (T)all[T0];
}

// f called with the type as an integral constant.
template <class F>
void by_type(int dtype, F f)
{
    if (dtype == IOLB_F32) f(std::integral_constant<int, IOLB_F32>{});
    else if (dtype == IOLB_F16) f(std::integral_constant<int, IOLB_F16>{});
    else f(std::integral_constant<int, IOLB_BF16>{});
}

// Which of the column sums are wanted.
unsigned column_sums(const BlockNormBackward& p)
{
    return (p.dgate || p.dpost_weight ? 1u << S1 : 0u) | (p.dpost_bias || (p.dgate && p.post_bias) ? 1u << S0 : 0u) | (p.dpre_weight ? 1u << T1 : 0u) |
           (p.dpre_bias ? 1u << T0 : 0u);
}

constexpr int MOST_IN_REGISTERS = 512 * 8 * 4;          // values of a row, forward
constexpr int MOST_BACKWARD = 512 * 8 * 2;              // backward, with the columns' sums

// f called with the threads that take a row, and how many times eight values each; 0 where the row is not held in registers.
// Sixteen lanes take up to 256 columns: 100000 x 256 bf16 39 us, gradients 78, by a wave 70 / 150.  Of more columns a wave is faster (30000 x 512 bf16 28 / 57,
// sixteen lanes with four pieces each 35 / 73), and of more than 1024 four waves (10000 x 2048 32 / 77, a wave 34 / 89).
template <class F>
void by_row(int N, F f)
{
    const auto call = [&](auto tr, auto c) { f(tr, c); };
#define IOLB_ROW(TR, C) if (N <= 8 * TR * C) return call(std::integral_constant<int, TR>{}, std::integral_constant<int, C>{})
    IOLB_ROW(16, 1);
    IOLB_ROW(16, 2);
    IOLB_ROW(64, 1);
    IOLB_ROW(64, 2);
    IOLB_ROW(256, 1);
    IOLB_ROW(256, 2);
    IOLB_ROW(512, 2);
    if (N <= MOST_IN_REGISTERS) return call(std::integral_constant<int, 512>{}, std::integral_constant<int, 4>{});
#undef IOLB_ROW
    call(std::integral_constant<int, 256>{}, std::integral_constant<int, 0>{});
}

// f called with how the rows end, of a kernel that takes up to PIECES times eight values.
template <int PIECES, class F>
void by_end(int N, F f)
{
    if (N % 8 == 0) return f(std::integral_constant<int, WHOLE>{});
    if constexpr (PIECES == 16) {
        if (N < 8) return f(std::integral_constant<int, SHORT>{});
    }
    f(std::integral_constant<int, CUT>{});
}

// The call as a launch sees it that starts with this group.
template <int DT>
BlockNormBackward from_group(BlockNormBackward p, const NormPieces& pieces, long long group)
{
    typedef typename DenseType<DT>::type T;
    const long long row = group * p.rows_per_group;
    const auto move = [](const void*& t, long long by) { if (t) t = static_cast<const T*>(t) + by; };
    move(p.dy, row * p.lddy);
    move(p.dout, row * p.lddout);
    move(p.x, row * p.ldx);
    move(p.h, row * p.ldh);
    move(p.gate, group * p.N);
    if (p.dgate) p.dgate = static_cast<T*>(p.dgate) + group * p.N;
    if (p.rows) p.rows += row * NORM_ROW_SUMS;
    p.columns += group * pieces.in_group * NORM_COLUMN_SUMS * ((p.N + 7) / 8 * 8);
    return p;
}

// launch(call, workgroups) for all groups, `each` workgroups to a group, about a million at a time: a launch counts its threads in 32 bits, and one of a
// million workgroups takes so long that another one behind it does not show.
template <int DT, class F>
void in_turns(const BlockNormBackward& p, const NormPieces& pieces, long long each, F launch)
{
    const long long most = each < 1 << 20 ? (1 << 20) / each : 1;
    for (long long group = 0; group < p.groups; group += most)
        launch(from_group<DT>(p, pieces, group), (unsigned)(each * (p.groups - group < most ? p.groups - group : most)));
}

unsigned row_groups(int M) { return (unsigned)(M < 65536 ? M : 65536); }

}  // namespace

// Outputs past the caches: 16384 x 1024 bf16 28.2 us, so 23.1; 8192 x 4096 52.3 / 50.8, gradients 107 / 103; 4096 x 8192 101 / 97.
static bool past_caches(long long M, long long N, int dtype, int tensors) { return past_caches((double)M * N * (dtype == IOLB_F32 ? 4 : 2) * tensors); }

hipError_t launch_block_norm(const BlockNorm& p, int dtype, hipStream_t st)
{
    const bool past = past_caches(p.M, p.N, dtype, (p.h ? 3 : 1) + (p.y ? 1 : 0));
    by_type(dtype, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        by_row(p.N, [&](auto tr, auto c) {
            constexpr int TR = decltype(tr)::value, C = decltype(c)::value;
            if constexpr (C == 0) {
                block_norm_long_kernel<DT><<<row_groups(p.M), 256, 0, st>>>(p);
            } else {
                constexpr int ROWS = TR > 256 ? 1 : 256 / TR;
                by_end<TR * C>(p.N, [&](auto end) {
                    constexpr int ENDS = decltype(end)::value;
                    const auto kernel = past ? block_norm_rows_kernel<DT, TR, C, ENDS, true> : block_norm_rows_kernel<DT, TR, C, ENDS, false>;
                    kernel<<<row_groups((int)((p.M + (ROWS - 1LL)) / ROWS)), TR > 256 ? TR : 256, 0, st>>>(p);
                });
            }
        });
    });
    return hipGetLastError();
}

NormBackwardPlan block_norm_backward_plan(const BlockNormBackward& p, int)
{
    NormBackwardPlan plan{};
    const bool in_registers = p.N <= MOST_BACKWARD;
    const long long across = in_registers ? 1 : (p.N + 63) / 64;
    const int R = p.rows_per_group;
    // Rows in registers: two workgroups of 256 threads to a compute unit, or one of 512, and no more: each writes a row of sums.  8192 x 4096 bf16: 768
    // pieces 126 us, 512 111; 16384 x 1024 66 / 57; 4096 x 8192: 512 115, 256 106.  fp32 takes the same numbers, unmeasured against others: of 2049 to 4096
    // values a workgroup's registers fill a unit, so that two follow one another.
    const int at_once = !in_registers ? 32 : p.N <= 256 ? 16 : p.N <= 1024 ? 4 : 1, all = !in_registers ? 2048 : p.N <= 4096 ? 512 : 256;
    long long wanted = all / across / p.groups;
    if (wanted > (R + at_once - 1) / at_once) wanted = (R + at_once - 1) / at_once;
    if (wanted < 1) wanted = 1;
    plan.pieces = {1, 1};                           // (no rows: sums of nothing)
    if (R > 0) {
        plan.pieces.per = (int)((R + wanted - 1) / wanted);
        plan.pieces.in_group = (R + plan.pieces.per - 1) / plan.pieces.per;
    }
    if (!column_sums(p)) return plan;
    // (blocks of 16 columns and a group: more of them than 2^32 have sums of 2^40 bytes and more)
    const long long pieces = (long long)plan.pieces.in_group * p.groups;
    plan.launchable = (p.N + 15LL) / 16 * p.groups <= 0xffffffffLL;
    plan.row_bytes = in_registers ? 0 : (size_t)p.M * NORM_ROW_SUMS * 4;
    plan.column_bytes = (size_t)pieces * NORM_COLUMN_SUMS * ((p.N + 7) / 8 * 8) * 4;
    return plan;
}

hipError_t launch_block_norm_backward(const BlockNormBackward& p, const NormBackwardPlan& plan, int dtype, hipStream_t st)
{
    const bool past = past_caches(p.M, p.N, dtype, (p.dy ? 2 : 0) + (p.dout ? 1 : 0) + (p.h ? 1 : 0) + (p.dx ? 1 : 0) + (p.dh ? 1 : 0));
    const unsigned wanted = column_sums(p), pieces = (unsigned)(plan.pieces.in_group * p.groups);
    by_type(dtype, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        by_row(p.N, [&](auto tr, auto c) {
            constexpr int TR = decltype(tr)::value, C = decltype(c)::value;
            if constexpr (C == 0 || 8 * TR * C > MOST_BACKWARD) {
                if constexpr (C == 0) {
                    if (p.M) norm_backward_long_kernel<DT><<<row_groups(p.M), 256, 0, st>>>(p);
                } else if (p.M) {
                    by_end<TR * C>(p.N, [&](auto end) { norm_backward_wide_kernel<DT, TR * C / 1024, decltype(end)::value><<<(unsigned)(p.M < 256 ? p.M : 256), 1024, 0, st>>>(p); });
                }
                if (wanted)
                    in_turns<DT>(p, plan.pieces, (p.N + 63LL) / 64 * plan.pieces.in_group, [&](const BlockNormBackward& turn, unsigned n) {
                        norm_backward_columns_kernel<DT><<<n, 256, 0, st>>>(turn, plan.pieces);
                    });
            } else {
                const bool biases = wanted >> S0 & 1 || wanted >> T0 & 1;
                by_end<TR * C>(p.N, [&](auto end) {
                    constexpr int ENDS = decltype(end)::value;
                    const auto kernel = biases ? (past ? norm_backward_rows_kernel<DT, TR, C, true, ENDS, true> : norm_backward_rows_kernel<DT, TR, C, true, ENDS, false>)
                                               : (past ? norm_backward_rows_kernel<DT, TR, C, false, ENDS, true> : norm_backward_rows_kernel<DT, TR, C, false, ENDS, false>);
                    kernel<<<pieces, TR > 256 ? TR : 256, 0, st>>>(p, plan.pieces, wanted);
                });
            }
        });
        if (!wanted) return;
        const auto weights = [&](auto biases) {
            constexpr bool BIASES = decltype(biases)::value;
            const unsigned across = (unsigned)((p.N + 15) / 16);
            if (p.groups >= 4 && p.groups <= 64) {
                norm_backward_groups_kernel<DT, BIASES><<<across, 1024, 0, st>>>(p, plan.pieces.in_group);
                return;
            }
            in_turns<DT>(p, plan.pieces, across, [&](const BlockNormBackward& turn, unsigned n) {
                norm_backward_weights_kernel<DT, BIASES><<<n, 1024, 0, st>>>(turn, plan.pieces.in_group, false);
            });
            if (p.groups > 1 && (p.dpost_weight || p.dpost_bias || p.dpre_weight || p.dpre_bias))
                norm_backward_weights_kernel<DT, BIASES><<<across, 1024, 0, st>>>(p, plan.pieces.in_group, true);
        };
        if (wanted >> S0 & 1 || wanted >> T0 & 1) weights(std::true_type{});
        else weights(std::false_type{});
    });
    return hipGetLastError();
}

}  // namespace iolb
