// Norms before and after a block with its gate and residual scale, and their gradients.  Streaming kernels: bound by memory.
#include "block.h"
#include "dense_math.h"

namespace iolb {

namespace {

template <int WAVES>
__device__ __forceinline__ float group_sum(float v, float (&part)[2][WAVES], int& turn)
{
#pragma unroll
    for (int d = 1; d < 64; d *= 2) v += __shfl_xor(v, d);
    if constexpr (WAVES > 1) {
        // (two buffers in turn: who writes one again has passed the barrier behind all reads of it)
        float* const at = part[turn];
        turn ^= 1;
        if ((threadIdx.x & 63) == 0) at[threadIdx.x >> 6] = v;
        __syncthreads();
        v = 0.f;
#pragma unroll
        for (int i = 0; i < WAVES; ++i) v += at[i];
    }
    return v;
}

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

template <class T>
__device__ __forceinline__ void store_columns_of(T* p, int have, const float (&v)[8])
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

// A workgroup to a row, which it reads again from the caches for each step.
template <int DT>
__global__ void __launch_bounds__(256)
block_norm_kernel(BlockNorm p)
{
    typedef typename DenseType<DT>::type T;
    __shared__ float part[2][4];
    int turn = 0;
    const auto sum = [&](float v) { return group_sum<4>(v, part, turn); };
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
norm_backward_rows_kernel(BlockNormBackward p)
{
    typedef typename DenseType<DT>::type T;
    __shared__ float part[2][4];
    int turn = 0;
    const auto sum = [&](float v) { return group_sum<4>(v, part, turn); };
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

// What weights, biases and gate get.  First the pieces of a group (its rows of the gate are done then, and all of it where there is one group); then
// (`across`) the groups, whose sums lie in the place of their first piece.  A workgroup takes 16 columns, 16 threads to each.
template <int DT>
__global__ void __launch_bounds__(256)
norm_backward_weights_kernel(BlockNormBackward p, int in_group, bool across)
{
    typedef typename DenseType<DT>::type T;
    __shared__ float part[NORM_COLUMN_SUMS][16][16 + 1];
    const unsigned blocks = (unsigned)(p.N + 15) / 16;
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4, n = (int)(blockIdx.x % blocks * 16) + tx;
    const long long ld = (p.N + 7) / 8 * 8;
    const int group = (int)(blockIdx.x / blocks), count = across ? p.groups : in_group;
    const T* const gates = static_cast<const T*>(p.gate);
    float sums[NORM_COLUMN_SUMS] = {0.f, 0.f, 0.f, 0.f};
    float* const at = p.columns + (long long)group * in_group * NORM_COLUMN_SUMS * ld + n;
    if (n < p.N)
        for (int i = ty; i < count; i += 16) {
            const float* const from = at + (long long)(across ? i * (long long)in_group : i) * NORM_COLUMN_SUMS * ld;
            const float g = across && gates ? (float)gates[(long long)i * p.N + n] : 1.f;
            sums[S1] += g * from[S1 * ld];
            sums[S0] += g * from[S0 * ld];
            sums[T1] += from[T1 * ld];
            sums[T0] += from[T0 * ld];
        }
#pragma unroll
    for (int k = 0; k < NORM_COLUMN_SUMS; ++k) part[k][ty][tx] = sums[k];
    __syncthreads();
    if (ty != 0 || n >= p.N) return;
#pragma unroll
    for (int k = 0; k < NORM_COLUMN_SUMS; ++k) {
        sums[k] = 0.f;
        for (int i = 0; i < 16; ++i) sums[k] += part[k][i][tx];
    }
    const T *const wp = static_cast<const T*>(p.post_weight), *const bp = static_cast<const T*>(p.post_bias);
    if (!across && p.dgate)
        static_cast<T*>(p.dgate)[(long long)group * p.N + n] = (T)((wp ? (float)wp[n] : 1.f) * sums[S1] + (bp ? (float)bp[n] * sums[S0] : 0.f));
    if (!across && p.groups > 1) {
#pragma unroll
        for (int k = 0; k < NORM_COLUMN_SUMS; ++k) at[k * ld] = sums[k];
        return;
    }
    const float g = !across && gates ? (float)gates[n] : 1.f;
    if (p.dpost_weight) static_cast<T*>(p.dpost_weight)[n] = (T)(g * sums[S1]);
    if (p.dpost_bias) static_cast<T*>(p.dpost_bias)[n] = (T)(g * sums[S0]);
    if (p.dpre_weight) static_cast<T*>(p.dpre_weight)[n] = (T)sums[T1];
    if (p.dpre_bias) static_cast<T*>(p.dpre_bias)[n] = (T)sums[T0];
}

// f called with the type as an integral constant.
template <class F>
void by_type(int dtype, F f)
{
    if (dtype == IOLB_F32) f(std::integral_constant<int, IOLB_F32>{});
    else if (dtype == IOLB_F16) f(std::integral_constant<int, IOLB_F16>{});
    else f(std::integral_constant<int, IOLB_BF16>{});
}

bool column_sums(const BlockNormBackward& p) { return p.dgate || p.dpost_weight || p.dpost_bias || p.dpre_weight || p.dpre_bias; }

unsigned row_groups(int M) { return (unsigned)(M < 65536 ? M : 65536); }

}  // namespace

hipError_t launch_block_norm(const BlockNorm& p, int dtype, hipStream_t st)
{
    by_type(dtype, [&](auto t) { block_norm_kernel<decltype(t)::value><<<row_groups(p.M), 256, 0, st>>>(p); });
    return hipGetLastError();
}

NormBackwardPlan block_norm_backward_plan(const BlockNormBackward& p, int)
{
    NormBackwardPlan plan{};
    if (!column_sums(p)) return plan;
    const int across = (p.N + 63) / 64, R = p.rows_per_group;
    int wanted = 2048 / across / p.groups;
    if (wanted > (R + 31) / 32) wanted = (R + 31) / 32;
    if (wanted < 1) wanted = 1;
    plan.pieces = {1, 1};                           // (no rows: sums of nothing)
    if (R > 0) {
        plan.pieces.per = (R + wanted - 1) / wanted;
        plan.pieces.in_group = (R + plan.pieces.per - 1) / plan.pieces.per;
    }
    // (a launch counts its threads in 32 bits)
    plan.launchable = (long long)(p.N + 15) / 16 * p.groups * 256 <= 0xffffffffLL && (long long)across * plan.pieces.in_group * p.groups * 256 <= 0xffffffffLL;
    plan.row_bytes = (size_t)p.M * NORM_ROW_SUMS * 4;
    plan.column_bytes = (size_t)plan.pieces.in_group * p.groups * NORM_COLUMN_SUMS * ((p.N + 7) / 8 * 8) * 4;
    return plan;
}

hipError_t launch_block_norm_backward(const BlockNormBackward& p, const NormBackwardPlan& plan, int dtype, hipStream_t st)
{
    by_type(dtype, [&](auto t) {
        constexpr int DT = decltype(t)::value;
        if (p.M) norm_backward_rows_kernel<DT><<<row_groups(p.M), 256, 0, st>>>(p);
        if (!column_sums(p)) return;
        norm_backward_columns_kernel<DT><<<(unsigned)((p.N + 63) / 64) * (unsigned)(plan.pieces.in_group * p.groups), 256, 0, st>>>(p, plan.pieces);
        norm_backward_weights_kernel<DT><<<(unsigned)((p.N + 15) / 16) * (unsigned)p.groups, 256, 0, st>>>(p, plan.pieces.in_group, false);
        if (p.groups > 1 && (p.dpost_weight || p.dpost_bias || p.dpre_weight || p.dpre_bias))
            norm_backward_weights_kernel<DT><<<(unsigned)((p.N + 15) / 16), 256, 0, st>>>(p, plan.pieces.in_group, true);
    });
    return hipGetLastError();
}

}  // namespace iolb
