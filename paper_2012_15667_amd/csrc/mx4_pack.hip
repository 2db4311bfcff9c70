// Tensors into microscaled 4-bit floating point and back.  Streaming kernels: bound by memory.
#include "mx4_math.h"

namespace iolb {

namespace {

// Four lanes share a block of 32, eight values each.  A workgroup covers `wide` threads of a row, up to its padded end, and 256 / wide rows, one after the
// other, the next one on its way meanwhile.  PAST: values past the caches.
template <int DT, bool PAST>
__global__ void __launch_bounds__(256)
mx4_pack_kernel(const void* x, long long ldx, int rows, int cols, uint8_t* codes, uint8_t* scales, int wide_log)
{
    typedef typename DenseType<DT>::type T;
    typedef typename Piece<T, 8>::type Eight;
    const int wide = 1 << wide_log, tx = threadIdx.x & (wide - 1), ty = threadIdx.x >> wide_log;
    const long long pitch = (cols + MX4_WIDE - 1LL) / MX4_WIDE * (MX4_WIDE / 2), step = (long long)gridDim.y * (256 >> wide_log);
    const int c = (int)((blockIdx.x * (unsigned)wide + tx) * 8), have = cols - c;
    const T* const xs = static_cast<const T*>(x) + c;
    Eight next{};
    const auto load = [&](long long r) {
        if (r >= rows || have <= 0) return;
        const T* const from = xs + r * ldx;
        if (have >= 8) {
            if constexpr (PAST) next = __builtin_nontemporal_load(reinterpret_cast<const Eight*>(from));
            else next = *reinterpret_cast<const Eight*>(from);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) next[i] = from[i];
        }
    };
    long long r = (long long)blockIdx.y * (256 >> wide_log) + ty;
    load(r);
    for (; r - ty < rows; r += step) {
        const Eight now = next;
        load(r + step);
        float v[8];
        unsigned most = 0;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            v[i] = (float)now[i];
            const unsigned b = magnitude_bits(v[i]);
            most = b > most ? b : most;
        }
        most = most_of_four(most);
        const int s = mx4_scale(most);
        if (r >= rows || c / 2 >= pitch) continue;
        *reinterpret_cast<unsigned*>(codes + r * pitch + c / 2) = s == MX4_NAN ? 0u : mx4_codes(v, mx4_unit(s));
        if ((tx & 3) == 0) scales[r * (pitch / 16) + c / MX4_BLOCK] = (uint8_t)s;
    }
}

template <int DT> __device__ __forceinline__ float largest()
{
    return DT == IOLB_F16 ? 65504.f : DT == IOLB_BF16 ? 0x1.fep127f : 0x1.fffffep127f;
}

template <int DT, bool PAST>
__global__ void __launch_bounds__(256)
mx4_unpack_kernel(const uint8_t* codes, const uint8_t* scales, int rows, int cols, void* y, long long ldy, int wide_log)
{
    typedef typename DenseType<DT>::type T;
    const int wide = 1 << wide_log, tx = threadIdx.x & (wide - 1), ty = threadIdx.x >> wide_log;
    const long long pitch = (cols + MX4_WIDE - 1LL) / MX4_WIDE * (MX4_WIDE / 2);
    const int c = (int)((blockIdx.x * (unsigned)wide + tx) * 8), have = cols - c;
    if (have <= 0) return;
    const long long step = (long long)gridDim.y * (256 >> wide_log);
    int next_s = 0;
    unsigned next_w = 0;
    const auto load = [&](long long r) {
        if (r >= rows) return;
        next_s = scales[r * (pitch / 16) + c / MX4_BLOCK];
        next_w = *reinterpret_cast<const unsigned*>(codes + r * pitch + c / 2);
    };
    long long r = (long long)blockIdx.y * (256 >> wide_log) + ty;
    load(r);
    for (; r < rows; r += step) {
        const int s = next_s;
        const unsigned w = next_w;
        load(r + step);
        const float unit = mx4_unit(s);
        const f32x2 pair[4] = {__builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 0), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 1),
                               __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 2), __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(w, unit, 3)};
        typename Piece<T, 8>::type t;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float v = fminf(fmaxf(pair[i / 2][i % 2], -largest<DT>()), largest<DT>());
            t[i] = s == MX4_NAN ? (T)__builtin_nanf("") : (T)v;
        }
        T* const to = static_cast<T*>(y) + r * ldy + c;
        if (have >= 8) {
            if constexpr (PAST) __builtin_nontemporal_store(t, reinterpret_cast<typename Piece<T, 8>::type*>(to));
            else *reinterpret_cast<typename Piece<T, 8>::type*>(to) = t;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) to[i] = t[i];
        }
    }
}

// Workgroups, more than fill the chip at once.
constexpr int GROUPS = 16384;

struct RowGrid { dim3 grid; int wide_log; };
RowGrid row_grid(int rows, long long cols, long long each)
{
    int wide_log = 2;                               // whole blocks of 32
    while (wide_log < 8 && (each << wide_log) < cols) ++wide_log;
    const long long gx = (cols + (each << wide_log) - 1) / (each << wide_log), per = 256 >> wide_log;
    const long long gy = (rows + per - 1) / per, most = (GROUPS + gx - 1) / gx;
    return {dim3((unsigned)gx, (unsigned)(gy < most ? gy : most)), wide_log};
}

}  // namespace

// f called with the type and with whether the values go past the caches, as integral constants.  Measured, 16384 x 8192 bf16: packed 61 us, past the
// caches 58; unpacked 69 / 49, both in turn 143 / 109.  4096 x 4096 fp32 is faster through them: packed 12.3 / 14.4, unpacked 15.4 / 23.3.
template <class F>
static hipError_t by_type(int dtype, int rows, int cols, F f)
{
    const auto call = [&](auto type) {
        if (past_caches((double)rows * cols * (sizeof(typename DenseType<decltype(type)::value>::type) + 0.53))) f(type, std::true_type{});
        else f(type, std::false_type{});
    };
    if (dtype == IOLB_F32) call(std::integral_constant<int, IOLB_F32>{});
    else if (dtype == IOLB_F16) call(std::integral_constant<int, IOLB_F16>{});
    else call(std::integral_constant<int, IOLB_BF16>{});
    return hipGetLastError();
}

hipError_t launch_mx4_pack(const void* x, long long ldx, int rows, int cols, int dtype, uint8_t* codes, uint8_t* scales, hipStream_t st)
{
    const RowGrid g = row_grid(rows, 2 * mx4_pitch(cols), 8);
    return by_type(dtype, rows, cols, [&](auto type, auto past) {
        mx4_pack_kernel<decltype(type)::value, decltype(past)::value><<<g.grid, 256, 0, st>>>(x, ldx, rows, cols, codes, scales, g.wide_log);
    });
}

hipError_t launch_mx4_unpack(const uint8_t* codes, const uint8_t* scales, int rows, int cols, int dtype, void* y, long long ldy, hipStream_t st)
{
    const RowGrid g = row_grid(rows, cols, 8);
    return by_type(dtype, rows, cols, [&](auto type, auto past) {
        mx4_unpack_kernel<decltype(type)::value, decltype(past)::value><<<g.grid, 256, 0, st>>>(codes, scales, rows, cols, y, ldy, g.wide_log);
    });
}

}  // namespace iolb
