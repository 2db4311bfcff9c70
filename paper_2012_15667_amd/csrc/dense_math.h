// Device arithmetic of dense layers and checkpoints: types, activations and their slopes, the 8-bit code.
#ifndef IOLB_DENSE_MATH_H
#define IOLB_DENSE_MATH_H

#include "dense.h"
#include "split_mfma.h"

#include <type_traits>

namespace iolb {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

template <int DT> struct DenseType;
template <> struct DenseType<IOLB_F32> { typedef float type; };
template <> struct DenseType<IOLB_F16> { typedef _Float16 type; };
template <> struct DenseType<IOLB_BF16> { typedef __bf16 type; };

// ---- activations, in 32 bits ----------------------------------------------------------------------
// P(normal > |z|) by formula 7.1.26 of Abramowitz and Stegun (error of erf at most 1.5e-7): nothing cancels in the tail, where the formula itself is off by
// 5e-5 of the result at -3 and 5e-4 at -4 (1 + erf in 32 bits: 7e-6 at -3, more than this from -4.5 on).
__device__ __forceinline__ float normal_tail(float z, float gauss /* e^(-z^2 / 2) */)
{
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.3275911f * 0.70710678f, fabsf(z), 1.f));
    const float p = t * (0.127414796f + t * (-0.142248368f + t * (0.7107068705f + t * (-0.7265760135f + t * 0.5307027145f))));
    return p * gauss;
}

__device__ __forceinline__ float gauss_of(float z) { return __builtin_amdgcn_exp2f(z * z * -0.72134752f); }     // e^(-z^2 / 2)

__device__ __forceinline__ float sigmoid(float z) { return __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(z * -1.44269504f)); }

constexpr float GELU_TANH_K = 1.5957691216f;      // 2 sqrt(2 / pi): (1 + tanh u) / 2 is the sigmoid of 2 u

// Smooth activations tend to zero at -inf, where their formula is 0 x inf: the factor z is kept from going beyond -10^4 (which gives zero), while a
// NaN, which such a comparison drops, comes through the other factor.
template <int ACT>
__device__ __forceinline__ float activate(float z)
{
    if constexpr (ACT == IOLB_ACT_NONE) return z;
    if constexpr (ACT == IOLB_ACT_RELU) return z <= 0.f ? 0.f : z;
    if constexpr (ACT == IOLB_ACT_SILU) return fmaxf(z, -1e4f) * sigmoid(z);
    // z Phi(z) = max(z, 0) - |z| P(normal > |z|)
    if constexpr (ACT == IOLB_ACT_GELU) return __builtin_fmaf(-fminf(fabsf(z), 1e4f), normal_tail(z, gauss_of(z)), fmaxf(z, 0.f));
    if constexpr (ACT == IOLB_ACT_GELU_TANH) return fmaxf(z, -1e4f) * sigmoid(z * __builtin_fmaf(GELU_TANH_K * 0.044715f, z * z, GELU_TANH_K));
}

// dy act'(z).  Beyond |z| = 60 the slopes are 0 or 1 to every bit; cutting z there keeps its powers finite.
// (Comparisons, not fmin: a NaN stays one.)
template <int ACT>
__device__ __forceinline__ float through_activation(float dy, float z)
{
    if constexpr (ACT == IOLB_ACT_NONE) return dy;
    if constexpr (ACT == IOLB_ACT_RELU) return z <= 0.f ? 0.f : z > 0.f ? dy : z;
    z = z > 60.f ? 60.f : z < -60.f ? -60.f : z;
    float slope;
    if constexpr (ACT == IOLB_ACT_SILU) {
        const float s = sigmoid(z);
        slope = s * (1.f + z * (1.f - s));
    }
    if constexpr (ACT == IOLB_ACT_GELU) {
        const float g = gauss_of(z), tail = normal_tail(z, g);
        slope = __builtin_fmaf(z * g, 0.3989422804f, z > 0.f ? 1.f - tail : tail);
    }
    if constexpr (ACT == IOLB_ACT_GELU_TANH) {
        const float s = sigmoid(z * __builtin_fmaf(GELU_TANH_K * 0.044715f, z * z, GELU_TANH_K));
        slope = s + z * s * (1.f - s) * GELU_TANH_K * (1.f + 0.134145f * z * z);
    }
    return dy * slope;
}

// f called with the activation as an integral constant.
template <class F>
__device__ __forceinline__ void by_activation(int act, F f)
{
    switch (act) {
    case IOLB_ACT_RELU: f(std::integral_constant<int, IOLB_ACT_RELU>{}); break;
    case IOLB_ACT_SILU: f(std::integral_constant<int, IOLB_ACT_SILU>{}); break;
    case IOLB_ACT_GELU: f(std::integral_constant<int, IOLB_ACT_GELU>{}); break;
    case IOLB_ACT_GELU_TANH: f(std::integral_constant<int, IOLB_ACT_GELU_TANH>{}); break;
    default: f(std::integral_constant<int, IOLB_ACT_NONE>{}); break;
    }
}

// ---- the 8-bit code ---------------------------------------------------------------------------------
// A block's values are q 2^e, q from -127 to 127, e the least exponent with |x| <= 127 2^e for its finite values, kept so that
// every value is one of the tensor's type (fp16: multiples of 2^-24 up to 65504; else of 2^-126).  A power of two as the scale makes
// the values exact in bf16: the backward pass hands them to the matrix cores without a second rounding, and an fp32 layer's
// weight gradient needs three products of parts instead of six.  It costs up to one bit against a scale of max / 127.
// q = -128 is a value that is not finite; it reads back as NaN.
struct CkptRange { int lo, hi; };
template <int DT> __device__ __forceinline__ CkptRange ckpt_range() { return DT == IOLB_F16 ? CkptRange{-24, 10} : CkptRange{-126, 122}; }

__device__ __forceinline__ float finite_magnitude(float x)
{
    const float a = fabsf(x);
    return a < __builtin_inff() ? a : 0.f;              // (false for NaN too)
}

__device__ __forceinline__ float two_to(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }   // -126 <= e <= 127

template <int DT>
__device__ __forceinline__ int ckpt_exponent(float most)
{
    const unsigned u = __float_as_uint(most);
    const int e = (int)(u >> 23) - 127 - ((u & 0x7fffffu) <= 0x7e0000u ? 6 : 5);    // 127 = 1.984375 * 2^6
    const CkptRange r = ckpt_range<DT>();
    return e < r.lo ? r.lo : e > r.hi ? r.hi : e;
}

// W neighbouring values of a block, of which the lane's `have` exist; LANES lanes hold the block.  Returns their codes, four to a word, and
// the block's exponent.  Every lane of the wave calls.
//   A block of finite values below the largest exponent is the rule: its largest magnitude is the largest of the bits, and 1.5 2^23 added to
// x 2^-e (one rounding, to nearest even) leaves the code in the low byte.  Where a lane of the wave meets anything else, all take the other
// way: values that are not finite are left out of the largest and become -128, and at the largest exponent, where 64 2^e is beyond the type,
// codes end at 63.
template <int DT, int W, int LANES>
__device__ __forceinline__ void ckpt_codes(const float (&x)[W], int have, unsigned (&codes)[W / 4], int& exponent)
{
    unsigned bits = 0;
#pragma unroll
    for (int i = 0; i < W; ++i) {
        const unsigned b = __float_as_uint(x[i]) & 0x7fffffffu;
        bits = i < have && b > bits ? b : bits;
    }
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) {
        const unsigned b = (unsigned)__shfl_xor((int)bits, d);
        bits = b > bits ? b : bits;
    }
    int e = ckpt_exponent<DT>(__uint_as_float(bits));
    unsigned c[W];
    if (!__any(bits >= 0x7f800000u || e == ckpt_range<DT>().hi)) {
        const float unit = two_to(-e);
#pragma unroll
        for (int i = 0; i < W; ++i) c[i] = __float_as_uint(__builtin_fmaf(x[i], unit, 12582912.f));
    } else {
        float most = 0.f;
#pragma unroll
        for (int i = 0; i < W; ++i) most = i < have ? fmaxf(most, finite_magnitude(x[i])) : most;
#pragma unroll
        for (int d = 1; d < LANES; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
        e = ckpt_exponent<DT>(most);
        const float unit = two_to(-e), top = e == ckpt_range<DT>().hi ? 63.f : 127.f;
#pragma unroll
        for (int i = 0; i < W; ++i) {
            float q = __builtin_rintf(x[i] * unit);
            q = q > top ? top : q < -top ? -top : q;
            c[i] = fabsf(x[i]) < __builtin_inff() ? (unsigned)(int)q : 0x80u;
        }
    }
    exponent = e;
#pragma unroll
    for (int w = 0; w < W / 4; ++w) {
        const unsigned lo = __builtin_amdgcn_perm(c[4 * w + 1], c[4 * w], 0x0c0c0400u), hi = __builtin_amdgcn_perm(c[4 * w + 3], c[4 * w + 2], 0x04000c0cu);
        codes[w] = lo | hi;
    }
}

__device__ __forceinline__ float ckpt_value(int code, float unit) { return code == -128 ? __builtin_nanf("") : (float)code * unit; }

// ---- three bf16 parts of an fp32 value ----------------------------------------------------------------
__device__ __forceinline__ void dense_parts(float a, unsigned short& h, unsigned short& m, unsigned short& l)
{
    const unsigned u = __float_as_uint(a);
    unsigned short hh = __builtin_bit_cast(unsigned short, (__bf16)a);
    const bool finite = (u & 0x7f800000u) != 0x7f800000u;
    if (finite && (hh & 0x7f80u) == 0x7f80u) hh = (unsigned short)(u >> 16);
    const float r = finite ? a - __uint_as_float((unsigned)hh << 16) : 0.f;
    const unsigned short mm = __builtin_bit_cast(unsigned short, (__bf16)r);
    h = hh;
    m = mm;
    l = __builtin_bit_cast(unsigned short, (__bf16)(r - __uint_as_float((unsigned)mm << 16)));
}

// ---- products -----------------------------------------------------------------------------------------
template <bool F16>
__device__ __forceinline__ f32x4 multiply(const u32x4& a, const u32x4& b, const f32x4& c)
{
    if constexpr (F16)
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(f16x8, a), __builtin_bit_cast(f16x8, b), c, 0, 0, 0);
    else
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
}

// Where 16-byte piece c of a 128-byte row lies in LDS: sixteen rows' pieces of the same c fall on different banks.
__device__ __forceinline__ int place(int row, int piece) { return piece ^ (row & 7); }

// N 32-bit words from any address that is one for a T.
template <int N, class T>
__device__ __forceinline__ auto words_at(const T* p)
{
    typedef unsigned Words __attribute__((ext_vector_type(N)));
    typedef unsigned Anywhere __attribute__((ext_vector_type(N), aligned(sizeof(T))));
    return (Words)*reinterpret_cast<const Anywhere*>(p);
}

// The same four words of 16-bit values at odd addresses, by aligned accesses: memory takes the others at a third of the rate (4 x 14464 x 1152 fp16
// with rows 1153 apart 33 us, with this 20; 1154 apart 14).  The fifth word is read only where a value of the four lies in it.
template <class T>
__device__ __forceinline__ u32x4 words_at_odd(const T* p)
{
    const size_t at = reinterpret_cast<size_t>(p);
    const unsigned off = (unsigned)at & 2;
    const unsigned* const q = reinterpret_cast<const unsigned*>(at - off);
    const u32x4 d = words_at<4>(q);
    const unsigned last = q[off ? 4 : 3];
    return u32x4{__builtin_amdgcn_alignbyte(d[1], d[0], off), __builtin_amdgcn_alignbyte(d[2], d[1], off), __builtin_amdgcn_alignbyte(d[3], d[2], off),
                 __builtin_amdgcn_alignbyte(last, d[3], off)};
}

// ---- the end of a product: W (4 or 8) neighbouring columns n ... of row m --------------------------------
// W values of T in one piece, at any address that is one for a T: rows start where their length and the caller's strides put them, and global
// memory takes such accesses (a row of 1151 fp16 weights read value by value on 4 rows for 14464 outputs cost 68 us, in pieces 22).
template <class T, int W> struct Piece { typedef T type __attribute__((ext_vector_type(W), aligned(sizeof(T)))); };

template <int W, class T>
__device__ __forceinline__ void load_columns(const T* p, int have, float (&v)[W])
{
    if (have >= W) {
        const auto t = *reinterpret_cast<const typename Piece<T, W>::type*>(p);
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = (float)t[i];
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) v[i] = i < have ? (float)p[i] : 0.f;
    }
}

template <int DT, int W>
__device__ __forceinline__ void load_bias(const DenseFinish& f, int n, float (&b)[W])
{
    typedef typename DenseType<DT>::type T;
    if (f.bias) {
        load_columns(static_cast<const T*>(f.bias) + n, f.N - n, b);
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i) b[i] = 0.f;
    }
}

template <int DT, int W>
__device__ __forceinline__ void add_residual(const DenseFinish& f, int m, int n, float (&z)[W])
{
    typedef typename DenseType<DT>::type T;
    float v[W];
    load_columns(static_cast<const T*>(f.residual) + m * f.ldr + n, f.N - n, v);
#pragma unroll
    for (int i = 0; i < W; ++i) z[i] += v[i];
}

// W columns' codes, and from the block's first lane its exponent.
template <int W>
__device__ __forceinline__ void store_codes(const DenseFinish& f, int m, int n, const unsigned (&codes)[W / 4], int e)
{
    typedef unsigned Words __attribute__((ext_vector_type(W / 4), aligned(1)));
    const int have = f.N - n;
    int8_t* const to = f.zq + (long long)m * f.N + n;
    if (have >= W) {
        Words t;
#pragma unroll
        for (int w = 0; w < W / 4; ++w) t[w] = codes[w];
        *reinterpret_cast<Words*>(to) = t;
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < have) to[i] = (int8_t)(codes[i / 4] >> 8 * (i % 4));
    }
    if (n % CKPT_BLOCK == 0) f.ze[(long long)m * ((f.N + CKPT_BLOCK - 1) / CKPT_BLOCK) + n / CKPT_BLOCK] = (uint8_t)(e + 127);
}

// y = act(z) (+ residual, if it comes after); the one rounding to y's type
template <int DT, int ACT, int W>
__device__ __forceinline__ void store_columns(const DenseFinish& f, int m, int n, float (&z)[W])
{
    typedef typename DenseType<DT>::type T;
    typedef typename Piece<T, W>::type TW;
    const int have = f.N - n;
#pragma unroll
    for (int i = 0; i < W; ++i) z[i] = activate<ACT>(z[i]);
    if (f.residual && !f.first) add_residual<DT>(f, m, n, z);
    T* y = static_cast<T*>(f.y) + m * f.ldy + n;
    if (have >= W) {
        TW t;
#pragma unroll
        for (int i = 0; i < W; ++i) t[i] = (T)z[i];
        *reinterpret_cast<TW*>(y) = t;
    } else {
#pragma unroll
        for (int i = 0; i < W; ++i)
            if (i < have) y[i] = (T)z[i];
    }
}

// Four columns without a checkpoint, for a wave that holds them in one lane.
template <int DT>
__device__ __forceinline__ void finish_four(const DenseFinish& f, int m, int n, const float (&bias)[4], const f32x4& sum)
{
    if (m >= f.M || n >= f.N) return;
    float z[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) z[i] = sum[i] + bias[i];
    if (f.residual && f.first) add_residual<DT>(f, m, n, z);
    by_activation(f.act, [&](auto act) __attribute__((always_inline)) { store_columns<DT, decltype(act)::value>(f, m, n, z); });
}

// ---- sums of operands in two fp16 parts ----------------------------------------------------------------
__device__ __forceinline__ bool not_wanted(const DenseProduct& p)
{
    return p.uneven && ((p.uneven[0] | (p.when ? p.uneven[1] : 0)) != 0) != (p.when != 0);
}

// A scaled sum below this may owe more than 2^-20 of itself to what the parts left out: a row's loss times the other row's largest value, which is
// below 2^15.  (A row of zeros: nothing is lost.)
__device__ __forceinline__ float least_sum(float lost_a, float lost_b)
{
    return lost_a < 0.f || lost_b < 0.f ? 0.f : 0x1p35f * (lost_a + lost_b);
}

// Such a sum as fp32 products of the operands themselves: this wave's share of it among `waves`.
__device__ __forceinline__ float share_again(const DenseProduct& p, int m, int n, int wave, int waves, int lane)
{
    const float *const a = p.values_a + m * p.ld_values_a, *const b = p.values_b + n * p.ld_values_b;
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
    for (int k = 256 * wave + 4 * lane; k + 4 <= p.values_k; k += 256 * waves) {
        const u32x4 u = words_at<4>(a + k), v = words_at<4>(b + k);
#pragma unroll
        for (int i = 0; i < 4; ++i) s[i] = __builtin_fmaf(__uint_as_float(u[i]), __uint_as_float(v[i]), s[i]);
    }
    const int tail = p.values_k / 4 * 4 + lane;
    if (wave == 0 && tail < p.values_k) s[0] = __builtin_fmaf(a[tail], b[tail], s[0]);
    float sum = (s[0] + s[1]) + (s[2] + s[3]);
#pragma unroll
    for (int d = 1; d < 64; d *= 2) sum += __shfl_xor(sum, d);
    return sum;
}

// Columns that a lane finishes: 16 bytes of the output.
template <int DT> constexpr int FINISH_COLUMNS = DT == IOLB_F32 ? 4 : 8;

// W columns of row m, which 32 / W neighbouring lanes continue to a checkpoint's block.  Every lane of the wave calls.
template <int DT, int ACT, int W>
__device__ __forceinline__ void finish_columns(const DenseFinish& f, int m, int n, const float (&bias)[W], float (&z)[W])
{
    const bool live = m < f.M && n < f.N;
#pragma unroll
    for (int i = 0; i < W; ++i) z[i] += bias[i];
    if (live && f.residual && f.first) add_residual<DT>(f, m, n, z);
    if (f.zq) {
        unsigned codes[W / 4];
        int e;
        ckpt_codes<DT, W, CKPT_BLOCK / W>(z, f.N - n, codes, e);
        if (live) store_codes<W>(f, m, n, codes, e);
    }
    if (live) store_columns<DT, ACT>(f, m, n, z);
}

}  // namespace iolb

#endif
