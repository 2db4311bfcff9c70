// Dropout whose mask is a function of key and counter, with residual and 8-bit checkpoint.
#include "block.h"
#include "dense_math.h"

namespace iolb {

namespace {

// Philox4x32 with ten rounds (Salmon, Moraes, Dror, Shaw, "Parallel random numbers: as easy as 1, 2, 3", 2011).
__device__ __forceinline__ u32x4 philox(unsigned long long low, unsigned long long high, unsigned long long key)
{
    unsigned c0 = (unsigned)low, c1 = (unsigned)(low >> 32), c2 = (unsigned)high, c3 = (unsigned)(high >> 32);
    unsigned k0 = (unsigned)key, k1 = (unsigned)(key >> 32);
#pragma unroll
    for (int round = 0; round < 10; ++round) {
        const unsigned long long a = (unsigned long long)c0 * 0xD2511F53u, b = (unsigned long long)c2 * 0xCD9E8D57u;
        const unsigned n0 = (unsigned)(b >> 32) ^ c1 ^ k0, n2 = (unsigned)(a >> 32) ^ c3 ^ k1;
        c1 = (unsigned)b;
        c3 = (unsigned)a;
        c0 = n0;
        c2 = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

// A thread takes the eight columns of a counter, a workgroup `wide` threads of a row and 256 / wide rows; four threads hold a checkpoint's block.
template <int DT>
__global__ void __launch_bounds__(256)
dropout_kernel(Dropout p, int wide_log)
{
    typedef typename DenseType<DT>::type T;
    const int wide = 1 << wide_log, tx = threadIdx.x & (wide - 1), ty = threadIdx.x >> wide_log;
    const int c = (int)((blockIdx.x * (unsigned)wide + tx) * 8);
    const long long counters = (p.cols + 7) / 8, blocks = (p.cols + CKPT_BLOCK - 1) / CKPT_BLOCK;
    unsigned long long seed = p.seed, offset = p.offset;
    if (p.counter) {
        seed += p.counter[0];
        offset += p.counter[1];
    }
    for (long long r = (long long)blockIdx.y * (256 >> wide_log) + ty; r - ty < p.rows; r += (long long)gridDim.y * (256 >> wide_log)) {
        const int have = r < p.rows ? p.cols - c : 0;
        float v[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (have > 0) {
            // (a rounding before the residual and one behind it, however the two are joined)
#pragma clang fp contract(off)
            load_columns(static_cast<const T*>(p.x) + r * p.ldx + c, have, v);
            const u32x4 bits = philox((unsigned long long)(r * counters + c / 8), offset, seed);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = (bits[i / 2] >> 16 * (i % 2) & 0xffffu) >= p.least ? v[i] * p.scale : 0.f;
            if (p.residual) {
                float res[8];
                load_columns(static_cast<const T*>(p.residual) + r * p.ldr + c, have, res);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = v[i] + res[i];
            }
            typename Piece<T, 8>::type t;
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                t[i] = (T)v[i];
                v[i] = i < have ? (float)t[i] : 0.f;
            }
            T* const to = static_cast<T*>(p.y) + r * p.ldy + c;
            if (have >= 8) {
                *reinterpret_cast<typename Piece<T, 8>::type*>(to) = t;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < have) to[i] = t[i];
            }
        }
        if (!p.zq) continue;
        unsigned words[2];
        int e;
        ckpt_codes<DT, 8, 4>(v, have, words, e);
        if (have <= 0) continue;
        typedef unsigned Codes __attribute__((ext_vector_type(2), aligned(1)));
        int8_t* const to = p.zq + r * p.cols + c;
        if (have >= 8) {
            *reinterpret_cast<Codes*>(to) = Codes{words[0], words[1]};
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (i < have) to[i] = (int8_t)(words[i / 4] >> 8 * (i % 4));
        }
        if (c % CKPT_BLOCK == 0) p.ze[r * blocks + c / CKPT_BLOCK] = (uint8_t)(e + 127);
    }
}

}  // namespace

hipError_t launch_dropout(const Dropout& p, int dtype, hipStream_t st)
{
    int wide_log = 2;                               // whole blocks of 32
    while (wide_log < 8 && (8LL << wide_log) < p.cols) ++wide_log;
    const long long gx = (p.cols + (8LL << wide_log) - 1) / (8LL << wide_log), per = 256 >> wide_log, gy = (p.rows + per - 1) / per;
    const dim3 grid((unsigned)gx, (unsigned)(gy < 65535 ? gy : 65535));
    if (dtype == IOLB_F32) dropout_kernel<IOLB_F32><<<grid, 256, 0, st>>>(p, wide_log);
    else if (dtype == IOLB_F16) dropout_kernel<IOLB_F16><<<grid, 256, 0, st>>>(p, wide_log);
    else dropout_kernel<IOLB_BF16><<<grid, 256, 0, st>>>(p, wide_log);
    return hipGetLastError();
}

}  // namespace iolb
