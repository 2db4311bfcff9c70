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
        const unsigned n0 = __builtin_amdgcn_bitop3_b32((unsigned)(b >> 32), c1, k0, 0x96), n2 = __builtin_amdgcn_bitop3_b32((unsigned)(a >> 32), c3, k1, 0x96);   // x ^ y ^ z
        c1 = (unsigned)b;
        c3 = (unsigned)a;
        c0 = n0;
        c2 = n2;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
    return u32x4{c0, c1, c2, c3};
}

// Eight values as memory holds them; zeros beyond the row's end.
template <class T> using Eight = typename Piece<T, 8>::type;

template <bool PAST, class T>
__device__ __forceinline__ Eight<T> load_eight(const T* p, int have)
{
    if (have >= 8) {
        if constexpr (PAST) return __builtin_nontemporal_load(reinterpret_cast<const Eight<T>*>(p));
        return *reinterpret_cast<const Eight<T>*>(p);
    }
    Eight<T> t;
#pragma unroll
    for (int i = 0; i < 8; ++i) t[i] = i < have ? p[i] : (T)0.f;
    return t;
}

// A thread takes the eight columns of a counter in one row after the other, the next one on its way meanwhile; a workgroup `wide` threads of a row and
// 256 / wide rows; four threads hold a checkpoint's block.  CHECKPOINT, RESIDUAL: whether there is one; PAST: past the caches.
// Memory and the generator's 20 products a counter bind it alike: 16384 x 8192 bf16 87 us (6.1 TB/s); through the caches 96, and 94 without the generator.
template <int DT, bool RESIDUAL, bool CHECKPOINT, bool PAST>
__global__ void __launch_bounds__(256)
dropout_kernel(Dropout p, int wide_log)
{
    typedef typename DenseType<DT>::type T;
    const int wide = 1 << wide_log, tx = threadIdx.x & (wide - 1), ty = threadIdx.x >> wide_log;
    const int c = (int)((blockIdx.x * (unsigned)wide + tx) * 8), have = p.cols - c;
    const long long counters = (p.cols + 7) / 8, blocks = (p.cols + CKPT_BLOCK - 1) / CKPT_BLOCK, step = (long long)gridDim.y * (256 >> wide_log);
    unsigned long long seed = p.seed, offset = p.offset;
    if (p.counter) {
        seed += p.counter[0];
        offset += p.counter[1];
    }
    // (of a word's halves the upper one is compared in place, the lower one moved up)
    const unsigned least = p.least << 16;
    const bool some = p.least < 65536;
    const T *const xs = static_cast<const T*>(p.x) + c, *const rs = static_cast<const T*>(p.residual) + c;
    long long r = (long long)blockIdx.y * (256 >> wide_log) + ty;
    Eight<T> x{}, res{};
    const auto load = [&](long long at) {
        if (at >= p.rows || have <= 0) return;
        x = load_eight<PAST>(xs + at * p.ldx, have);
        if constexpr (RESIDUAL) res = load_eight<PAST>(rs + at * p.ldr, have);
    };
    load(r);
    for (; r - ty < p.rows; r += step) {
        const bool live = r < p.rows && have > 0;
        const Eight<T> now = x, now_res = res;
        load(r + step);
        const u32x4 bits = philox((unsigned long long)(r * counters + c / 8), offset, seed);
        Eight<T> t;
        {
            // (a rounding before the residual and one behind it, however the two are joined)
#pragma clang fp contract(off)
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const unsigned u = i % 2 ? bits[i / 2] : bits[i / 2] << 16;
                float v = some && u >= least ? (float)now[i] * p.scale : 0.f;
                if constexpr (RESIDUAL) v = v + (float)now_res[i];
                t[i] = (T)v;
            }
        }
        if (live) {
            T* const to = static_cast<T*>(p.y) + r * p.ldy + c;
            if (have >= 8) {
                if constexpr (PAST) __builtin_nontemporal_store(t, reinterpret_cast<Eight<T>*>(to));
                else *reinterpret_cast<Eight<T>*>(to) = t;
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (i < have) to[i] = t[i];
            }
        }
        if constexpr (CHECKPOINT) {
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = live && i < have ? (float)t[i] : 0.f;
            unsigned words[2];
            int e;
            ckpt_codes<DT, 8, 4>(v, have, words, e);
            if (!live) continue;
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
}

// Workgroups, more than fill the chip at once (16384 x 8192 bf16: 2048 101 us, 4096 102, 8192 99, 16384 96, as many as rows take 120).
constexpr int GROUPS = 16384;

template <int DT, bool PAST>
void launch(const Dropout& p, const dim3& grid, int wide_log, hipStream_t st)
{
    if (p.zq && p.residual) dropout_kernel<DT, true, true, PAST><<<grid, 256, 0, st>>>(p, wide_log);
    else if (p.zq) dropout_kernel<DT, false, true, PAST><<<grid, 256, 0, st>>>(p, wide_log);
    else if (p.residual) dropout_kernel<DT, true, false, PAST><<<grid, 256, 0, st>>>(p, wide_log);
    else dropout_kernel<DT, false, false, PAST><<<grid, 256, 0, st>>>(p, wide_log);
}

template <int DT>
void launch(const Dropout& p, const dim3& grid, int wide_log, hipStream_t st)
{
    if (past_caches((double)p.rows * p.cols * (sizeof(typename DenseType<DT>::type) * (p.residual ? 3 : 2) + (p.zq ? 1 : 0)))) launch<DT, true>(p, grid, wide_log, st);
    else launch<DT, false>(p, grid, wide_log, st);
}

}  // namespace

hipError_t launch_dropout(const Dropout& p, int dtype, hipStream_t st)
{
    int wide_log = 2;                               // whole blocks of 32
    while (wide_log < 8 && (8LL << wide_log) < p.cols) ++wide_log;
    const long long gx = (p.cols + (8LL << wide_log) - 1) / (8LL << wide_log), per = 256 >> wide_log, gy = (p.rows + per - 1) / per;
    // (rows beyond what fills the chip are taken in turn)
    const long long most = (GROUPS + gx - 1) / gx;
    const dim3 grid((unsigned)gx, (unsigned)(gy < most ? gy : most));
    if (dtype == IOLB_F32) launch<IOLB_F32>(p, grid, wide_log, st);
    else if (dtype == IOLB_F16) launch<IOLB_F16>(p, grid, wide_log, st);
    else launch<IOLB_BF16>(p, grid, wide_log, st);
    return hipGetLastError();
}

}  // namespace iolb
