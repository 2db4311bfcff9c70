// Products with few rows (single tokens and small batches): C[m][n] = sum_k A[m][k] B[n][k], or with B summed along its rows
// (across: C[m][n] = sum_k A[m][k] B[k][n], the input's gradient).  What bounds them is reading B once, so B goes from memory
// straight to the registers of the one wave that multiplies it, as the caller holds it; fp32 values are cut into their three
// bf16 parts there (5.5 vector instructions a value).
//
// Measured, kernel alone: 1 x 4096 -> 4096 bf16 8.2 us (4.1 TB/s of weights), 1 x 512 -> 1000 fp32 4.7 us (latency: the launch, one trip to memory,
// the waves' sums through LDS); 64 x 25088 -> 4096 fp32 96 us and a join of 5 (4.3 TB/s; its six bf16 products would take 48 us at the
// rate of large library products); across, 64 x 4096 -> 25088 fp32 with its join 111-115 us by itself (3.6 TB/s; with every load of B from the same 64 rows,
// in cache, 107 of 116: matrix and vector instructions bind it), and 139 in a whole backward call, whose other kernels leave less of B in the caches.
//
// Infinities, NaN and values whose leading part rounds to infinity make sums that are not finite; a workgroup that meets one
// takes its sums again, now with parts that are zero beside such values, and the product of leading parts last (dense.h).
#include "dense_math.h"
#include "kernels.h"

#include <cmath>

namespace iolb {

namespace {

constexpr int STEP = 64;                              // k of a step
enum { ALL_PRODUCTS, SMALL_PRODUCTS, LEADING_PRODUCT };   // the last two: taken again, in this order

// Two fp32 values in three bf16 parts each, packed.  SAFE: nothing beside a value that is not finite, and none that rounds to infinity.
template <bool SAFE>
__device__ __forceinline__ void parts_of_two(float a, float b, unsigned& h, unsigned& m, unsigned& l)
{
    if constexpr (SAFE) {
        unsigned short h0, m0, l0, h1, m1, l1;
        dense_parts(a, h0, m0, l0);
        dense_parts(b, h1, m1, l1);
        h = h0 | (unsigned)h1 << 16;
        m = m0 | (unsigned)m1 << 16;
        l = l0 | (unsigned)l1 << 16;
    } else {
        const bf16x2 hv = {(__bf16)a, (__bf16)b};
        h = packed(hv);
        const float ra = a - __uint_as_float(h << 16), rb = b - __uint_as_float(h & 0xffff0000u);
        const bf16x2 mv = {(__bf16)ra, (__bf16)rb};
        m = packed(mv);
        const float sa = ra - __uint_as_float(m << 16), sb = rb - __uint_as_float(m & 0xffff0000u);
        const bf16x2 lv = {(__bf16)sa, (__bf16)sb};
        l = __builtin_bit_cast(unsigned, lv);
    }
}

// The operand of a lane for 32 k, in one part (16-bit types) or three.
template <int DT> struct Fragment { u32x4 part[DT == IOLB_F32 ? 3 : 1]; };

// c[i] += a[i % NA] b[i / NA], smallest products of parts first; product by product, so that neighbouring matrix instructions do not wait for
// each other's sums.
template <int DT, int MODE, int NA, int NB>
__device__ __forceinline__ void multiply_parts(const Fragment<DT> (&b)[NB], const Fragment<DT> (&a)[NA], f32x4* const (&c)[NA * NB])
{
    constexpr int part_b[6] = {2, 0, 1, 1, 0, 0}, part_a[6] = {0, 2, 1, 0, 1, 0};
    constexpr int from = DT != IOLB_F32 || MODE == LEADING_PRODUCT ? 5 : 0, to = DT == IOLB_F32 && MODE == SMALL_PRODUCTS ? 5 : 6;
#pragma unroll
    for (int q = from; q < to; ++q)
#pragma unroll
        for (int i = 0; i < NA * NB; ++i)
            *c[i] = multiply<DT == IOLB_F16>(b[i / NA].part[DT == IOLB_F32 ? part_b[q] : 0], a[i % NA].part[DT == IOLB_F32 ? part_a[q] : 0], *c[i]);
}

// Eight values of a row as they lie in memory.  fp32: two runs of four, so that four lanes read 64 neighbouring bytes at a time.
template <int DT> struct Raw { u32x4 v[DT == IOLB_F32 ? 2 : 1]; };

// How a step is read.  WHOLE: all of it exists.  ENDING: pieces are read from where they still end with the row (rows have eight values or more) and
// moved down; what comes in is zero (4 x 14464 x 1151 fp16, whose last step was read value by value: 37 us, now 26).  The kinds have loops of
// their own: where two meet in one, the compiler waits for all loads on their way, and what was asked for ahead is lost.
enum { WHOLE, ENDING };

// 128 bits moved down by 16 n (0 ... 8) bits.
__device__ __forceinline__ u32x4 moved_down(const u32x4& v, int n)
{
    unsigned long long lo = v[0] | (unsigned long long)v[1] << 32, hi = v[2] | (unsigned long long)v[3] << 32;
    const int s = 16 * (n & 3);
    lo = s ? lo >> s | hi << (64 - s) : lo;
    hi = s ? hi >> s : hi;
    if (n & 4) { lo = hi; hi = 0; }
    if (n & 8) lo = hi = 0;
    return u32x4{(unsigned)lo, (unsigned)(lo >> 32), (unsigned)hi, (unsigned)(hi >> 32)};
}

// The N values at p (16 bytes) of a row in which `have` are left from there on; the others are zero.
template <int N, bool ODD = false, class T>
__device__ __forceinline__ u32x4 ending_at(const T* p, int have)
{
    const int in = have < 0 ? 0 : have < N ? have : N;
    const T* const at = p + (have < N ? have : N) - N;
    if constexpr (ODD) return moved_down(words_at_odd(at), (N - in) * (8 / N));
    else return moved_down(words_at<4>(at), (N - in) * (8 / N));
}

// Piece g of 32 values that start at p, of which `have` exist.
template <int DT, int KIND, bool ODD = false>
__device__ __forceinline__ void load_raw(Raw<DT>& r, const typename DenseType<DT>::type* p, int g, int have)
{
    if constexpr (KIND == WHOLE) {
        if constexpr (DT == IOLB_F32) {
            r.v[0] = words_at<4>(p + 4 * g);
            r.v[1] = words_at<4>(p + 16 + 4 * g);
        } else {
            if constexpr (ODD) r.v[0] = words_at_odd(p + 8 * g);
            else r.v[0] = words_at<4>(p + 8 * g);
        }
    } else {
        if constexpr (DT == IOLB_F32) {
            r.v[0] = ending_at<4>(p + 4 * g, have - 4 * g);
            r.v[1] = ending_at<4>(p + 16 + 4 * g, have - 16 - 4 * g);
        } else {
            r.v[0] = ending_at<8, ODD>(p + 8 * g, have - 8 * g);
        }
    }
}

// What was loaded ahead is first used here and not earlier: the compiler, free to, moves the arithmetic on it up to the load, across the barrier
// and into the step before, and waits for it there.
template <int DT>
__device__ __forceinline__ void used_from_here(Raw<DT>& r)
{
#pragma unroll
    for (auto& v : r.v) asm volatile("" : "+v"(v));
}

template <int DT, bool SAFE>
__device__ __forceinline__ void cut(const Raw<DT>& r, Fragment<DT>& f)
{
    if constexpr (DT == IOLB_F32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            unsigned h, m, l;
            parts_of_two<SAFE>(__uint_as_float(r.v[i / 2][2 * (i % 2)]), __uint_as_float(r.v[i / 2][2 * (i % 2) + 1]), h, m, l);
            f.part[0][i] = h; f.part[1][i] = m; f.part[2][i] = l;
        }
    } else {
        f.part[0] = r.v[0];
    }
}

__device__ __forceinline__ bool all_finite(const f32x4& c)
{
    return fabsf(c[0]) < __builtin_inff() && fabsf(c[1]) < __builtin_inff() && fabsf(c[2]) < __builtin_inff() && fabsf(c[3]) < __builtin_inff();
}
__device__ __forceinline__ void clear_not_finite(f32x4& c)
{
#pragma unroll
    for (int i = 0; i < 4; ++i) c[i] = fabsf(c[i]) < __builtin_inff() ? c[i] : 0.f;
}

// Steps from s0 on up to the one returned exist whole.
__device__ __forceinline__ int whole_steps(const DenseProduct& p, int s0, int s1)
{
    const int full = p.K / STEP;
    return full < s0 ? s0 : full < s1 ? full : s1;
}

template <int N> using Constant = std::integral_constant<int, N>;

__device__ __forceinline__ void keep_partial(const DenseProduct& p, int split, int m, int n, const f32x4& c)
{
    const long long ld = (p.N + 3) / 4 * 4;
    if (m < p.M && n < p.N) *reinterpret_cast<f32x4*>(p.partial + ((long long)split * p.M + m) * ld + n) = c;
}

// ---- up to sixteen rows: the eight waves of a workgroup share K of sixteen columns of C -----------------------
// A step of a wave is 64 k: of B sixteen rows (16 lanes) by 64 or 128 neighbouring bytes at a time (4 lanes), of A likewise, from L2.
// The waves take the steps in turn, so that a workgroup reads runs of 8 * 64 values of a row.  Sixteen waves are no faster, and neither are steps
// three, four or six ahead.
template <int DT, bool ODD>
__global__ void __launch_bounds__(512)
dense_few_kernel(DenseProduct p, int join)
{
    typedef typename DenseType<DT>::type T;
    constexpr int WAVES = 8, AHEAD = 2;
    __shared__ __align__(16) f32x4 shares[WAVES][64];
    const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int n0 = blockIdx.x * 16;
    const int steps_all = (p.K + STEP - 1) / STEP;
    const int s0 = (int)((long long)steps_all * blockIdx.y / p.splits), s1 = (int)((long long)steps_all * (blockIdx.y + 1) / p.splits);
    // rows that do not exist are read from the last one: their sums are not stored
    const T* const b = static_cast<const T*>(p.b) + (n0 + l16 < p.N ? n0 + l16 : p.N - 1) * p.ldb;
    const T* const a = static_cast<const T*>(p.a) + (l16 < p.M ? l16 : p.M - 1) * p.lda;

    const int whole_to = whole_steps(p, s0, s1);
    float bias[4] = {0.f, 0.f, 0.f, 0.f};                              // (on its way while the products are taken)
    if (!join && n0 + 4 * grp < p.N) load_bias<DT>(p.f, n0 + 4 * grp, bias);
    // the sums of steps from ... to - 1, of which this wave has every eighth
    auto range = [&](auto mode, auto kind, int from, int to, f32x4 (&c)[2]) __attribute__((always_inline)) {
        constexpr int MODE = decltype(mode)::value, KIND = decltype(kind)::value;
        Raw<DT> rb[AHEAD][2], ra[AHEAD][2];
        auto load = [&](int s, Raw<DT> (&to_b)[2], Raw<DT> (&to_a)[2]) __attribute__((always_inline)) {
#pragma unroll
            for (int kk = 0; kk < 2; ++kk) {
                const int k = s * STEP + 32 * kk;
                load_raw<DT, KIND, ODD>(to_b[kk], b + k, grp, p.K - k);
                load_raw<DT, KIND, ODD>(to_a[kk], a + k, grp, p.K - k);
            }
        };
        const int first = from + ((wave - (from - s0)) & (WAVES - 1));          // (an ending goes to the wave that is next)
        if (first >= to) return;
        // (only what exists is loaded ahead: most waves have one to three steps, and the last ones again instead of a condition, which costs nothing
        // in a long run, made 16 x 1648 -> 1600 fp32 11.7 us of 8.0)
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (first + i * WAVES < to) load(first + i * WAVES, rb[i], ra[i]);
        for (int s = first; s < to; s += AHEAD * WAVES) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (s + i * WAVES < to) {
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk) {
                        Fragment<DT> fb[1], fa[1];
                        used_from_here<DT>(rb[i][kk]);
                        used_from_here<DT>(ra[i][kk]);
                        cut<DT, MODE != ALL_PRODUCTS>(rb[i][kk], fb[0]);
                        cut<DT, MODE != ALL_PRODUCTS>(ra[i][kk], fa[0]);
                        multiply_parts<DT, MODE, 1, 1>(fb, fa, {&c[kk]});
                    }
                    if (s + (i + AHEAD) * WAVES < to) load(s + (i + AHEAD) * WAVES, rb[i], ra[i]);
                }
            }
        }
    };
    auto sums = [&](auto mode) __attribute__((always_inline)) {
        f32x4 c[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
        range(mode, Constant<WHOLE>{}, s0, whole_to, c);
        range(mode, Constant<ENDING>{}, whole_to, s1, c);
        return c[0] + c[1];
    };
    f32x4 c = sums(std::integral_constant<int, ALL_PRODUCTS>{});
    if constexpr (DT == IOLB_F32) {
        if (__any(!all_finite(c))) {                                     // (nothing is shared yet: a wave may decide for itself)
            c = sums(std::integral_constant<int, SMALL_PRODUCTS>{});
            clear_not_finite(c);
            c += sums(std::integral_constant<int, LEADING_PRODUCT>{});
        }
    }
    shares[wave][lane] = c;
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int w = 1; w < WAVES; ++w) c += shares[w][lane];
    const int m = l16, n = n0 + 4 * grp;
    if (join) {
        keep_partial(p, blockIdx.y, m, n, c);
    } else {
        finish_four<DT>(p.f, m, n, bias, c);
    }
}

// ---- more rows: A through LDS, 64 rows at a time, each wave its own columns of C -------------------------------------------------
// A step is 64 k.  A's rows are cut into parts once for the workgroup and lie in two LDS buffers in turn; the loads of A two steps
// ahead and of B one are kept in registers.  Along (not across): a wave takes sixteen or thirty-two rows of B.  Across: 32 columns of
// B, two neighbours a lane, so that the eight rows a lane reads are its operand's eight k for each of the two without
// an exchange between lanes (four neighbours a lane read longer runs, but leave half as many workgroups to a compute unit: slower).
constexpr int NC = 2;                                  // columns of B that a lane reads side by side, across
constexpr int rows_waves(bool across) { return across ? 4 : 8; }
// Fragments of B of a wave.  Along, each reads all of A's from LDS, and from 65 rows on that binds: with two they serve twice the columns, but there are half as
// many workgroups.  One against two, fp32, us: 256 x 6456 -> 12224 322 / 233, 96 x 25088 -> 4096 181 / 154, 256 x 4096 -> 4096 57 / 54,
// 128 x 4096 -> 4096 34 / 35, 256 x 2048 -> 2048 22 / 28; 64 x 6456 -> 12224 86 / 89.
constexpr int rows_side(long long M, long long N, long long K, bool across) { return across ? NC : M > 64 && M * N * K >= 4000000000LL ? 2 : 1; }
// workgroups on a compute unit, by their registers: of 16 rows or less, of 17 to 32, of more
constexpr int rows_resident(int dtype, int tiles, bool across)
{
    return across ? (dtype == IOLB_F32 ? (tiles > 2 ? 2 : 3) : (tiles > 2 ? 3 : 4)) : (tiles > 2 ? 1 : 2);
}

template <int DT, int MT, bool ACROSS, int NF>
__global__ void __launch_bounds__(64 * rows_waves(ACROSS), rows_waves(ACROSS) * rows_resident(DT, MT, ACROSS) / 4)
dense_rows_kernel(DenseProduct p, int join)
{
    typedef typename DenseType<DT>::type T;
    constexpr int WAVES = rows_waves(ACROSS), THREADS = 64 * WAVES, COLS = 16 * NF, PARTS = DT == IOLB_F32 ? 3 : 1;
    constexpr int ROWS = 16 * MT, ITEMS = ROWS * 8, PER = (ITEMS + THREADS - 1) / THREADS;
    constexpr int WORDS = DT == IOLB_F32 ? NF : NF / 2;                   // of a lane and row of B, across
    constexpr int UNITS = 2;
    __shared__ __align__(16) u32x4 rows[2][PARTS][ROWS * 8];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const T* const a = static_cast<const T*>(p.a);
    const T* const b = static_cast<const T*>(p.b);
    const int m0 = blockIdx.y * ROWS;
    const long long steps = (p.K + STEP - 1) / STEP, total = steps * ((p.N + WAVES * COLS - 1) / (WAVES * COLS));
    const long long end = (blockIdx.x + 1LL) * p.per < total ? (blockIdx.x + 1LL) * p.per : total;
    // the workgroup's run of steps, block by block
    for (long long at_step = (long long)blockIdx.x * p.per; at_step < end;) {
    const int block = (int)(at_step / steps), s0 = (int)(at_step % steps), s1 = (int)(steps < s0 + end - at_step ? steps : s0 + end - at_step);
    at_step += s1 - s0;
    const int n0 = (block * WAVES + wave) * COLS;
    // rows (columns) that do not exist are read from the last one: their sums are not stored
    int along_row[NF];
#pragma unroll
    for (int j = 0; j < NF; ++j) along_row[j] = n0 + 16 * j + l16 < p.N ? n0 + 16 * j + l16 : p.N - 1;
    const int first_col = n0 + NC * l16;
    const int whole_to = whole_steps(p, s0, s1);
    const bool edge = ACROSS && first_col == p.N - 1;            // (a pair of columns ends there: it is read one column earlier)
    const T* const across_col = ACROSS ? b + (first_col < p.N - NC ? first_col : p.N - NC) : b;
    const T* const across_at = across_col + 8 * grp * p.ldb;
    f32x4 acc[MT][NF];

    auto range = [&](auto mode, auto kind, int from, int to) __attribute__((always_inline)) {
        constexpr int MODE = decltype(mode)::value, KIND = decltype(kind)::value;
        constexpr bool SAFE = MODE != ALL_PRODUCTS;
        if (from >= to) return;
        // ---- B in registers: 32 k of sixteen NF rows, or of 32 columns
        struct Unit { Raw<DT> along[ACROSS ? 1 : NF]; unsigned across[8][ACROSS ? WORDS : 1]; };
        Unit ub[UNITS];
        auto load_b = [&](int k, Unit& u) __attribute__((always_inline)) {                     // k: of the unit's first
            if constexpr (!ACROSS) {
#pragma unroll
                for (int j = 0; j < NF; ++j) load_raw<DT, KIND>(u.along[j], b + along_row[j] * p.ldb + k, grp, p.K - k);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int row = k + 8 * grp + i;
                    // (whole: a lane's part of the address stays, the step's part is the same for all lanes)
                    const T* const at = KIND == WHOLE ? across_at + (long long)(k + i) * p.ldb : across_col + (row < p.K ? row : p.K - 1) * p.ldb;
                    const auto t = words_at<WORDS>(at);
#pragma unroll
                    for (int w = 0; w < WORDS; ++w) u.across[i][w] = KIND == WHOLE || row < p.K ? t[w] : 0u;
                }
            }
        };
        // ---- A: registers, then LDS (across: plain order of k, as the eight rows of B that a lane reads are neighbours)
        Raw<DT> ra[PER];
        auto load_a = [&](int s) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int item = tid + i * THREADS, row = m0 + (item >> 3), piece = item & 7, g = piece & 3;
                const T* const at = a + (row < p.M ? row : p.M - 1) * p.lda + s * STEP + 32 * (piece >> 2);
                const int have = p.K - s * STEP - 32 * (piece >> 2);
                if constexpr (ACROSS && DT == IOLB_F32) {
                    if constexpr (KIND == WHOLE) {
                        ra[i].v[0] = words_at<4>(at + 8 * g);
                        ra[i].v[1] = words_at<4>(at + 8 * g + 4);
                    } else {
                        ra[i].v[0] = ending_at<4>(at + 8 * g, have - 8 * g);
                        ra[i].v[1] = ending_at<4>(at + 8 * g + 4, have - 8 * g - 4);
                    }
                } else {
                    load_raw<DT, KIND>(ra[i], at, g, have);
                }
            }
        };
        auto store_a = [&](int buf) __attribute__((always_inline)) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int item = tid + i * THREADS, row = item >> 3, piece = item & 7;
                if (ITEMS % THREADS == 0 || item < ITEMS) {
                    Fragment<DT> f;
                    used_from_here<DT>(ra[i]);
                    cut<DT, SAFE>(ra[i], f);
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) rows[buf][q][row * 8 + place(row, piece)] = f.part[q];
                }
            }
        };
        __syncthreads();                                      // (an earlier range's last step may still be read)
        load_a(from);
        store_a(from & 1);
        // In the order of the loop, A before B: a wait for A at its head then leaves B on its way.  (Beyond the last step B's last is loaded
        // again: without a condition on them, loads ahead stay in their registers.)
        if (from + 1 < to) load_a(from + 1);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) {
            load_b(from * STEP + 32 * u, ub[u]);
            __builtin_amdgcn_sched_barrier(0);
        }
        for (int s = from; s < to; ++s) {
            const int after = s + 1 < to ? s + 1 : s;
            __syncthreads();
            if (s + 1 < to) store_a((s + 1) & 1);
            if (s + 2 < to) load_a(s + 2);
            __builtin_amdgcn_sched_barrier(0);                // loads ahead are issued here, not where their registers are used
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                Fragment<DT> fb[NF];
                if constexpr (!ACROSS) {
#pragma unroll
                    for (int j = 0; j < NF; ++j) {
                        used_from_here<DT>(ub[u].along[j]);
                        cut<DT, SAFE>(ub[u].along[j], fb[j]);
                    }
                } else {
#pragma unroll
                    for (auto& row : ub[u].across) {
#pragma unroll
                        for (unsigned& v : row) asm volatile("" : "+v"(v));
                        row[0] = !edge ? row[0] : WORDS == 2 ? row[WORDS - 1] : row[0] >> 16;
                    }
#pragma unroll
                    for (int j = 0; j < NF; ++j)
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            if constexpr (DT == IOLB_F32) {
                                unsigned h, m, l;
                                parts_of_two<SAFE>(__uint_as_float(ub[u].across[2 * i][j]), __uint_as_float(ub[u].across[2 * i + 1][j]), h, m, l);
                                fb[j].part[0][i] = h; fb[j].part[1][i] = m; fb[j].part[2][i] = l;
                            } else {
                                // column j of rows 2 i and 2 i + 1, side by side
                                fb[j].part[0][i] = __builtin_amdgcn_perm(ub[u].across[2 * i + 1][j / 2], ub[u].across[2 * i][j / 2],
                                                                         j % 2 ? 0x07060302u : 0x05040100u);
                            }
                        }
                }
                __builtin_amdgcn_sched_barrier(0);
                load_b(after * STEP + 32 * u, ub[u]);
                if constexpr (!ACROSS) __builtin_amdgcn_sched_barrier(0);
                Fragment<DT> fa[MT];
                f32x4* sum[MT * NF];
#pragma unroll
                for (int i = 0; i < MT; ++i) {
                    const int row = 16 * i + l16;
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) fa[i].part[q] = rows[s & 1][q][row * 8 + place(row, 4 * u + grp)];
#pragma unroll
                    for (int j = 0; j < NF; ++j) sum[j * MT + i] = &acc[i][j];
                }
                multiply_parts<DT, MODE, MT, NF>(fb, fa, sum);
            }
        }
    };
    auto sums = [&](auto mode) __attribute__((always_inline)) {
        range(mode, Constant<WHOLE>{}, s0, whole_to);
        range(mode, Constant<ENDING>{}, whole_to, s1);
    };
    auto clear = [&](bool all) {
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int j = 0; j < NF; ++j) {
                if (all) acc[t][j] = f32x4{0, 0, 0, 0};
                else clear_not_finite(acc[t][j]);
            }
    };
    clear(true);
    sums(std::integral_constant<int, ALL_PRODUCTS>{});
    if constexpr (DT == IOLB_F32) {
        bool fine = true;
#pragma unroll
        for (int t = 0; t < MT; ++t)
#pragma unroll
            for (int j = 0; j < NF; ++j) fine = fine && all_finite(acc[t][j]);
        if (__syncthreads_or(!fine)) {
            clear(true);
            sums(std::integral_constant<int, SMALL_PRODUCTS>{});
            clear(false);
            sums(std::integral_constant<int, LEADING_PRODUCT>{});
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = m0 + 16 * t + l16;
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            // across: column NC (4 grp + r) + j of the wave's is value r of fragment j
            const int n = n0 + (ACROSS ? 4 * NC * grp + 4 * i : 16 * i + 4 * grp);
            f32x4 c = acc[t][i];
            if constexpr (ACROSS) {
#pragma unroll
                for (int v = 0; v < 4; ++v) c[v] = acc[t][(4 * i + v) % NC][(4 * i + v) / NC];
            }
            if (join) {
                keep_partial(p, (int)(blockIdx.x - block * steps / p.per), m, n, c);
            } else {
                float bias[4] = {0.f, 0.f, 0.f, 0.f};
                if (n < p.N) load_bias<DT>(p.f, n, bias);
                finish_four<DT>(p.f, m, n, bias, c);
            }
        }
    }
    }
}

// ---- products of which the summed axis is short (the weights' gradient of up to 64 rows): bound by writing C ---------
// A is [M][K], B [N][K], K at most 64, both in planes.  A wave keeps sixteen NT rows of A in registers and goes along a run of columns: their
// fragments of B come from L2, 64 columns ahead, there is neither LDS nor a barrier, and the stores stream.  A lane ends with 16 bytes of
// neighbouring columns of one row (16-bit types: rows r of two tiles are columns 8 (r / 4) + r % 4 and four further), four lanes with 64; the lanes of
// two rows exchange pieces, so that a store writes whole lines of 128 bytes.
// Calls with their layouts, 4096 x 25088 from 64 rows, fp32 (411 MB written, a fill takes 62 us): 92 us, with stores of 64 bytes 99; bf16 59 of 63.  In a whole
// backward call, behind dx, the kernel alone takes 105.

// Neighbouring lanes: the even one keeps a and gives b, the odd one keeps b and gives a; a is of the even lane's row then, b of the odd one's.
__device__ __forceinline__ void exchange(u32x4& a, u32x4& b, bool odd)
{
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        const unsigned give = odd ? a[r] : b[r];
        const unsigned got = (unsigned)__builtin_amdgcn_mov_dpp((int)give, 0xB1, 0xf, 0xf, true);      // (lane ^ 1's)
        a[r] = odd ? got : a[r];
        b[r] = odd ? b[r] : got;
    }
}

template <int DT, int PB, int KK>
__global__ void __launch_bounds__(256, PB == 3 ? 1 : KK == 2 ? 2 : 3)
dense_outer_kernel(DenseProduct p, long long plane_a, long long plane_b)
{
    constexpr int PA = DT == IOLB_F32 ? 3 : 1, NT = DT == IOLB_F32 ? 2 : 4, AHEAD = DT == IOLB_F32 ? 2 : 1;
    constexpr int TILES = DT == IOLB_F32 ? 2 : 4, COLUMNS = 16 * TILES, EACH = DT == IOLB_F32 ? 4 : 8;       // EACH: columns of a piece of 16 bytes
    typedef typename DenseType<DT>::type T;
    const int lane = threadIdx.x & 63, l16 = lane & 15, grp = lane >> 4;
    const int m0 = (blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * 16 * NT;
    if (m0 >= p.M) return;
    const unsigned short* const a = static_cast<const unsigned short*>(p.a);
    const unsigned short* const b = static_cast<const unsigned short*>(p.b);
    u32x4 fa[NT][KK][PA];
#pragma unroll
    for (int t = 0; t < NT; ++t)
#pragma unroll
        for (int kk = 0; kk < KK; ++kk)
#pragma unroll
            for (int q = 0; q < PA; ++q) {
                const int row = m0 + 16 * t + l16, k = 32 * kk + 8 * grp;
                fa[t][kk][q] = k < p.K ? *reinterpret_cast<const u32x4*>(a + q * plane_a + (row < p.M ? row : p.M - 1) * p.lda + k) : u32x4{0, 0, 0, 0};
            }
    const int n_from = blockIdx.x * p.per, n_to = n_from + p.per < p.N ? n_from + p.per : p.N;
    u32x4 fb[AHEAD][TILES][KK][PB];
    // (pieces beyond the summed axis: zero in A, any finite values here, so those of its first piece; B's rows beyond its last: that one's)
    auto load = [&](int n, u32x4 (&to)[TILES][KK][PB]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < TILES; ++j) {
            const int col = n + (DT == IOLB_F32 ? 16 * j + l16 : 32 * (j / 2) + 8 * (l16 >> 2) + 4 * (j % 2) + (l16 & 3));
            const unsigned short* const row = b + (col < p.N ? col : p.N - 1) * p.ldb;
#pragma unroll
            for (int kk = 0; kk < KK; ++kk) {
                const int k = 32 * kk + 8 * grp;
#pragma unroll
                for (int q = 0; q < PB; ++q) to[j][kk][q] = *reinterpret_cast<const u32x4*>(row + q * plane_b + (k < p.K ? k : 0));
            }
        }
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) load(n_from + COLUMNS * i, fb[i]);
    // EVERY: every store is a 16-byte piece that exists.  (Under conditions the stores' number is not known, and a wait for a load would be
    // one for the stores before it.)
    auto run = [&](auto every) __attribute__((always_inline)) {
    constexpr bool EVERY = decltype(every)::value;
    for (int n0 = n_from; n0 < n_to; n0 += COLUMNS * AHEAD) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) {
            const int n = n0 + COLUMNS * i;
            f32x4 c[NT][TILES] = {};
            constexpr int part_a[6] = {2, 0, 1, 1, 0, 0}, part_b[6] = {0, 2, 1, 0, 1, 0};
#pragma unroll
            for (int q = 0; q < 6; ++q) {
                if (part_a[q] >= PA || part_b[q] >= PB) continue;
                if (q == 5 && PB == 3) {
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < TILES; ++j) clear_not_finite(c[t][j]);
                }
#pragma unroll
                for (int kk = 0; kk < KK; ++kk)
#pragma unroll
                    for (int t = 0; t < NT; ++t)
#pragma unroll
                        for (int j = 0; j < TILES; ++j)
                            c[t][j] = multiply<DT == IOLB_F16>(fb[i][j][kk][part_b[q]], fa[t][kk][part_a[q]], c[t][j]);
            }
            load(n + COLUMNS * AHEAD < n_to ? n + COLUMNS * AHEAD : n_from, fb[i]);
            if (EVERY || n < n_to) {
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    const auto value = [&](int piece, int v) { return c[t][DT == IOLB_F32 ? piece : 2 * piece + v / 4][v % 4]; };
                    if constexpr (EVERY) {
                        typedef typename Piece<T, EACH>::type TW;
                        u32x4 z[2];
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            TW w;
#pragma unroll
                            for (int v = 0; v < EACH; ++v) w[v] = (T)value(g, v);
                            z[g] = __builtin_bit_cast(u32x4, w);
                        }
                        exchange(z[0], z[1], l16 & 1);
                        T* const to = static_cast<T*>(p.f.y) + (m0 + 16 * t + (l16 & ~1)) * p.f.ldy + n + EACH * (4 * (l16 & 1) + grp);
                        *reinterpret_cast<TW*>(to) = __builtin_bit_cast(TW, z[0]);
                        *reinterpret_cast<TW*>(to + p.f.ldy) = __builtin_bit_cast(TW, z[1]);
                    } else {
#pragma unroll
                        for (int g = 0; g < 2; ++g) {
                            const int m = m0 + 16 * t + l16, col = n + EACH * (4 * g + grp);
                            float z[EACH];
#pragma unroll
                            for (int v = 0; v < EACH; ++v) z[v] = value(g, v);
                            if (m < p.M && col < p.N) store_columns<DT, IOLB_ACT_NONE>(p.f, m, col, z);
                        }
                    }
                }
            }
        }
    }
    };
    if (m0 + 16 * NT <= p.M && (n_to - n_from) % (COLUMNS * AHEAD) == 0) run(std::true_type{});
    else run(std::false_type{});
}

template <int DT, int PB>
hipError_t launch_outer(DenseProduct p, long long plane_a, long long plane_b, hipStream_t st)
{
    const int rows = 4 * 16 * (DT == IOLB_F32 ? 2 : 4);
    const long long gy = ((long long)p.M + rows - 1) / rows;
    if (gy > 65535) return hipErrorInvalidValue;
    // a wave's run of columns: each starts with a wait for its rows of A, so there are at most eight waves to a SIMD, and two where that would make
    // runs shorter than 256 columns (4096 x 4096 fp32, runs of 64 31 us, of 256 28)
    const long long columns = (long long)p.N * gy * 4, eight = (columns / 8192 + 63) / 64 * 64, two = (columns / 2048 + 63) / 64 * 64;
    const long long run = eight >= 256 ? eight : two < 256 ? two : 256;
    p.per = (int)(run < 64 ? 64 : run > 4096 ? 4096 : run);
    const dim3 grid((unsigned)(((long long)p.N + p.per - 1) / p.per), (unsigned)gy);
    if (p.K <= 32) dense_outer_kernel<DT, PB, 1><<<grid, 256, 0, st>>>(p, plane_a, plane_b);
    else dense_outer_kernel<DT, PB, 2><<<grid, 256, 0, st>>>(p, plane_a, plane_b);
    return hipGetLastError();
}

// Workgroups of the kernel for more than DENSE_FEW rows along the first axis.
long long rows_groups(int M, int N, int K, int per, bool across)
{
    const int cols = rows_waves(across) * 16 * rows_side(M, N, K, across);
    const long long total = (K + STEP - 1LL) / STEP * ((N + cols - 1LL) / cols);
    return (total + per - 1) / per;
}

template <int DT>
hipError_t launch(const DenseProduct& p, bool across, bool join, hipStream_t st)
{
    if (!across && p.M <= DENSE_FEW) {
        const dim3 grid((p.N + 15) / 16, p.splits);
        const bool odd = DT != IOLB_F32 && ((reinterpret_cast<uintptr_t>(p.a) | reinterpret_cast<uintptr_t>(p.b)) % 4 || p.ldb % 2 || (p.M > 1 && p.lda % 2));
        if (odd) dense_few_kernel<DT, DT != IOLB_F32><<<grid, 512, 0, st>>>(p, join);
        else dense_few_kernel<DT, false><<<grid, 512, 0, st>>>(p, join);
        return hipGetLastError();
    }
    const int mt = p.M <= 16 ? 1 : p.M <= 32 ? 2 : 4;
    const int side = rows_side(p.M, p.N, p.K, across), threads = 64 * rows_waves(across);
    const dim3 grid((unsigned)rows_groups(p.M, p.N, p.K, p.per, across), (p.M + 16 * mt - 1) / (16 * mt));
    if (across) {
        if (mt == 1) dense_rows_kernel<DT, 1, true, NC><<<grid, threads, 0, st>>>(p, join);
        else if (mt == 2) dense_rows_kernel<DT, 2, true, NC><<<grid, threads, 0, st>>>(p, join);
        else dense_rows_kernel<DT, 4, true, NC><<<grid, threads, 0, st>>>(p, join);
    } else if constexpr (DT == IOLB_F32) {
        if (mt <= 2) dense_rows_kernel<DT, 2, false, 1><<<grid, threads, 0, st>>>(p, join);
        else if (side == 1) dense_rows_kernel<DT, 4, false, 1><<<grid, threads, 0, st>>>(p, join);
        else dense_rows_kernel<DT, 4, false, 2><<<grid, threads, 0, st>>>(p, join);
    } else {
        return hipErrorInvalidValue;                  // 16-bit types, along: up to DENSE_FEW rows only
    }
    return hipGetLastError();
}

}  // namespace

// How the steps are dealt out: the least modelled time.  Up to sixteen rows: `splits` workgroups share the K of sixteen columns.  Beyond: the steps of
// all blocks of columns, one after the other, are cut into equal runs, one a workgroup, so that every compute unit has the same to do (with
// whole shares of K, 196 blocks of 25088 columns left some with twice the others': 64 x 4096 -> 25088 fp32 across 117 us, dealt out evenly 113).  What a step
// takes lies between its share of the memory's bandwidth (4.9 TB/s) and its own latency `alone`; one goes before the first.  A second launch
// adds the partial sums, which go through memory.  Fitted to a sweep of 22 products of 1 to 64 rows and 0.5 M to 103 M weights, 1 to 64 shares.
DenseRowsPlan dense_rows_plan(int M, int N, int K, int dtype, bool across, bool checkpoint)
{
    const bool few = !across && M <= DENSE_FEW, wide = dtype == IOLB_F32;
    const int tiles = M <= 16 ? 1 : M <= 32 ? 2 : 4;
    const double alone = few ? (wide ? 1000 : 600) : !across ? (rows_side(M, N, K, false) == 2 ? 1600 : 1000) : !wide ? 550 : tiles == 1 ? 1050 : tiles == 2 ? 1350 : 1900;
    const long long steps = (K + STEP - 1) / STEP, cols = few ? 16 : rows_waves(across) * 16 * rows_side(M, N, K, across);
    const long long blocks = (N + cols - 1) / cols, waves = few ? 8 : 1;           // (few: the waves share the steps)
    const long long capacity = 256 * (few ? 2 : rows_resident(dtype, tiles, across)) / ((M + 63) / 64);   // (each 64 rows have workgroups of their own)
    const double step_ns = (double)cols * waves * STEP * (wide ? 4 : 2) / 4900;                        // of one workgroup
    DenseRowsPlan best{1, 0, checkpoint, 0};
    double least = -1;
    const auto consider = [&](long long groups, long long each, int pieces, const DenseRowsPlan& plan) {
        double ns = (double)(groups / capacity * (each + 1)) * std::hypot(alone, capacity * step_ns);
        if (groups % capacity) ns += (each + 1) * std::hypot(alone, groups % capacity * step_ns);
        if (pieces > 1) ns += 2000 + 80 * pieces + 8.0 * pieces * M * N / 10000;
        if (least < 0 || ns < least) { least = ns; best = plan; }
    };
    if (few) {
        for (int s = 1; s <= 64 && s <= steps; ++s)
            consider(blocks * s, (steps + s * waves - 1) / (s * waves), s, {s, 0, s > 1 || checkpoint, 0});
    } else {
        consider(blocks, steps, 1, {1, (int)steps, checkpoint, (int)cols});
        for (long long groups = 32; groups <= capacity; groups += groups < 256 ? 32 : 256) {
            const long long per = (blocks * steps + groups - 1) / groups;
            if (per >= steps) continue;
            const int pieces = (int)((steps + per - 2) / per + 1);            // of a block, at most
            consider((blocks * steps + per - 1) / per, per, pieces, {pieces, (int)per, true, (int)cols});
        }
    }
    return best;
}

bool dense_rows_launchable(const DenseRowsPlan& plan, int M, int N, int K, bool across)
{
    if (!across && M <= DENSE_FEW) return (N + 15LL) / 16 * 512 <= 0xffffffffLL;
    return rows_groups(M, N, K, plan.per, across) * 64 * rows_waves(across) <= 0xffffffffLL;
}

hipError_t launch_dense_outer(const DenseProduct& p, int planes_b, long long plane_a, long long plane_b, int dtype, hipStream_t st)
{
    if (dtype == IOLB_F32)
        return planes_b == 3 ? launch_outer<IOLB_F32, 3>(p, plane_a, plane_b, st) : launch_outer<IOLB_F32, 1>(p, plane_a, plane_b, st);
    return dtype == IOLB_F16 ? launch_outer<IOLB_F16, 1>(p, plane_a, plane_b, st) : launch_outer<IOLB_BF16, 1>(p, plane_a, plane_b, st);
}

hipError_t launch_dense_rows(const DenseProduct& p, bool across, bool join, int dtype, hipStream_t st)
{
    const hipError_t e = dtype == IOLB_F32 ? launch<IOLB_F32>(p, across, join, st)
                       : dtype == IOLB_F16 ? launch<IOLB_F16>(p, across, join, st) : launch<IOLB_BF16>(p, across, join, st);
    return e != hipSuccess || !join ? e : launch_dense_join(p, dtype, st);
}

}  // namespace iolb
