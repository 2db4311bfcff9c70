// Products with few rows (single tokens and small batches): C[m][n] = sum_k A[m][k] B[n][k], or with B summed along its rows
// (across: C[m][n] = sum_k A[m][k] B[k][n], the input's gradient).  What bounds them is reading B once, so B goes from memory
// straight to the registers of the one wave that multiplies it, as the caller holds it; fp32 values are cut into their three
// bf16 parts there (5.5 vector instructions a value).
//
// Infinities, NaN and values whose leading part rounds to infinity make sums that are not finite; a workgroup that meets one
// takes its sums again, now with parts that are zero beside such values, and the product of leading parts last (dense.h).
#include "dense_math.h"
#include "kernels.h"

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

template <int DT, int MODE>
__device__ __forceinline__ f32x4 multiply_parts(const Fragment<DT>& b, const Fragment<DT>& a, f32x4 c)
{
    if constexpr (DT != IOLB_F32) {
        return multiply<DT == IOLB_F16>(b.part[0], a.part[0], c);
    } else {
        if constexpr (MODE != LEADING_PRODUCT) {
            c = multiply<false>(b.part[2], a.part[0], c);
            c = multiply<false>(b.part[0], a.part[2], c);
            c = multiply<false>(b.part[1], a.part[1], c);
            c = multiply<false>(b.part[1], a.part[0], c);
            c = multiply<false>(b.part[0], a.part[1], c);
        }
        if constexpr (MODE != SMALL_PRODUCTS) c = multiply<false>(b.part[0], a.part[0], c);
        return c;
    }
}

// Eight values of a row as they lie in memory.  fp32: two runs of four, so that four lanes read 64 neighbouring bytes at a time.
template <int DT> struct Raw { u32x4 v[DT == IOLB_F32 ? 2 : 1]; };

// k of value i of piece g (0 ... 3) of 32
template <int DT>
__device__ __forceinline__ int k_of(int g, int i) { return DT == IOLB_F32 ? (i < 4 ? 4 * g + i : 12 + 4 * g + i) : 8 * g + i; }

// Piece g of 32 values that start at p, of which `have` exist (the others are zero).
template <int DT>
__device__ __forceinline__ void load_raw(Raw<DT>& r, const typename DenseType<DT>::type* p, int g, int have, bool vec)
{
    if (vec && have >= 32) {
        if constexpr (DT == IOLB_F32) {
            r.v[0] = *reinterpret_cast<const u32x4*>(p + 4 * g);
            r.v[1] = *reinterpret_cast<const u32x4*>(p + 16 + 4 * g);
        } else {
            r.v[0] = *reinterpret_cast<const u32x4*>(p + 8 * g);
        }
    } else if constexpr (DT == IOLB_F32) {
#pragma unroll
        for (int i = 0; i < 8; ++i) r.v[i / 4][i % 4] = k_of<DT>(g, i) < have ? __float_as_uint(p[k_of<DT>(g, i)]) : 0u;
    } else {
        const unsigned short* const q = reinterpret_cast<const unsigned short*>(p) + 8 * g;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const unsigned lo = 8 * g + 2 * i < have ? q[2 * i] : 0u, hi = 8 * g + 2 * i + 1 < have ? q[2 * i + 1] : 0u;
            r.v[0][i] = lo | hi << 16;
        }
    }
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

__device__ __forceinline__ void keep_partial(const DenseProduct& p, int split, int m, int n, const f32x4& c)
{
    const long long ld = (p.N + 3) / 4 * 4;
    if (m < p.M && n < p.N) *reinterpret_cast<f32x4*>(p.partial + ((long long)split * p.M + m) * ld + n) = c;
}

// ---- up to sixteen rows: the eight waves of a workgroup share K of sixteen columns of C -----------------------
// A step of a wave is 64 k: of B sixteen rows (16 lanes) by 64 or 128 neighbouring bytes at a time (4 lanes), of A likewise, from L2.
// The waves take the steps in turn, so that a workgroup reads runs of 8 * 64 values of a row.
template <int DT>
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
    const int row_b = n0 + l16 < p.N ? n0 + l16 : p.N - 1;            // (sums of rows that do not exist are not stored)
    const bool live_a = l16 < p.M;
    const T* const b = static_cast<const T*>(p.b) + row_b * p.ldb;
    const T* const a = static_cast<const T*>(p.a) + (live_a ? l16 : 0) * p.lda;

    Raw<DT> rb[AHEAD][2], ra[AHEAD][2];
    auto load = [&](int s, Raw<DT> (&to_b)[2], Raw<DT> (&to_a)[2]) {
#pragma unroll
        for (int kk = 0; kk < 2; ++kk) {
            const int k = s * STEP + 32 * kk, have = p.K - k;
            load_raw<DT>(to_b[kk], b + k, grp, have, p.vec_b);
            if (live_a) load_raw<DT>(to_a[kk], a + k, grp, have, p.vec_a);
        }
    };
    auto sums = [&](auto mode) {
        constexpr int MODE = decltype(mode)::value;
        f32x4 c[2] = {f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}};
#pragma unroll
        for (int i = 0; i < AHEAD; ++i)
            if (s0 + wave + i * WAVES < s1) load(s0 + wave + i * WAVES, rb[i], ra[i]);
        for (int s = s0 + wave; s < s1; s += AHEAD * WAVES) {
#pragma unroll
            for (int i = 0; i < AHEAD; ++i) {
                if (s + i * WAVES < s1) {
#pragma unroll
                    for (int kk = 0; kk < 2; ++kk) {
                        Fragment<DT> fb, fa;
                        cut<DT, MODE != ALL_PRODUCTS>(rb[i][kk], fb);
                        cut<DT, MODE != ALL_PRODUCTS>(ra[i][kk], fa);
                        c[kk] = multiply_parts<DT, MODE>(fb, fa, c[kk]);
                    }
                    if (s + (i + AHEAD) * WAVES < s1) load(s + (i + AHEAD) * WAVES, rb[i], ra[i]);
                }
            }
        }
        return c[0] + c[1];
    };
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
#pragma unroll
        for (int kk = 0; kk < 2; ++kk)
#pragma unroll
            for (auto& v : ra[i][kk].v) v = u32x4{0, 0, 0, 0};          // rows of A that do not exist
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
        finish_four<DT>(p.f, m, n, c);
    }
}

// ---- up to 64 rows: A through LDS, each wave its own columns of C -------------------------------------------------
// A step is 64 k.  A's rows are cut into parts once for the workgroup and lie in two LDS buffers in turn; the loads of A two steps
// ahead and of B one or two are kept in registers.  Along (not across): a wave takes sixteen rows of B.  Across: 64 columns of
// B, four neighbours a lane, so that the eight rows a lane reads are its operand's eight k for each of the four without
// an exchange between lanes.
template <int DT, int MT, bool ACROSS>
__global__ void __launch_bounds__(ACROSS ? 256 : 512, 2)
dense_rows_kernel(DenseProduct p, int join)
{
    typedef typename DenseType<DT>::type T;
    constexpr int WAVES = ACROSS ? 4 : 8, THREADS = 64 * WAVES, COLS = ACROSS ? 64 : 16, PARTS = DT == IOLB_F32 ? 3 : 1;
    constexpr int ROWS = 16 * MT, ITEMS = ROWS * 8, PER = (ITEMS + THREADS - 1) / THREADS;
    constexpr int NF = ACROSS ? 4 : 1;                                   // fragments of B side by side
    constexpr int UNITS = 2;                                             // loads of B: 32 k each
    __shared__ __align__(16) u32x4 rows[2][PARTS][ROWS * 8];
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int n0 = (blockIdx.x * WAVES + wave) * COLS;
    const int m0 = blockIdx.z * ROWS;
    const int steps_all = (p.K + STEP - 1) / STEP;
    const int s0 = (int)((long long)steps_all * blockIdx.y / p.splits), s1 = (int)((long long)steps_all * (blockIdx.y + 1) / p.splits);
    const T* const a = static_cast<const T*>(p.a);
    const T* const b = static_cast<const T*>(p.b);

    // ---- B in registers
    struct Unit { Raw<DT> along; u32x4 across[ACROSS ? 8 : 1]; };
    Unit ub[UNITS];
    const int along_row = n0 + l16 < p.N ? n0 + l16 : p.N - 1;
    const int first_col = n0 + 4 * l16;
    auto load_b = [&](int k, Unit& u) {                                  // k: of the unit's first
        if constexpr (!ACROSS) {
            load_raw<DT>(u.along, b + along_row * p.ldb + k, grp, p.K - k, p.vec_b);
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const int row = k + 8 * grp + i;
                const T* const from = b + (row < p.K ? row : p.K - 1) * p.ldb + first_col;
                u32x4 v = {0, 0, 0, 0};
                if (row < p.K) {
                    if (p.vec_b && first_col + 4 <= p.N) {
                        if constexpr (DT == IOLB_F32) {
                            v = *reinterpret_cast<const u32x4*>(from);
                        } else {
                            const u32x2 t = *reinterpret_cast<const u32x2*>(from);
                            v[0] = t[0]; v[1] = t[1];
                        }
                    } else if constexpr (DT == IOLB_F32) {
#pragma unroll
                        for (int j = 0; j < 4; ++j) v[j] = first_col + j < p.N ? __float_as_uint(from[j]) : 0u;
                    } else {
                        const unsigned short* const q = reinterpret_cast<const unsigned short*>(from);
#pragma unroll
                        for (int j = 0; j < 2; ++j) {
                            const unsigned lo = first_col + 2 * j < p.N ? q[2 * j] : 0u, hi = first_col + 2 * j + 1 < p.N ? q[2 * j + 1] : 0u;
                            v[j] = lo | hi << 16;
                        }
                    }
                }
                u.across[i] = v;
            }
        }
    };
    // ---- A: registers, then LDS
    Raw<DT> ra[PER];
    auto load_a = [&](int s) {
#pragma unroll
        for (int i = 0; i < PER; ++i) {
            const int item = tid + i * THREADS, row = m0 + (item >> 3), piece = item & 7, k = s * STEP + 32 * (piece >> 2);
            if (ITEMS % THREADS == 0 || item < ITEMS) {
                if (row < p.M) {
                    if constexpr (ACROSS && DT == IOLB_F32) {
                        // plain order of k: the eight rows of B that a lane reads are neighbours
                        const float* const from = a + row * p.lda + k + 8 * (piece & 3);
                        const int have = p.K - k - 8 * (piece & 3);
                        if (p.vec_a && have >= 8) {
                            ra[i].v[0] = *reinterpret_cast<const u32x4*>(from);
                            ra[i].v[1] = *reinterpret_cast<const u32x4*>(from + 4);
                        } else {
#pragma unroll
                            for (int j = 0; j < 8; ++j) ra[i].v[j / 4][j % 4] = j < have ? __float_as_uint(from[j]) : 0u;
                        }
                    } else {
                        load_raw<DT>(ra[i], a + row * p.lda + k, piece & 3, p.K - k, p.vec_a);
                    }
                } else {
#pragma unroll
                    for (auto& v : ra[i].v) v = u32x4{0, 0, 0, 0};
                }
            }
        }
    };

    f32x4 acc[MT][NF];
    auto sums = [&](auto mode) {
        constexpr int MODE = decltype(mode)::value;
        constexpr bool SAFE = MODE != ALL_PRODUCTS;
        auto store_a = [&](int buf) {
#pragma unroll
            for (int i = 0; i < PER; ++i) {
                const int item = tid + i * THREADS, row = item >> 3, piece = item & 7;
                if (ITEMS % THREADS == 0 || item < ITEMS) {
                    Fragment<DT> f;
                    cut<DT, SAFE>(ra[i], f);
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) rows[buf][q][row * 8 + place(row, piece)] = f.part[q];
                }
            }
        };
        if (s0 >= s1) return;
        load_a(s0);
#pragma unroll
        for (int u = 0; u < UNITS; ++u) load_b(s0 * STEP + 32 * u, ub[u]);
        store_a(s0 & 1);
        if (s0 + 1 < s1) load_a(s0 + 1);
        for (int s = s0; s < s1; ++s) {
            __syncthreads();
            if (s + 1 < s1) store_a((s + 1) & 1);
            if (s + 2 < s1) load_a(s + 2);
#pragma unroll
            for (int u = 0; u < UNITS; ++u) {
                Fragment<DT> fb[NF];
                if constexpr (!ACROSS) {
                    cut<DT, SAFE>(ub[u].along, fb[0]);
                } else {
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
                if (s + 1 < s1) load_b((s + 1) * STEP + 32 * u, ub[u]);
#pragma unroll
                for (int t = 0; t < MT; ++t) {
                    Fragment<DT> fa;
                    const int row = 16 * t + l16;
#pragma unroll
                    for (int q = 0; q < PARTS; ++q) fa.part[q] = rows[s & 1][q][row * 8 + place(row, 4 * u + grp)];
#pragma unroll
                    for (int j = 0; j < NF; ++j) acc[t][j] = multiply_parts<DT, MODE>(fb[j], fa, acc[t][j]);
                }
            }
        }
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
            __syncthreads();
            sums(std::integral_constant<int, LEADING_PRODUCT>{});
        }
    }
#pragma unroll
    for (int t = 0; t < MT; ++t) {
        const int m = m0 + 16 * t + l16;
#pragma unroll
        for (int i = 0; i < NF; ++i) {
            // across: column 4 (4 grp + i) + j of the wave's is value i of fragment j
            const int n = n0 + (ACROSS ? 16 * grp + 4 * i : 4 * grp);
            f32x4 c = acc[t][0];
            if constexpr (ACROSS) c = f32x4{acc[t][0][i], acc[t][1][i], acc[t][2][i], acc[t][3][i]};
            if (join) {
                keep_partial(p, blockIdx.y, m, n, c);
            } else {
                finish_four<DT>(p.f, m, n, c);
            }
        }
    }
}

constexpr int FEW = 16;                                // rows of the first kernel

template <int DT>
hipError_t launch(const DenseProduct& p, bool across, bool join, hipStream_t st)
{
    if (!across && p.M <= FEW) {
        dense_few_kernel<DT><<<dim3((p.N + 15) / 16, p.splits), 512, 0, st>>>(p, join);
        return hipGetLastError();
    }
    const int mt = p.M <= 16 ? 1 : p.M <= 32 ? 2 : 4;
    const unsigned cols = across ? 256 : 128;
    const dim3 grid((p.N + cols - 1) / cols, p.splits, (p.M + 16 * mt - 1) / (16 * mt));
    if (across) {
        if (mt == 1) dense_rows_kernel<DT, 1, true><<<grid, 256, 0, st>>>(p, join);
        else if (mt == 2) dense_rows_kernel<DT, 2, true><<<grid, 256, 0, st>>>(p, join);
        else dense_rows_kernel<DT, 4, true><<<grid, 256, 0, st>>>(p, join);
    } else {
        if (mt <= 2) dense_rows_kernel<DT, 2, false><<<grid, 512, 0, st>>>(p, join);
        else dense_rows_kernel<DT, 4, false><<<grid, 512, 0, st>>>(p, join);
    }
    return hipGetLastError();
}

}  // namespace

// Enough workgroups to have all compute units read, as long as each keeps eight steps (a wave of the first kernel: one).
DenseRowsPlan dense_rows_plan(int M, int N, int K, int dtype, bool across, bool checkpoint)
{
    const int steps = (K + STEP - 1) / STEP;
    const bool few = !across && M <= FEW;
    const int cols = few ? 16 : across ? 256 : 128;
    const long long blocks = (N + cols - 1) / cols;
    const int wanted = few ? 256 : 512;
    long long splits = (wanted + blocks - 1) / blocks;
    const long long most = few ? steps / 32 : steps / 8;
    if (blocks * 2 > wanted || splits > most) splits = blocks * 2 > wanted ? 1 : most;
    if (splits < 1) splits = 1;
    (void)dtype;
    return {(int)splits, splits > 1 || checkpoint};
}

hipError_t launch_dense_rows(const DenseProduct& p, bool across, bool join, int dtype, hipStream_t st)
{
    const hipError_t e = dtype == IOLB_F32 ? launch<IOLB_F32>(p, across, join, st)
                       : dtype == IOLB_F16 ? launch<IOLB_F16>(p, across, join, st) : launch<IOLB_BF16>(p, across, join, st);
    return e != hipSuccess || !join ? e : launch_dense_join(p, dtype, st);
}

}  // namespace iolb
