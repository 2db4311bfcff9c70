// C = A B^T on the 16-bit matrix cores, both operands contiguous along the summed axis, with bias, activation, residual and
// 8-bit checkpoint in the epilogue.
//
// A workgroup takes BM x BN sums.  Stages of 64 k go to LDS by LDS-direct loads (16 bytes a lane), two buffers: stage t + 1 is on its
// way while stage t is multiplied.  A row of a stage is 128 bytes, eight pieces of 16; piece c of row r lies in place
// c ^ (r & 7), so that the sixteen rows a fragment read touches fall on different banks.  The LDS end of such a load is fixed by
// the lane, so it is the address in memory that is exchanged.  Products are taken with B as the first operand: a lane then holds
// four neighbouring columns of one row.
//
// Measured: 8192 x 16384 -> 4096 fp16 896-922 us (1190-1230 TFLOP/s), 8192 x 4096 -> 16384 bf16 855-925, with gelu 911, 8192 x 4096 -> 8192 bf16 410-445
// (1240-1340 TFLOP/s); products of the vendor's library, in turn on the same card once that has run for some tenths of a second, 700, 692 and 342 (1570-1650; in
// its first tens of milliseconds 8192 x 8192 x 8192 runs at 1235 in bf16 and 1390 in fp16).  So the matrix cores could do a quarter more, at this card's power too.
// Of that, loads account for 4 to 10% (with every stage read from the same addresses, all from L2); the rest has not
// been taken apart.  Small ones, 1023 x 1001 -> 777 fp16 13.3 us, wait for their chain of stages.
#include "dense_math.h"
#include "kernels.h"
#include "lds_dma.h"

namespace iolb {

namespace {

constexpr int STEP = 64;                               // k of a stage
constexpr int ROW_BYTES = 2 * STEP;

// Sums in two fp16 parts that may be too small for what the parts left out (dense_math.h) are taken again, up to one in 128 of a workgroup's by all of its
// waves; blocks with more are left to three bf16 parts.
template <int WAVES> struct Again { int m, n; float share[WAVES]; };
constexpr int again_most(int outputs) { return outputs / 128; }
constexpr int again_bytes(int outputs, int waves) { return 16 + again_most(outputs) * 4 * (2 + waves); }
template <int WAVES>
__device__ __forceinline__ float whole(const Again<WAVES>& again)
{
    float sum = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += again.share[w];
    return sum;
}

// How many times a block's sums go through LDS, and where the sums taken again are listed: behind them.
constexpr int stage_bytes(int bm, int bn) { return (bm + bn) * ROW_BYTES; }
constexpr int finish_passes(int bm, int bn) { return bm * bn * 4 > 2 * stage_bytes(bm, bn) ? 2 : 1; }
constexpr int again_at(int bm, int bn) { return bm * bn * 4 / finish_passes(bm, bn); }
constexpr int lds_bytes(int bm, int bn, int waves, bool halves)
{
    const int listed = halves ? again_at(bm, bn) + again_bytes(bm * bn, waves) : 0;
    return listed > 2 * stage_bytes(bm, bn) ? listed : 2 * stage_bytes(bm, bn);
}

__device__ __forceinline__ void dma16(const char* base, unsigned offset, unsigned lds)
{
    lds_dma_load_16(reinterpret_cast<const float*>(base), offset, lds);
}

template <bool F16, int DT, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN, 2)
dense_tile_kernel(DenseProduct p, int tiles_m, int tiles_n)
{
    if (not_wanted(p)) return;
    constexpr bool HALVES = F16 && DT == IOLB_F32;
    constexpr int WAVES = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
    constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;           // loads of a wave and stage: 8 rows each
    constexpr unsigned STAGE = stage_bytes(BM, BN);
    static_assert(NI % 2 == 0 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "blocks of 32 columns, whole loads");
    extern __shared__ u32x4 lds16[];
    char* const lds = reinterpret_cast<char*>(lds16);
    const unsigned lds0 = lds_byte_address(reinterpret_cast<const float*>(lds));
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // Workgroups go to the eight XCDs in turn; each XCD takes a run of neighbouring tiles, in bands of eight tile rows, so that
    // its L2 holds the operands of a compact patch.  (Bands of four and six rows are within 2%, of 16 and 32 slower.)
    int bm, bn;
    {
        const int n = gridDim.x, q = n >> 3, r = n & 7, xcd = blockIdx.x & 7;
        const int t = xcd * q + (xcd < r ? xcd : r) + ((int)blockIdx.x >> 3);
        const int band = t / (8 * tiles_n), in = t % (8 * tiles_n);
        const int high = tiles_m - 8 * band < 8 ? tiles_m - 8 * band : 8;
        bm = 8 * band + in % high;
        bn = in / high;
    }
    const int tile = bm * tiles_n + bn;
    if (!HALVES && p.left && p.splits == 1 && !p.uneven[0] && !p.left[tile]) return;
    const int m0 = bm * BM, n0 = bn * BN;
    const int steps_all = (p.K + STEP - 1) / STEP;
    const int s0 = (int)((long long)steps_all * blockIdx.y / p.splits), s1 = (int)((long long)steps_all * (blockIdx.y + 1) / p.splits);

    // Rows beyond the operand are read from its last row: their sums are never stored.
    unsigned a_off[LA], b_off[LB];
    const int from_piece = place(lane >> 3, lane & 7);           // (a load's rows start at a multiple of 8)
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int r = (i * WAVES + wave) * 8 + (lane >> 3), have = p.M - 1 - m0;
        a_off[i] = (unsigned)(2 * (r < have ? r : have)) * (unsigned)p.lda + 16u * from_piece;
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int r = (i * WAVES + wave) * 8 + (lane >> 3), have = p.N - 1 - n0;
        b_off[i] = (unsigned)(2 * (r < have ? r : have)) * (unsigned)p.ldb + 16u * from_piece;
    }
    const char* const a0 = static_cast<const char*>(p.a) + 2 * (m0 * p.lda);
    const char* const b0 = static_cast<const char*>(p.b) + 2 * (n0 * p.ldb);
    const int my_k = 8 * from_piece;                              // first k of the piece this lane fetches

    auto load = [&](int seg, int step, int buf) {
        const char* const a = a0 + 2 * (p.a_plane[seg] + (long long)step * STEP);
        const char* const b = b0 + 2 * (p.b_plane[seg] + (long long)step * STEP);
        const unsigned to = lds0 + buf * STAGE;
        if ((step + 1) * STEP <= p.K) {
#pragma unroll
            for (int i = 0; i < LA; ++i) dma16(a, a_off[i], to + (i * WAVES + wave) * 1024);
#pragma unroll
            for (int i = 0; i < LB; ++i) dma16(b, b_off[i], to + BM * ROW_BYTES + (i * WAVES + wave) * 1024);
        } else {
            // the end of the summed axis: pieces beyond it are zero on both sides
            if (step * STEP + my_k < p.K) {
#pragma unroll
                for (int i = 0; i < LA; ++i) dma16(a, a_off[i], to + (i * WAVES + wave) * 1024);
#pragma unroll
                for (int i = 0; i < LB; ++i) dma16(b, b_off[i], to + BM * ROW_BYTES + (i * WAVES + wave) * 1024);
            } else {
                char* const at = lds + buf * STAGE + wave * 1024 + lane * 16;
#pragma unroll
                for (int i = 0; i < LA; ++i) *reinterpret_cast<u32x4*>(at + i * WAVES * 1024) = u32x4{0, 0, 0, 0};
#pragma unroll
                for (int i = 0; i < LB; ++i) *reinterpret_cast<u32x4*>(at + BM * ROW_BYTES + i * WAVES * 1024) = u32x4{0, 0, 0, 0};
            }
        }
    };

    f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    const int rounds = s1 > s0 ? p.segments * (s1 - s0) : 0;
    const int clear_at = p.segments > 1 ? rounds - (s1 - s0) : -1;
    int seg = 0, step = s0;                            // of the stage that is loaded next
    auto load_next = [&](int buf) {
        load(seg, step, buf);
        if (++step == s1) { step = s0; ++seg; }
    };

    // A stage is 2 MI groups of NI matrix instructions: half kk (32 k), sixteen rows i of A.  The order is written out and held: after
    // each group the reads of the operands of a later one are issued, A into a ring of MI registers, `AHEAD` groups ahead, B a half
    // ahead, so that matrix instructions do not wait for LDS.  The one barrier of a stage stands before its last groups, when all
    // of it has been read: the next stage has arrived then, its first reads go out behind the last groups, and the buffer is free
    // for the stage after it.
    constexpr int GROUPS = 2 * MI, AHEAD = MI > 2 ? MI - 2 : 1, LAST = MI == 8 ? 3 : MI == 4 ? 2 : 1;
    static_assert(AHEAD < MI && LAST <= AHEAD && NI <= GROUPS - LAST, "a stage is read before its barrier");
    u32x4 fa[MI], fb[2][NI];
    // fragments: row l16 of sixteen, piece 4 kk + grp; the rest is the same for all lanes
    const int frag_a = (wm * (BM / WM) + l16) * ROW_BYTES + 16 * place(l16, grp);
    const int frag_b = (BM + wn * (BN / WN) + l16) * ROW_BYTES + 16 * place(l16, grp);
    auto read_a = [&](const char* at, int g) {
        fa[g % MI] = *reinterpret_cast<const u32x4*>(at + (frag_a ^ 64 * (g / MI)) + g % MI * 16 * ROW_BYTES);
    };
    auto read_b = [&](const char* at, int kk, int j) {
        fb[kk][j] = *reinterpret_cast<const u32x4*>(at + (frag_b ^ 64 * kk) + j * 16 * ROW_BYTES);
    };
    if (rounds) {
        load_next(0);
        lds_dma_wait_all();
        __syncthreads();
        if (rounds > 1) load_next(1);
#pragma unroll
        for (int j = 0; j < NI; ++j) read_b(lds, 0, j);
#pragma unroll
        for (int g = 0; g < AHEAD; ++g) read_a(lds, g);
    }
    for (int t = 0; t < rounds; ++t) {
        if (t == clear_at) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[i][j][c] = fabsf(acc[i][j][c]) < __builtin_inff() ? acc[i][j][c] : 0.f;
        }
        const char* const at = lds + (t & 1) * STAGE;
        const char* const next = lds + (~t & 1) * STAGE;      // (after the last stage: read, not used)
        static_range<0, GROUPS>([&](auto group) {
            constexpr int g = decltype(group)::value;
            if constexpr (g == GROUPS - LAST) {
                lds_dma_wait_all();
                __syncthreads();
                if (t + 2 < rounds) load_next(t & 1);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[g % MI][j] = multiply<F16>(fb[g / MI][j], fa[g % MI], acc[g % MI][j]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (g < NI) read_b(at, 1, g);
            if constexpr (g + AHEAD < GROUPS) read_a(at, g + AHEAD);
            if constexpr (g == GROUPS - LAST) {
#pragma unroll
                for (int j = 0; j < NI; ++j) read_b(next, 0, j);
            }
            if constexpr (g >= GROUPS - LAST) {
                constexpr int done = g - (GROUPS - LAST);                   // reads of A's next fragments: evenly over the last groups
#pragma unroll
                for (int i = AHEAD * done / LAST; i < AHEAD * (done + 1) / LAST; ++i) read_a(next, i);
            }
        });
    }

    if (p.splits > 1) {
        const int mw = m0 + wm * (BM / WM) + l16, nw = n0 + wn * (BN / WN) + 4 * grp;
        const long long ld = (p.N + 3) / 4 * 4;
        float* const out = p.partial + (long long)blockIdx.y * p.M * ld;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int m = mw + i * 16, n = nw + j * 16;
                if (m < p.M && n < p.N) *reinterpret_cast<f32x4*>(out + m * ld + n) = acc[i][j];
            }
        return;
    }

    int* const again_count = reinterpret_cast<int*>(lds + again_at(BM, BN));
    Again<WAVES>* const again = reinterpret_cast<Again<WAVES>*>(lds + again_at(BM, BN) + 16);
    int taken_again = 0;
    if constexpr (HALVES) {
        const int mw = m0 + wm * (BM / WM) + l16, nw = n0 + wn * (BN / WN) + 4 * grp;
        __syncthreads();
        if (tid == 0) *again_count = 0;
        __syncthreads();
        DenseScale scale_a[MI];
#pragma unroll
        for (int i = 0; i < MI; ++i) scale_a[i] = p.scales_a[mw + i * 16 < p.M ? mw + i * 16 : p.M - 1];
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            const int n = nw + j * 16;
            DenseScale scale_b[4];
#pragma unroll
            for (int c = 0; c < 4; ++c) scale_b[c] = p.scales_b[n + c < p.N ? n + c : p.N - 1];
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const int m = mw + i * 16;
#pragma unroll
                for (int c = 0; c < 4; ++c) {
                    if (fabsf(acc[i][j][c]) < least_sum(scale_a[i].lost, scale_b[c].lost) && m < p.M && n + c < p.N) {
                        const int at = atomicAdd(again_count, 1);
                        if (at < again_most(BM * BN)) { again[at].m = m; again[at].n = n + c; }
                    }
                    acc[i][j][c] = ldexpf(acc[i][j][c], scale_a[i].exponent + scale_b[c].exponent);
                }
            }
        }
        __syncthreads();
        taken_again = *again_count;
        const bool left = taken_again > again_most(BM * BN);
        if (tid == 0) {
            p.left[tile] = left;
            if (left) p.uneven[1] = 1;
        }
        if (left) return;
        for (int i = 0; i < taken_again; ++i) {
            const float share = share_again(p, again[i].m, again[i].n, wave, WAVES, lane);
            if (lane == 0) again[i].share[wave] = share;
        }
    }

    // The sums go through LDS, as many rows at a time as fit, so that a thread finishes 16 bytes of a row and a wave's loads
    // and stores are whole rows.  16-byte piece c of row r lies at c ^ (r & 15).
    constexpr int PASSES = finish_passes(BM, BN), PI = MI / PASSES, PASS_ROWS = WM * PI * 16;
    constexpr int W = FINISH_COLUMNS<DT>, LANES = BN / W, AT_ONCE = 64 * WAVES / LANES;   // threads of a row, rows of an iteration
    static_assert(PASS_ROWS * BN * 4 <= 2 * (int)STAGE && PASS_ROWS % AT_ONCE == 0, "a pass fits the stages' buffers");
    f32x4* const sums = reinterpret_cast<f32x4*>(lds);
    const int n = n0 + (tid % LANES) * W;
    float bias[W];
    load_bias<DT>(p.f, n, bias);
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        if (pass || rounds) __syncthreads();
#pragma unroll
        for (int i = 0; i < PI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int r = (wm * PI + i) * 16 + l16, c = wn * (BN / WN / 4) + j * 4 + grp;
                sums[r * (BN / 4) + (c ^ l16)] = acc[pass * PI + i][j];
            }
        __syncthreads();
        if (HALVES && taken_again) {
            for (int i = tid; i < taken_again; i += 64 * WAVES) {
                const int m = again[i].m - m0, nn = again[i].n - n0, in = m % (BM / WM), r = m / (BM / WM) * (PI * 16) + in % (PI * 16);
                if (in / (PI * 16) == pass) reinterpret_cast<float*>(&sums[r * (BN / 4) + (nn / 4 ^ (r & 15))])[nn & 3] = whole(again[i]);
            }
            __syncthreads();
        }
        by_activation(p.f.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll 1
            for (int r = tid / LANES; r < PASS_ROWS; r += AT_ONCE) {
                float z[W];
#pragma unroll
                for (int h = 0; h < W / 4; ++h) {
                    const f32x4 four = sums[r * (BN / 4) + ((W / 4 * (tid % LANES) + h) ^ (r & 15))];
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[4 * h + i] = four[i];
                }
                const int m = m0 + r / (PI * 16) * (BM / WM) + pass * PI * 16 + r % (PI * 16);
                finish_columns<DT, decltype(act)::value>(p.f, m, n, bias, z);
            }
        });
    }
}

// The sums of the workgroups that shared a tile's K, added in their order, and the epilogue.
template <int DT, bool HALVES = false>
__global__ void __launch_bounds__(256)
dense_join_kernel(DenseProduct p, int wide_log)
{
    if (not_wanted(p)) return;
    constexpr int MOST = again_most(256 * 8);
    __shared__ Again<4> again[HALVES ? MOST : 1];
    __shared__ int again_count;
    const int wide = 1 << wide_log, tx = threadIdx.x & (wide - 1), rows = 256 >> wide_log;
    const int n = (int)((blockIdx.x * (unsigned)wide + tx) * 8);
    const long long ld = (p.N + 3) / 4 * 4;
    by_activation(p.f.act, [&](auto act) __attribute__((always_inline)) {
        float bias[8];
        load_bias<DT>(p.f, n, bias);
        DenseScale scale_b[HALVES ? 8 : 1];
        if constexpr (HALVES) {
#pragma unroll
            for (int c = 0; c < 8; ++c) scale_b[c] = p.scales_b[n + c < p.N ? n + c : p.N - 1];
        }
        int pieces = p.splits;
        if (p.block_columns && n < p.N) {
            // the runs that meet the block of columns n is in (all eight are in one)
            const long long steps = (p.K + DENSE_ROWS_STEP - 1) / DENSE_ROWS_STEP, first = n / p.block_columns * steps;
            pieces = (int)((first + steps - 1) / p.per - first / p.per) + 1;
        }
        for (long long m = (long long)blockIdx.y * rows + (threadIdx.x >> wide_log); m - (threadIdx.x >> wide_log) < p.M; m += (long long)gridDim.y * rows) {
            const long long block = (m - (threadIdx.x >> wide_log)) / rows * gridDim.x + blockIdx.x;
            if (DT == IOLB_F32 && !HALVES && p.left && !p.uneven[0] && !p.left[block]) continue;
            DenseScale scale_a{};
            if constexpr (HALVES) scale_a = p.scales_a[m < p.M ? m : 0];
            float z[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
            if (m < p.M && n < p.N) {
                const float* from = p.partial + m * ld + n;
                const bool both = n + 4 < p.N;
#pragma unroll 4
                for (int s = 0; s < pieces; ++s, from += p.M * ld) {
                    const f32x4 lo = *reinterpret_cast<const f32x4*>(from), hi = both ? *reinterpret_cast<const f32x4*>(from + 4) : f32x4{0, 0, 0, 0};
#pragma unroll
                    for (int c = 0; c < 4; ++c) { z[c] += lo[c]; z[4 + c] += hi[c]; }
                }
            }
            if constexpr (HALVES) {
                unsigned small = 0;
#pragma unroll
                for (int c = 0; c < 8; ++c) {
                    small |= m < p.M && n + c < p.N && fabsf(z[c]) < least_sum(scale_a.lost, scale_b[c].lost) ? 1u << c : 0u;
                    z[c] = ldexpf(z[c], scale_a.exponent + scale_b[c].exponent);
                }
                const bool any = __syncthreads_or(small != 0);
                int at = 0, count = 0;
                if (any) {
                    if (threadIdx.x == 0) again_count = 0;
                    __syncthreads();
                    if (small) {
                        at = atomicAdd(&again_count, __builtin_popcount(small));
                        int to = at;
#pragma unroll
                        for (int c = 0; c < 8; ++c)
                            if (small >> c & 1 && to < MOST) { again[to].m = (int)m; again[to].n = n + c; ++to; }
                    }
                    __syncthreads();
                    count = again_count;
                    for (int i = 0; i < count && count <= MOST; ++i) {
                        const float share = share_again(p, again[i].m, again[i].n, threadIdx.x >> 6, 4, threadIdx.x & 63);
                        if ((threadIdx.x & 63) == 0) again[i].share[threadIdx.x >> 6] = share;
                    }
                    __syncthreads();
                }
                if (threadIdx.x == 0) {
                    p.left[block] = count > MOST;
                    if (count > MOST) p.uneven[1] = 1;
                }
                if (count > MOST) continue;
#pragma unroll
                for (int c = 0; c < 8; ++c)
                    if (small >> c & 1) z[c] = whole(again[at++]);
            }
            finish_columns<DT, decltype(act)::value>(p.f, (int)(m < p.M ? m : p.M), n, bias, z);
        }
    });
}

template <bool F16, int DT, int BM, int BN, int WM, int WN>
hipError_t launch(const DenseProduct& p, hipStream_t st)
{
    const auto kernel = dense_tile_kernel<F16, DT, BM, BN, WM, WN>;
    const hipError_t e = allow_large_lds(reinterpret_cast<const void*>(kernel));
    if (e != hipSuccess) return e;
    const int tm = (p.M + BM - 1) / BM, tn = (p.N + BN - 1) / BN;
    if ((long long)tm * tn > 0x7fffffffLL) return hipErrorInvalidValue;
    kernel<<<dim3(tm * tn, p.splits), 64 * WM * WN, lds_bytes(BM, BN, WM * WN, F16 && DT == IOLB_F32), st>>>(p, tm, tn);
    return hipGetLastError();
}

template <bool F16, int DT>
hipError_t launch_tile(const DenseProduct& p, int tile, hipStream_t st)
{
    switch (tile) {
    case DENSE_TILE_256: return launch<F16, DT, 256, 256, 2, 4>(p, st);
    case DENSE_TILE_128: return launch<F16, DT, 128, 128, 2, 2>(p, st);
    case DENSE_TILE_64x128: return launch<F16, DT, 64, 128, 1, 4>(p, st);
    default: return launch<F16, DT, 64, 64, 2, 2>(p, st);
    }
}

struct Block { int m, n, alone, each; };
constexpr Block blocks[DENSE_TILES] = {{256, 256, 1450, 1550}, {128, 128, 720, 510}, {64, 128, 570, 350}, {64, 64, 490, 190}};

}  // namespace

// Block and number of workgroups that share K: the least modelled time.  A stage takes a workgroup `alone` ns while it has a compute unit
// to itself (bound by its chain of loads, reads and products) and `each` ns of the unit's time among several.  Sharing K costs a
// second launch and the partial sums' way through memory.  Fitted to a sweep of 20 shapes, 64 <= M, N <= 25088, 64 <= K <= 16384; of these
// the model's pick is within 8% of the best measured one.  Examples (us, bf16, 256 x 256 / 128 x 128 / 64 x 128 / 64 x 64, each with its
// best share of K): 128 x 4096 x 4096 24.9 / 19.0 / 17.7 / 17.4, 1024 x 1024 x 1024 26.7 / 14.6 / 11.4 / 9.7, 2048 x 4096 x 4096 79 / 69 / 94 / 100.
// Measured and not taken: three and four buffers for the small blocks, two workgroups of 128 x 128 with four (more stages on their way, fewer
// workgroups on a compute unit): 2048 x 2048 x 2048 27.0 -> 28.2, 1024 x 4096 x 1024 15.8 -> 16.7, 4096 x 4096 x 256 20.1 -> 28; a third buffer
// of A for the largest block (all of the LDS): 8192 x 16384 x 4096 862 -> 911; a higher wave priority around the products: 2 to 3% slower.
DenseTilePlan dense_tile_plan(int M, int N, int K, int segments)
{
    static const int shares[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
    const long long steps = (K + STEP - 1) / STEP;
    DenseTilePlan plan{DENSE_TILE_256, 1};
    long long least = -1;
    for (int b = 0; b < DENSE_TILES; ++b) {
        const Block& k = blocks[b];
        const long long tiles = (long long)((M + k.m - 1) / k.m) * ((N + k.n - 1) / k.n);
        for (const int s : shares) {
            if (s > 1 && s > steps) break;
            const long long on_unit = (tiles * s + 255) / 256, stage = k.each * on_unit > k.alone ? k.each * on_unit : k.alone;
            long long ns = stage * ((steps + s - 1) / s) * segments;
            if (s > 1) ns += 3000 + 80 * s + (long long)(8.0 * s * M * N / 5500);
            if (least < 0 || ns < least) { least = ns; plan = {b, s}; }
        }
    }
    return plan;
}

bool dense_tile_launchable(const DenseTilePlan& plan, int M, int N)
{
    const Block& b = blocks[plan.tile];
    const long long tiles = ((long long)M + b.m - 1) / b.m * (((long long)N + b.n - 1) / b.n);
    return tiles * (plan.tile == DENSE_TILE_256 ? 512 : 256) <= 0xffffffffLL;
}

static int join_wide_log(int N)
{
    int wide_log = 2;                               // threads of a row: whole blocks of 32 columns
    while (wide_log < 8 && (8LL << wide_log) < N) ++wide_log;
    return wide_log;
}

long long dense_finish_blocks(const DenseTilePlan& plan, int M, int N)
{
    const int wide_log = join_wide_log(N);
    const long long m = plan.splits == 1 ? blocks[plan.tile].m : 256 >> wide_log, n = plan.splits == 1 ? blocks[plan.tile].n : 8LL << wide_log;
    return ((M + m - 1) / m) * ((N + n - 1) / n);
}

hipError_t launch_dense_product(const DenseProduct& p, int tile, int dtype, hipStream_t st)
{
    hipError_t e = dtype == IOLB_F32 ? (p.scales_a ? launch_tile<true, IOLB_F32>(p, tile, st) : launch_tile<false, IOLB_F32>(p, tile, st))
                 : dtype == IOLB_F16 ? launch_tile<true, IOLB_F16>(p, tile, st) : launch_tile<false, IOLB_BF16>(p, tile, st);
    return e != hipSuccess || p.splits == 1 ? e : launch_dense_join(p, dtype, st);
}

hipError_t launch_dense_join(const DenseProduct& p, int dtype, hipStream_t st)
{
    const int wide_log = join_wide_log(p.N);
    const int rows = 256 >> wide_log;
    const long long gy = ((long long)p.M + rows - 1) / rows;
    const dim3 grid((unsigned)((p.N + (8LL << wide_log) - 1) / (8LL << wide_log)), (unsigned)(gy < 65535 ? gy : 65535));
    if (dtype == IOLB_F32 && p.scales_a) dense_join_kernel<IOLB_F32, true><<<grid, 256, 0, st>>>(p, wide_log);
    else if (dtype == IOLB_F32) dense_join_kernel<IOLB_F32><<<grid, 256, 0, st>>>(p, wide_log);
    else if (dtype == IOLB_F16) dense_join_kernel<IOLB_F16><<<grid, 256, 0, st>>>(p, wide_log);
    else dense_join_kernel<IOLB_BF16><<<grid, 256, 0, st>>>(p, wide_log);
    return hipGetLastError();
}

}  // namespace iolb
