// C = A B^T of operands in microscaled 4-bit floating point on the scaled matrix instructions, with bias, activation and residual in the epilogue.
//
// The shape of the dense layers' product kernel (dense_tile.hip) with stages of 256 k: a row of a stage is again 128 bytes, eight pieces of 16, and a piece is
// a block of 32 codes, which is what a lane gives to a matrix instruction of 64 k.  A stage also takes the rows' eight scales, 8 bytes.  The lanes of half h
// multiply pieces 4 h + kk of a row, kk = 0 ... 3 (both operands alike: the order of k does not matter), so their four scales are one word of LDS, from
// which the instruction takes byte kk.
//
// Bound by the stage: 2.0 us for 256 x 256 x 256 on a compute unit, where the matrix instructions alone need 1.3 at the rate that the card's power leaves them.
// 8192^3 276 us (4.0 PFLOP/s), 8192 x 4096 -> 16384 bf16 with gelu 368 to 393 with packing x (18) and a quarter of a block's time (12 of 44 us) in prologue, gelu and stores.
// Workgroups that stay and take block after block were slower (394 -> 418).
#include "dense_math.h"
#include "kernels.h"
#include "lds_dma.h"
#include "mx4_math.h"

namespace iolb {

namespace {

constexpr int STEP = 256;                              // k of a stage
constexpr int ROW_BYTES = STEP / 2, ROW_SCALES = STEP / MX4_BLOCK;

constexpr int code_bytes(int bm, int bn) { return (bm + bn) * ROW_BYTES; }
constexpr int stage_bytes(int bm, int bn) { return code_bytes(bm, bn) + (bm + bn) * ROW_SCALES; }
// How many times a block's sums go through LDS.
constexpr int finish_passes(int bm, int bn) { return bm * bn * 4 > 2 * stage_bytes(bm, bn) ? 2 : 1; }

// Where piece `piece` of a 128-byte row lies.  LDS serves a 16-byte read in turns of sixteen lanes, which are not neighbours: 0-3, 12-15 and 20-27 together,
// then 4-11, 16-19 and 28-31 (found by counting conflicts).  Rows r and r + 1 lie in different halves of the banks; of either set the rows' upper
// bits, 1 to 3, are eight different ones.
__device__ __forceinline__ int mx4_place(int row, int piece) { return piece ^ (row >> 1 & 7); }

__device__ __forceinline__ void dma16(const uint8_t* base, unsigned offset, unsigned lds)
{
    lds_dma_load_16(reinterpret_cast<const float*>(base), offset, lds);
}

// W columns of row m: bias, residual, activation, the one rounding to the type.  PAST: past the caches.
template <int DT, int ACT, bool PAST, int W>
__device__ __forceinline__ void finish_row(const DenseFinish& f, int m, int n, const float (&bias)[W], float (&z)[W])
{
    typedef typename DenseType<DT>::type T;
    typedef typename Piece<T, W>::type TW;
    const int have = f.N - n;
    if (m >= f.M || have <= 0) return;
#pragma unroll
    for (int i = 0; i < W; ++i) z[i] += bias[i];
    if (f.residual && f.first) add_residual<DT>(f, m, n, z);
    if (!PAST || have < W) return store_columns<DT, ACT>(f, m, n, z);
#pragma unroll
    for (int i = 0; i < W; ++i) z[i] = activate<ACT>(z[i]);
    if (f.residual && !f.first) add_residual<DT>(f, m, n, z);
    TW t;
#pragma unroll
    for (int i = 0; i < W; ++i) t[i] = (T)z[i];
    __builtin_nontemporal_store(t, reinterpret_cast<TW*>(static_cast<T*>(f.y) + m * f.ldy + n));
}

template <int DT, int BM, int BN, int WM, int WN, bool PAST>
__global__ void __launch_bounds__(64 * WM * WN, 2)
mx4_tile_kernel(Mx4Product p, int tiles_m, int tiles_n)
{
    constexpr int WAVES = WM * WN, MI = BM / WM / 32, NI = BN / WN / 32;
    constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;           // loads of a wave and stage: 8 rows each
    constexpr int SCALE_LOADS = (BM + BN) / 32;                       // of a stage: 32 rows each
    constexpr unsigned STAGE = stage_bytes(BM, BN);
    static_assert(BM % 32 == 0 && BN % 32 == 0 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "whole loads");
    extern __shared__ u32x4 lds16[];
    char* const lds = reinterpret_cast<char*>(lds16);
    const unsigned lds0 = lds_byte_address(reinterpret_cast<const float*>(lds));
    const int tid = threadIdx.x, lane = tid & 63, l32 = lane & 31, hi = lane >> 5;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // Workgroups go to the eight XCDs in turn; each takes a run of neighbouring tiles, in bands of eight tile rows.
    int bm, bn;
    {
        const int n = gridDim.x, q = n >> 3, r = n & 7, xcd = blockIdx.x & 7;
        const int t = xcd * q + (xcd < r ? xcd : r) + ((int)blockIdx.x >> 3);
        const int band = t / (8 * tiles_n), in = t % (8 * tiles_n);
        const int high = tiles_m - 8 * band < 8 ? tiles_m - 8 * band : 8;
        bm = 8 * band + in % high;
        bn = in / high;
    }
    const int m0 = bm * BM, n0 = bn * BN;
    const int words = (p.K + MX4_WIDE - 1) / MX4_WIDE, steps_all = (words + 1) / 2;         // four scales to a word
    const int s0 = (int)((long long)steps_all * blockIdx.y / p.splits), s1 = (int)((long long)steps_all * (blockIdx.y + 1) / p.splits);

    // A load takes eight rows.  Those beyond the operand are read from its last ones: their sums are never stored.  Registers are short, so a load's rows
    // are in its base, and what a lane adds is one of two offsets, the second for the operand's last eight rows, which may be fewer.  (The empty
    // assembly lines keep the compiler from working such things out before the loop: their registers would spill.)
    const unsigned pitch = (unsigned)words * 64u, scale_pitch = (unsigned)words * 4u;
    const int rows_a = p.M - m0 < BM ? p.M - m0 : BM, rows_b = p.N - n0 < BN ? p.N - n0 : BN;
    const int last_a = (rows_a - 1) & ~7, last_b = (rows_b - 1) & ~7;
    // (a load's rows start at a multiple of 8, and are alike in the bits that `place` looks at for all loads of a wave)
    static_assert(WAVES % 4 == 0, "as said");
    const int from_piece = mx4_place(wave * 8 + (lane >> 3), lane & 7);
    const auto offset_in = [&](int rows) {
        const int r = lane >> 3;
        unsigned at = __umul24(r < rows ? r : rows - 1, pitch) + 16u * from_piece;     // (a pitch is at most 2^21)
        asm volatile("" : "+v"(at));
        return at;
    };
    const unsigned inside = offset_in(8), end_a = offset_in(rows_a - last_a), end_b = offset_in(rows_b - last_b);
    unsigned scale_off[(SCALE_LOADS + WAVES - 1) / WAVES];
#pragma unroll
    for (int i = 0; i < (SCALE_LOADS + WAVES - 1) / WAVES; ++i) {
        const int at = i * WAVES + wave;
        const bool of_a = at < BM / 32;
        const int r = (of_a ? at : at - BM / 32) * 32 + (lane >> 1), rows = of_a ? rows_a : rows_b;
        scale_off[i] = __umul24(r < rows ? r : rows - 1, scale_pitch);
        asm volatile("" : "+v"(scale_off[i]));
    }
    const uint8_t* const a0 = p.a + (long long)m0 * pitch;
    const uint8_t* const b0 = p.b + (long long)n0 * pitch;
    const uint8_t* const a0_scales = p.a_scales + (long long)m0 * scale_pitch;
    const uint8_t* const b0_scales = p.b_scales + (long long)n0 * scale_pitch;

    auto load = [&](int step, int buf) {
        const uint8_t* const a = a0 + (long long)step * ROW_BYTES;
        const uint8_t* const b = b0 + (long long)step * ROW_BYTES;
        const unsigned to = lds0 + buf * STAGE;
        // rows are whole words of scales: the last stage may have one of two
        if (2 * step + (from_piece >> 2) < words) {
#pragma unroll
            for (int i = 0; i < LA; ++i) {
                const int r = (i * WAVES + wave) * 8;
                int at = r < last_a ? r : last_a;
                asm volatile("" : "+s"(at));
                dma16(a + (size_t)((unsigned)at * pitch), at < last_a ? inside : end_a, to + (i * WAVES + wave) * 1024);
            }
#pragma unroll
            for (int i = 0; i < LB; ++i) {
                const int r = (i * WAVES + wave) * 8;
                int at = r < last_b ? r : last_b;
                asm volatile("" : "+s"(at));
                dma16(b + (size_t)((unsigned)at * pitch), at < last_b ? inside : end_b, to + BM * ROW_BYTES + (i * WAVES + wave) * 1024);
            }
        } else {
            // the end of the summed axis: pieces beyond it are zero on both sides
            unsigned at = tid;
            asm volatile("" : "+v"(at));
            at = buf * STAGE + at * 16;
#pragma unroll
            for (int i = 0; i < LA; ++i) *reinterpret_cast<u32x4*>(lds + at + i * WAVES * 1024) = u32x4{0, 0, 0, 0};
#pragma unroll
            for (int i = 0; i < LB; ++i) *reinterpret_cast<u32x4*>(lds + at + BM * ROW_BYTES + i * WAVES * 1024) = u32x4{0, 0, 0, 0};
        }
        // (a word beyond the end: the row's last one again, whose scales meet zeros, and NaN only in a row that has one)
        const unsigned word = 4u * (2 * step + (lane & 1) < words ? 2 * step + (lane & 1) : words - 1);
#pragma unroll
        for (int i = 0; i < (SCALE_LOADS + WAVES - 1) / WAVES; ++i) {
            const int at = i * WAVES + wave;
            if (at < SCALE_LOADS)
                lds_dma_load_4(reinterpret_cast<const float*>(at < BM / 32 ? a0_scales : b0_scales), scale_off[i] + word, to + code_bytes(BM, BN) + at * 256);
        }
    };

    f32x16 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j)
#pragma unroll
            for (int c = 0; c < 16; ++c) acc[i][j][c] = 0.f;

    // A stage is 4 MI groups of NI matrix instructions: quarter kk, 32 rows i of A.  The order is written out and held: after each group the reads
    // of the operands of a later one are issued, A into a ring of four fragments, AHEAD groups ahead, B a quarter ahead.  The one barrier of a stage
    // stands before its last groups, when all of it has been read: the next stage has arrived then, its first reads go out behind the last groups, and
    // the buffer is free for the stage after it.
    constexpr int GROUPS = 4 * MI, RING = 4, AHEAD = MI == 1 ? 2 : 3, LAST = MI == 4 ? 3 : MI;
    static_assert(LAST <= AHEAD && 2 * MI + NI <= GROUPS - LAST, "a stage is read before its barrier");
    u32x4 fa[RING], fb[2][NI];
    unsigned sa[MI], sb[NI], next_sa[MI], next_sb[NI];
    // fragments: row l32 of 32, piece 4 hi + kk; the rest is the same for all lanes
    const int frag_a = (wm * (BM / WM) + l32) * ROW_BYTES + 16 * mx4_place(l32, 4 * hi);
    const int frag_b = (BM + wn * (BN / WN) + l32) * ROW_BYTES + 16 * mx4_place(l32, 4 * hi);
    const int frag_sa = code_bytes(BM, BN) + (wm * (BM / WM) + l32) * ROW_SCALES + 4 * hi;
    const int frag_sb = code_bytes(BM, BN) + (BM + wn * (BN / WN) + l32) * ROW_SCALES + 4 * hi;
    auto read_a = [&](const char* at, int g) { fa[g % RING] = *reinterpret_cast<const u32x4*>(at + (frag_a ^ 16 * (g / MI)) + g % MI * 32 * ROW_BYTES); };
    auto read_b = [&](const char* at, int kk, int j) { fb[kk % 2][j] = *reinterpret_cast<const u32x4*>(at + (frag_b ^ 16 * kk) + j * 32 * ROW_BYTES); };
    auto read_scales = [&](const char* at, unsigned (&a)[MI], unsigned (&b)[NI]) {
#pragma unroll
        for (int i = 0; i < MI; ++i) a[i] = *reinterpret_cast<const unsigned*>(at + frag_sa + i * 32 * ROW_SCALES);
#pragma unroll
        for (int j = 0; j < NI; ++j) b[j] = *reinterpret_cast<const unsigned*>(at + frag_sb + j * 32 * ROW_SCALES);
    };
    if (s1 > s0) {
        load(s0, 0);
        lds_dma_wait_all();
        __syncthreads();
        if (s1 - s0 > 1) load(s0 + 1, 1);
        read_scales(lds, sa, sb);
#pragma unroll
        for (int j = 0; j < NI; ++j) read_b(lds, 0, j);
#pragma unroll
        for (int g = 0; g < AHEAD; ++g) read_a(lds, g);
    }
    for (int t = s0; t < s1; ++t) {
        const char* const at = lds + (t - s0 & 1) * STAGE;
        const char* const next = lds + (~(t - s0) & 1) * STAGE;     // (after the last stage: read, not used)
        static_range<0, GROUPS>([&](auto group) {
            constexpr int g = decltype(group)::value, kk = g / MI, i = g % MI;
            if constexpr (g == GROUPS - LAST) {
                lds_dma_wait_all();
                __syncthreads();
                if (t + 2 < s1) load(t + 2, t - s0 & 1);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[i][j] = mx4_multiply_32<kk>(fb[kk % 2][j], sb[j], fa[g % RING], sa[i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
            if constexpr (kk < 3 && i < NI) {
#pragma unroll
                for (int j = i; j < NI; j += MI) read_b(at, kk + 1, j);
            }
            if constexpr (g + AHEAD < GROUPS) read_a(at, g + AHEAD);
            if constexpr (g == GROUPS - LAST) {
                read_scales(next, next_sa, next_sb);
#pragma unroll
                for (int j = 0; j < NI; ++j) read_b(next, 0, j);
            }
            if constexpr (g >= GROUPS - LAST) {
                constexpr int done = g - (GROUPS - LAST);                   // reads of A's next fragments: evenly over the last groups
#pragma unroll
                for (int n = AHEAD * done / LAST; n < AHEAD * (done + 1) / LAST; ++n) read_a(next, n);
            }
        });
#pragma unroll
        for (int i = 0; i < MI; ++i) sa[i] = next_sa[i];
#pragma unroll
        for (int j = 0; j < NI; ++j) sb[j] = next_sb[j];
    }

    // a lane's sums: row l32 of 32, columns 8 q + 4 hi + 0 ... 3 of 32 for q = 0 ... 3
    const auto four = [&](int i, int j, int q) { return f32x4{acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]}; };
    if (p.splits > 1) {
        const int mw = m0 + wm * (BM / WM) + l32, nw = n0 + wn * (BN / WN) + 4 * hi;
        const long long ld = (p.N + 3) / 4 * 4;
        float* const out = p.partial + (long long)blockIdx.y * p.M * ld;
#pragma unroll
        for (int i = 0; i < MI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int m = mw + i * 32, n = nw + j * 32 + q * 8;
                    if (m < p.M && n < p.N) *reinterpret_cast<f32x4*>(out + m * ld + n) = four(i, j, q);
                }
        return;
    }

    // The sums go through LDS, as many rows at a time as fit, so that a thread finishes 16 bytes of a row and a wave's loads and stores are whole
    // rows.  16-byte piece c of row r lies at c ^ (r & 15).
    constexpr int PASSES = finish_passes(BM, BN), PI = MI / PASSES, PASS_ROWS = WM * PI * 32;
    constexpr int W = FINISH_COLUMNS<DT>, LANES = BN / W, AT_ONCE = 64 * WAVES / LANES;   // threads of a row, rows of an iteration
    static_assert(PASS_ROWS * BN * 4 <= 2 * (int)STAGE && PASS_ROWS % AT_ONCE == 0, "a pass fits the stages' buffers");
    f32x4* const sums = reinterpret_cast<f32x4*>(lds);
    const int n = n0 + (tid % LANES) * W;
    float bias[W];
    load_bias<DT>(p.f, n, bias);
#pragma unroll
    for (int pass = 0; pass < PASSES; ++pass) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < PI; ++i)
#pragma unroll
            for (int j = 0; j < NI; ++j)
#pragma unroll
                for (int q = 0; q < 4; ++q) {
                    const int r = (wm * PI + i) * 32 + l32, c = wn * (BN / WN / 4) + j * 8 + 2 * q + hi;
                    sums[r * (BN / 4) + (c ^ (r & 15))] = four(pass * PI + i, j, q);
                }
        __syncthreads();
        by_activation(p.f.act, [&](auto act) __attribute__((always_inline)) {
#pragma unroll 1
            for (int r = tid / LANES; r < PASS_ROWS; r += AT_ONCE) {
                float z[W];
#pragma unroll
                for (int h = 0; h < W / 4; ++h) {
                    const f32x4 part = sums[r * (BN / 4) + ((W / 4 * (tid % LANES) + h) ^ (r & 15))];
#pragma unroll
                    for (int i = 0; i < 4; ++i) z[4 * h + i] = part[i];
                }
                const int m = m0 + r / (PI * 32) * (BM / WM) + pass * PI * 32 + r % (PI * 32);
                finish_row<DT, decltype(act)::value, PAST>(p.f, m, n, bias, z);
            }
        });
    }
}

template <int DT, int BM, int BN, int WM, int WN>
hipError_t launch(const Mx4Product& p, hipStream_t st)
{
    const bool past = past_caches((double)p.M * p.N * sizeof(typename DenseType<DT>::type));
    const auto kernel = past ? mx4_tile_kernel<DT, BM, BN, WM, WN, true> : mx4_tile_kernel<DT, BM, BN, WM, WN, false>;
    const hipError_t e = allow_large_lds(reinterpret_cast<const void*>(kernel));
    if (e != hipSuccess) return e;
    const int tm = (p.M + BM - 1) / BM, tn = (p.N + BN - 1) / BN;
    kernel<<<dim3(tm * tn, p.splits), 64 * WM * WN, 2 * stage_bytes(BM, BN), st>>>(p, tm, tn);
    return hipGetLastError();
}

template <int DT>
hipError_t launch_tile(const Mx4Product& p, int tile, hipStream_t st)
{
    switch (tile) {
    case DENSE_TILE_256: return launch<DT, 256, 256, 2, 4>(p, st);
    case DENSE_TILE_128: return launch<DT, 128, 128, 2, 2>(p, st);
    case DENSE_TILE_64x128: return launch<DT, 64, 128, 1, 4>(p, st);
    default: return launch<DT, 64, 64, 2, 2>(p, st);
    }
}

}  // namespace

// Block and number of workgroups that share K: the least modelled time, ns.  A stage of 256 k takes a workgroup `alone` while it has a compute unit to itself, and
// `each` of the unit's time among several; `end` is what a block's epilogue takes of it.  Sharing K costs a second launch and the partial sums' way through
// memory.  Fitted to a sweep of 22 shapes, 17 <= M <= 4096, 64 <= N <= 16384, 512 <= K <= 25088.  Examples (us, 256 x 256 / 128 x 128 / 64 x 128 / 64 x 64, each
// with its best share of K): 64 x 4096 x 4096 15.4 / 11.2 / 10.5 / 9.2, 64 x 25088 -> 4096 25.4 / 19.7 / 18.6 / 18.0, 2048 x 2048 x 2048 21.6 / 11.8 / 11.5 / 13.0,
// 700 x 5000 -> 9000 40 / 29 / 42 / 43, 4096 x 4096 x 4096 43 / 50 / 62 / 75.
DenseTilePlan mx4_tile_plan(int M, int N, int K)
{
    static const struct { int m, n, alone, each, end; } blocks[DENSE_TILES] = {{256, 256, 1390, 2050, 3300}, {128, 128, 600, 700, 1800}, {64, 128, 420, 430, 900}, {64, 64, 320, 265, 500}};
    static const int shares[] = {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64};
    const long long steps = ((long long)K + STEP - 1) / STEP;
    DenseTilePlan plan{DENSE_TILE_256, 1};
    double least = -1;
    for (int b = 0; b < DENSE_TILES; ++b) {
        const auto& k = blocks[b];
        const long long tiles = (((long long)M + k.m - 1) / k.m) * (((long long)N + k.n - 1) / k.n);
        for (const int s : shares) {
            if (s > 1 && s > steps) break;
            // (the largest block has a unit to itself: its rounds are whole ones)
            double load = (double)tiles * s / 256;
            if (b == DENSE_TILE_256 && load > 1) load = (double)((tiles * s + 255) / 256);
            const double stage = k.each * load > k.alone ? k.each * load : k.alone;
            double ns = stage * ((steps + s - 1) / s) + k.end * (load > 1 ? load : 1);
            if (s > 1) ns += 2500 + 0.48e-3 * s * M * N * 4;
            if (least < 0 || ns < least) { least = ns; plan = {b, s}; }
        }
    }
    return plan;
}

hipError_t launch_mx4_tile(const Mx4Product& p, int tile, int dtype, hipStream_t st)
{
    const hipError_t e = dtype == IOLB_F32 ? launch_tile<IOLB_F32>(p, tile, st) : dtype == IOLB_F16 ? launch_tile<IOLB_F16>(p, tile, st) : launch_tile<IOLB_BF16>(p, tile, st);
    if (e != hipSuccess || p.splits == 1) return e;
    DenseProduct join{};
    join.M = p.M; join.N = p.N; join.K = p.K;
    join.splits = p.splits;
    join.partial = p.partial;
    join.f = p.f;
    return launch_dense_join(join, dtype, st);
}

}  // namespace iolb
