// C = A B^T of operands in microscaled 4-bit floating point on the scaled matrix instructions, with bias, activation and residual in the epilogue.
//
// The shape of the dense layers' product kernel (dense_tile.hip) with stages of 256 k: a row of a stage is again 128 bytes, eight pieces of 16, and a piece is
// a block of 32 codes, which is what a lane gives to a matrix instruction of 128 k.  A stage also takes the rows' eight scales, 8 bytes.  Lane group g
// multiplies pieces 2 g and 2 g + 1 of a row, one in each half of the stage (both operands alike: the order of k does not matter), so its two scales
// are neighbours, and one 16-bit read of LDS gives the instruction both, each by its byte
// number.  (32 bits read at odd multiples of two bytes, of which the upper half is not looked at, take LDS 77 cycles an instruction.)
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

__device__ __forceinline__ void dma16(const uint8_t* base, unsigned offset, unsigned lds)
{
    lds_dma_load_16(reinterpret_cast<const float*>(base), offset, lds);
}

template <int DT, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN, 2)
mx4_tile_kernel(Mx4Product p, int tiles_m, int tiles_n)
{
    constexpr int WAVES = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
    constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;           // loads of a wave and stage: 8 rows each
    constexpr int SCALE_LOADS = (BM + BN) / 32;                       // of a stage: 32 rows each
    constexpr unsigned STAGE = stage_bytes(BM, BN);
    static_assert(BM % 32 == 0 && BN % 32 == 0 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "whole loads");
    extern __shared__ u32x4 lds16[];
    char* const lds = reinterpret_cast<char*>(lds16);
    const unsigned lds0 = lds_byte_address(reinterpret_cast<const float*>(lds));
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
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
    // (a load's rows start at a multiple of 8; piece 2 g + kk lies where piece 4 kk + g would: what neighbouring lane groups read together are neighbours)
    const int placed = place(lane >> 3, lane & 7), from_piece = 2 * (placed & 3) + (placed >> 2);
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

    f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    // A stage is 2 MI groups of NI matrix instructions: half kk, sixteen rows i of A.  The order is written out and held: after each group the reads
    // of the operands of a later one are issued, A into a ring of RING fragments, AHEAD groups ahead, B a half ahead.  The one barrier of a stage
    // stands before its last groups, when all of it has been read: the next stage has arrived then, its first reads go out behind the last groups, and
    // the buffer is free for the stage after it.
    constexpr int GROUPS = 2 * MI, RING = MI < 4 ? MI : 4, AHEAD = MI == 8 ? 3 : MI == 4 ? 2 : 1, LAST = AHEAD;
    static_assert(GROUPS % RING == 0 && AHEAD < RING && LAST < MI && NI <= GROUPS - LAST, "a stage is read before its barrier");
    u32x4 fa[RING], fb[2][NI];
    unsigned sa[MI], sb[NI], next_sb[NI];
    // fragments: row l16 of sixteen, piece 2 grp + kk; the rest is the same for all lanes
    const int frag_a = (wm * (BM / WM) + l16) * ROW_BYTES + 16 * place(l16, grp);
    const int frag_b = (BM + wn * (BN / WN) + l16) * ROW_BYTES + 16 * place(l16, grp);
    const int frag_sa = code_bytes(BM, BN) + (wm * (BM / WM) + l16) * ROW_SCALES + 2 * grp;
    const int frag_sb = code_bytes(BM, BN) + (BM + wn * (BN / WN) + l16) * ROW_SCALES + 2 * grp;
    auto read_a = [&](const char* at, int g) { fa[g % RING] = *reinterpret_cast<const u32x4*>(at + (frag_a ^ 64 * (g / MI)) + g % MI * 16 * ROW_BYTES); };
    auto read_b = [&](const char* at, int kk, int j) { fb[kk][j] = *reinterpret_cast<const u32x4*>(at + (frag_b ^ 64 * kk) + j * 16 * ROW_BYTES); };
    auto read_sa = [&](const char* at, int i) { sa[i] = *reinterpret_cast<const unsigned short*>(at + frag_sa + i * 16 * ROW_SCALES); };
    auto scale_b = [&](const char* at, int j) -> unsigned { return *reinterpret_cast<const unsigned short*>(at + frag_sb + j * 16 * ROW_SCALES); };
    if (s1 > s0) {
        load(s0, 0);
        lds_dma_wait_all();
        __syncthreads();
        if (s1 - s0 > 1) load(s0 + 1, 1);
#pragma unroll
        for (int i = 0; i < MI - LAST; ++i) read_sa(lds, i);
#pragma unroll
        for (int j = 0; j < NI; ++j) {
            sb[j] = scale_b(lds, j);
            read_b(lds, 0, j);
        }
#pragma unroll
        for (int g = 0; g < AHEAD; ++g) read_a(lds, g);
    }
    for (int t = s0; t < s1; ++t) {
        const char* const at = lds + (t - s0 & 1) * STAGE;
        const char* const next = lds + (~(t - s0) & 1) * STAGE;     // (after the last stage: read, not used)
        static_range<0, GROUPS>([&](auto group) {
            constexpr int g = decltype(group)::value;
            if constexpr (g == GROUPS - LAST) {
                lds_dma_wait_all();
                __syncthreads();
                if (t + 2 < s1) load(t + 2, t - s0 & 1);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < NI; ++j) acc[g % MI][j] = mx4_multiply<g / MI, g / MI>(fb[g / MI][j], sb[j], fa[g % RING], sa[g % MI], acc[g % MI][j]);
            __builtin_amdgcn_sched_barrier(0);
            // (the scales of the last rows of A: the others were read with the stage's first fragments)
            if constexpr (g == 0) {
#pragma unroll
                for (int i = MI - LAST; i < MI; ++i) read_sa(at, i);
            }
            if constexpr (g < NI) read_b(at, 1, g);
            if constexpr (g + AHEAD < GROUPS) read_a(at, g + AHEAD);
            if constexpr (g == GROUPS - LAST) {
#pragma unroll
                for (int i = 0; i < MI - LAST; ++i) read_sa(next, i);
#pragma unroll
                for (int j = 0; j < NI; ++j) {
                    next_sb[j] = scale_b(next, j);
                    read_b(next, 0, j);
                }
            }
            if constexpr (g >= GROUPS - LAST) {
                constexpr int done = g - (GROUPS - LAST);                   // reads of A's next fragments: evenly over the last groups
#pragma unroll
                for (int i = AHEAD * done / LAST; i < AHEAD * (done + 1) / LAST; ++i) read_a(next, i);
            }
        });
#pragma unroll
        for (int j = 0; j < NI; ++j) sb[j] = next_sb[j];
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

    // The sums go through LDS, as many rows at a time as fit, so that a thread finishes 16 bytes of a row and a wave's loads and stores are whole
    // rows.  16-byte piece c of row r lies at c ^ (r & 15).
    constexpr int PASSES = finish_passes(BM, BN), PI = MI / PASSES, PASS_ROWS = WM * PI * 16;
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
            for (int j = 0; j < NI; ++j) {
                const int r = (wm * PI + i) * 16 + l16, c = wn * (BN / WN / 4) + j * 4 + grp;
                sums[r * (BN / 4) + (c ^ l16)] = acc[pass * PI + i][j];
            }
        __syncthreads();
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

template <int DT, int BM, int BN, int WM, int WN>
hipError_t launch(const Mx4Product& p, hipStream_t st)
{
    const auto kernel = mx4_tile_kernel<DT, BM, BN, WM, WN>;
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

// A stage has as many bytes and matrix cycles as one of 64 k of 16-bit operands.
DenseTilePlan mx4_tile_plan(int M, int N, int K) { return dense_tile_plan(M, N, (K + STEP - 1) / STEP * 64, 1); }

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
