// C = A B^T on the 16-bit matrix cores, both operands contiguous along the summed axis, with bias, activation, residual and
// 8-bit checkpoint in the epilogue.
//
// A workgroup takes BM x BN sums.  Stages of 64 k go to LDS by LDS-direct loads (16 bytes a lane), two buffers: stage t + 1 is on its
// way while stage t is multiplied.  A row of a stage is 128 bytes, eight pieces of 16; piece c of row r lies in place
// c ^ (r & 7), so that the sixteen rows a fragment read touches fall on different banks.  The LDS end of such a load is fixed by
// the lane, so it is the address in memory that is exchanged.  Products are taken with B as the first operand: a lane then holds
// four neighbouring columns of one row, which it finishes and stores at once.
#include "dense_math.h"
#include "kernels.h"
#include "lds_dma.h"

namespace iolb {

namespace {

constexpr int STEP = 64;                               // k of a stage
constexpr int ROW_BYTES = 2 * STEP;

__device__ __forceinline__ void dma16(const char* base, unsigned offset, unsigned lds)
{
    lds_dma_load_16(reinterpret_cast<const float*>(base), offset, lds);
}

template <bool F16, int DT, int BM, int BN, int WM, int WN>
__global__ void __launch_bounds__(64 * WM * WN, 2)
dense_tile_kernel(DenseProduct p, int tiles_m, int tiles_n)
{
    constexpr int WAVES = WM * WN, MI = BM / WM / 16, NI = BN / WN / 16;
    constexpr int LA = BM / 8 / WAVES, LB = BN / 8 / WAVES;           // loads of a wave and stage: 8 rows each
    constexpr unsigned STAGE = (BM + BN) * ROW_BYTES;
    static_assert(NI % 2 == 0 && BM % (8 * WAVES) == 0 && BN % (8 * WAVES) == 0, "blocks of 32 columns, whole loads");
    extern __shared__ u32x4 lds16[];
    char* const lds = reinterpret_cast<char*>(lds16);
    const unsigned lds0 = lds_byte_address(reinterpret_cast<const float*>(lds));
    const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, grp = lane >> 4;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = wave / WN, wn = wave % WN;

    // Workgroups go to the eight XCDs in turn; each XCD takes a run of neighbouring tiles, in bands of eight tile rows, so that
    // its L2 holds the operands of a compact patch.
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
    const int steps_all = (p.K + STEP - 1) / STEP;
    const int s0 = (int)((long long)steps_all * blockIdx.y / p.splits), s1 = (int)((long long)steps_all * (blockIdx.y + 1) / p.splits);

    // Rows beyond the operand are read from its last row: their sums are never stored.
    unsigned a_off[LA], b_off[LB];
    const int piece = lane & 7;
#pragma unroll
    for (int i = 0; i < LA; ++i) {
        const int r = (i * WAVES + wave) * 8 + (lane >> 3), have = p.M - 1 - m0;
        a_off[i] = (unsigned)(2 * (r < have ? r : have)) * (unsigned)p.lda + 16u * place(r, piece);
    }
#pragma unroll
    for (int i = 0; i < LB; ++i) {
        const int r = (i * WAVES + wave) * 8 + (lane >> 3), have = p.N - 1 - n0;
        b_off[i] = (unsigned)(2 * (r < have ? r : have)) * (unsigned)p.ldb + 16u * place(r, piece);
    }
    const char* const a0 = static_cast<const char*>(p.a) + 2 * (m0 * p.lda);
    const char* const b0 = static_cast<const char*>(p.b) + 2 * (n0 * p.ldb);
    const int my_k = 8 * place(lane >> 3, piece);               // first k of the piece this lane fetches (rows step by 8)

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
            char* const at = lds + buf * STAGE;
            const bool inside = step * STEP + my_k < p.K;
#pragma unroll
            for (int i = 0; i < LA; ++i) {
                if (inside) dma16(a, a_off[i], to + (i * WAVES + wave) * 1024);
                else *reinterpret_cast<u32x4*>(at + (i * WAVES + wave) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
            }
#pragma unroll
            for (int i = 0; i < LB; ++i) {
                if (inside) dma16(b, b_off[i], to + BM * ROW_BYTES + (i * WAVES + wave) * 1024);
                else *reinterpret_cast<u32x4*>(at + BM * ROW_BYTES + (i * WAVES + wave) * 1024 + lane * 16) = u32x4{0, 0, 0, 0};
            }
        }
    };

    f32x4 acc[MI][NI];
#pragma unroll
    for (int i = 0; i < MI; ++i)
#pragma unroll
        for (int j = 0; j < NI; ++j) acc[i][j] = f32x4{0, 0, 0, 0};

    const int rounds = s1 > s0 ? p.segments * (s1 - s0) : 0;
    int seg = 0, step = s0;                            // of the stage that is loaded next
    if (rounds) load(seg, step, 0);
    int clear_at = p.segments > 1 ? (p.segments - 1) * (s1 - s0) : -1;
    for (int t = 0; t < rounds; ++t) {
        lds_dma_wait_all();
        __syncthreads();
        if (++step == s1) { step = s0; ++seg; }
        if (t + 1 < rounds) load(seg, step, (t + 1) & 1);
        if (t == clear_at) {
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[i][j][c] = fabsf(acc[i][j][c]) < __builtin_inff() ? acc[i][j][c] : 0.f;
        }
        const char* const at = lds + (t & 1) * STAGE;
#pragma unroll
        for (int kk = 0; kk < STEP / 32; ++kk) {
            u32x4 fa[MI], fb[NI];
#pragma unroll
            for (int j = 0; j < NI; ++j) {
                const int r = wn * (BN / WN) + j * 16 + l16;
                fb[j] = *reinterpret_cast<const u32x4*>(at + (BM + r) * ROW_BYTES + 16 * place(r, kk * 4 + grp));
            }
#pragma unroll
            for (int i = 0; i < MI; ++i) {
                const int r = wm * (BM / WM) + i * 16 + l16;
                fa[i] = *reinterpret_cast<const u32x4*>(at + r * ROW_BYTES + 16 * place(r, kk * 4 + grp));
            }
#pragma unroll
            for (int i = 0; i < MI; ++i)
#pragma unroll
                for (int j = 0; j < NI; ++j) acc[i][j] = multiply<F16>(fb[j], fa[i], acc[i][j]);
        }
    }

    const int mw = m0 + wm * (BM / WM) + l16, nw = n0 + wn * (BN / WN) + 4 * grp;
    if (p.splits > 1) {
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
#pragma unroll
    for (int i = 0; i < MI; ++i) {
        const int m = mw + i * 16;
        const bool row = m < p.M;
#pragma unroll
        for (int j = 0; j < NI; j += 2) {
            float z[2][4];
            float most = 0.f;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = nw + (j + h) * 16;
#pragma unroll
                for (int c = 0; c < 4; ++c) z[h][c] = acc[i][j + h][c];
                if (row && n < p.N) finish_sum<DT>(p.f, m, n, z[h]);
                if (p.f.zq) {
#pragma unroll
                    for (int c = 0; c < 4; ++c) most = n + c < p.N ? fmaxf(most, finite_magnitude(z[h][c])) : most;
                }
            }
            if (p.f.zq) {
                most = fmaxf(most, __shfl_xor(most, 16));
                most = fmaxf(most, __shfl_xor(most, 32));
            }
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int n = nw + (j + h) * 16;
                if (row && n < p.N) {
                    if (p.f.zq) finish_checkpoint<DT>(p.f, m, n, z[h], most, h == 0 && grp == 0);
                    finish_store<DT>(p.f, m, n, z[h]);
                }
            }
        }
    }
}

// The sums of the workgroups that shared a tile's K, added in their order, and the epilogue.
template <int DT>
__global__ void __launch_bounds__(256)
dense_join_kernel(DenseProduct p)
{
    const long long ld = (p.N + 3) / 4 * 4;
    const int n = (blockIdx.x * 256 + threadIdx.x) * 4;
    for (int m = blockIdx.y; m < p.M; m += gridDim.y) {
        float z[4] = {0.f, 0.f, 0.f, 0.f};
        if (n < p.N) {
            const float* from = p.partial + m * ld + n;
            for (int s = 0; s < p.splits; ++s, from += p.M * ld) {
                const f32x4 v = *reinterpret_cast<const f32x4*>(from);
#pragma unroll
                for (int c = 0; c < 4; ++c) z[c] += v[c];
            }
            finish_sum<DT>(p.f, m, n, z);
        }
        if (p.f.zq) {
            float most = 0.f;
#pragma unroll
            for (int c = 0; c < 4; ++c) most = n + c < p.N ? fmaxf(most, finite_magnitude(z[c])) : most;
#pragma unroll
            for (int d = 1; d < 8; d *= 2) most = fmaxf(most, __shfl_xor(most, d));
            if (n < p.N) finish_checkpoint<DT>(p.f, m, n, z, most, (threadIdx.x & 7) == 0);
        }
        if (n < p.N) finish_store<DT>(p.f, m, n, z);
    }
}

template <bool F16, int DT, int BM, int BN, int WM, int WN>
hipError_t launch(const DenseProduct& p, hipStream_t st)
{
    const auto kernel = dense_tile_kernel<F16, DT, BM, BN, WM, WN>;
    const hipError_t e = allow_large_lds(reinterpret_cast<const void*>(kernel));
    if (e != hipSuccess) return e;
    const int tm = (p.M + BM - 1) / BM, tn = (p.N + BN - 1) / BN;
    if ((long long)tm * tn > 0x7fffffffLL) return hipErrorInvalidValue;
    kernel<<<dim3(tm * tn, p.splits), 64 * WM * WN, 2 * (BM + BN) * ROW_BYTES, st>>>(p, tm, tn);
    return hipGetLastError();
}

template <bool F16, int DT>
hipError_t launch_tile(const DenseProduct& p, int tile, hipStream_t st)
{
    switch (tile) {
    case DENSE_TILE_256: return launch<F16, DT, 256, 256, 2, 4>(p, st);
    case DENSE_TILE_128: return launch<F16, DT, 128, 128, 2, 2>(p, st);
    default: return launch<F16, DT, 64, 128, 1, 4>(p, st);
    }
}

}  // namespace

// Blocks and shares.  A large block reads its operands less often; a small one, and K shared by several workgroups, fill
// the 256 compute units.
DenseTilePlan dense_tile_plan(int M, int N, int K, int segments)
{
    const auto tiles = [&](int bm, int bn) { return (long long)((M + bm - 1) / bm) * ((N + bn - 1) / bn); };
    DenseTilePlan plan{DENSE_TILE_256, 1};
    if (tiles(256, 256) >= 192) return plan;
    plan.tile = M <= 64 ? DENSE_TILE_64 : DENSE_TILE_128;
    const long long n = plan.tile == DENSE_TILE_64 ? tiles(64, 128) : tiles(128, 128);
    const int steps = (K + STEP - 1) / STEP;
    // at least four stages (of all segments together) a share
    const long long most = (long long)steps * segments / 4 < steps ? (long long)steps * segments / 4 : steps;
    long long splits = 512 / n;
    if (splits > most) splits = most;
    if (splits > 64) splits = 64;
    plan.splits = splits < 1 ? 1 : (int)splits;
    return plan;
}

hipError_t launch_dense_product(const DenseProduct& p, int tile, int dtype, hipStream_t st)
{
    hipError_t e = dtype == IOLB_F32 ? launch_tile<false, IOLB_F32>(p, tile, st)
                 : dtype == IOLB_F16 ? launch_tile<true, IOLB_F16>(p, tile, st) : launch_tile<false, IOLB_BF16>(p, tile, st);
    return e != hipSuccess || p.splits == 1 ? e : launch_dense_join(p, dtype, st);
}

hipError_t launch_dense_join(const DenseProduct& p, int dtype, hipStream_t st)
{
    const dim3 grid((unsigned)((p.N + 1023) / 1024), (unsigned)(p.M < 65535 ? p.M : 65535));
    if (dtype == IOLB_F32) dense_join_kernel<IOLB_F32><<<grid, 256, 0, st>>>(p);
    else if (dtype == IOLB_F16) dense_join_kernel<IOLB_F16><<<grid, 256, 0, st>>>(p);
    else dense_join_kernel<IOLB_BF16><<<grid, 256, 0, st>>>(p);
    return hipGetLastError();
}

}  // namespace iolb
