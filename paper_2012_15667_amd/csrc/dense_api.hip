// C entry points of dense layers, 8-bit checkpoints and gradients: argument checks, operand layouts, workspace, launches.
#include <algorithm>

#include "dense.h"

namespace {

using namespace iolb;

constexpr int64_t MOST = (int64_t)1 << 30;             // rows and columns
constexpr int64_t MOST_K = (int64_t)1 << 22;           // summed axis: a tile's rows are addressed with 32-bit offsets

bool known_type(int dtype) { return dtype == IOLB_F32 || dtype == IOLB_F16 || dtype == IOLB_BF16; }
bool known_act(int act) { return act >= IOLB_ACT_NONE && act <= IOLB_ACT_GELU_TANH; }
int64_t size_of(int dtype) { return dtype == IOLB_F32 ? 4 : 2; }
bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
int64_t up8(int64_t n) { return (n + 7) / 8 * 8; }
// A launch counts its threads along an axis in 32 bits.
bool launchable(int64_t workgroups, int threads) { return workgroups * threads <= 0xffffffffLL; }
int64_t layout_groups(int64_t rows, int64_t cols) { return (rows + 63) / 64 * ((cols + 63) / 64); }

// Hands out pieces of the caller's workspace; with no memory behind it, counts them.
struct Pieces {
    char* base;
    size_t used = 0;
    void* take(size_t bytes)
    {
        void* const p = base ? base + used : nullptr;
        used += (bytes + 255) & ~(size_t)255;
        return p;
    }
};

// A 16-bit operand that the product kernel can read in place.
bool direct(const void* p, int64_t ld, int64_t k, int dtype)
{
    return dtype != IOLB_F32 && k % 8 == 0 && ld % 8 == 0 && ld <= MOST_K && aligned_to(p, 16);
}

// The six products of three parts, smallest first; the three with a second operand that is one part exactly.
void segments(DenseProduct* p, int planes_a, int planes_b, int64_t a_elems, int64_t b_elems)
{
    static const int six[6][2] = {{2, 0}, {0, 2}, {1, 1}, {1, 0}, {0, 1}, {0, 0}};
    p->segments = 0;
    for (const auto& s : six)
        if (s[0] < planes_a && s[1] < planes_b) {
            p->a_plane[p->segments] = s[0] * a_elems;
            p->b_plane[p->segments] = s[1] * b_elems;
            ++p->segments;
        }
}

#define DENSE_HIP(call)                                          \
    do {                                                         \
        const hipError_t e__ = (call);                           \
        if (e__ != hipSuccess) return note_hip_error(e__);       \
    } while (0)

int check_linear(const iolb_linear_args& a)
{
    if (a.M < 0 || a.N < 0 || a.K < 0) return IOLB_EINVAL;
    if (!known_type(a.dtype) || !known_act(a.act)) return IOLB_EUNSUPPORTED;
    if (a.M > MOST || a.N > MOST || a.K > MOST_K) return IOLB_EUNSUPPORTED;
    if (a.M == 0 || a.N == 0) return IOLB_OK;
    if (!a.y || (a.K > 0 && (!a.x || !a.w)) || !a.zq != !a.ze) return IOLB_EINVAL;
    if ((a.M > 1 && (a.ldx < a.K || a.ldy < a.N || (a.residual && a.ldr < a.N))) || (a.N > 1 && a.ldw < a.K)) return IOLB_EINVAL;
    const size_t size = (size_t)size_of(a.dtype);
    for (const void* p : {a.x, a.w, a.bias, a.residual, (const void*)a.y})
        if (!aligned_to(p, size)) return IOLB_EINVAL;
    return IOLB_OK;
}

// Plans the call; with `launch`, makes it.  *need: bytes of workspace.
int run_linear(const iolb_linear_args& a, void* ws, size_t* need, bool launch)
{
    *need = 0;
    if (a.M == 0 || a.N == 0) return IOLB_OK;
    Pieces pieces{static_cast<char*>(ws)};
    const int64_t Kp = up8(a.K);
    DenseProduct p{};
    p.f = DenseFinish{a.bias, a.residual, a.y, a.zq, a.ze, a.ldr, a.ldy, (int)a.M, (int)a.N, a.act, a.residual_first != 0};
    p.M = (int)a.M; p.N = (int)a.N;
    if (dense_rows_wanted(a.M, a.N, a.K, a.dtype, false)) {
        p.a = a.x; p.lda = a.ldx;
        p.b = a.w; p.ldb = a.ldw;
        p.K = (int)a.K;
        const DenseRowsPlan plan = dense_rows_plan(p.M, p.N, p.K, a.dtype, false, a.zq != nullptr);
        if (!dense_rows_launchable(plan, p.M, p.N, p.K, false)) return IOLB_EUNSUPPORTED;
        p.splits = plan.splits; p.per = plan.per; p.block_columns = plan.block_columns;
        if (plan.join) p.partial = static_cast<float*>(pieces.take(dense_partial_bytes(plan.splits, a.M, a.N)));
        *need = pieces.used;
        if (launch) DENSE_HIP(launch_dense_rows(p, false, plan.join, a.dtype, call_stream()));
        return IOLB_OK;
    }
    p.K = (int)Kp;
    const int planes = a.dtype == IOLB_F32 ? 3 : 1;
    segments(&p, planes, planes, a.M * Kp, a.N * Kp);
    const bool x_direct = direct(a.x, a.ldx, a.K, a.dtype) || a.K == 0, w_direct = direct(a.w, a.ldw, a.K, a.dtype) || a.K == 0;
    p.a = a.x; p.lda = a.ldx;
    p.b = a.w; p.ldb = a.ldw;
    void *xp = nullptr, *wp = nullptr;
    if (!x_direct) { p.a = xp = pieces.take((size_t)planes * a.M * Kp * 2); p.lda = Kp; }
    if (!w_direct) { p.b = wp = pieces.take((size_t)planes * a.N * Kp * 2); p.ldb = Kp; }
    // Large fp32 products in two fp16 parts, three products in place of six.  Whether an operand's rows allow it is found out on the GPU; the
    // launches for three parts follow all the same and end at once if it does and no block of sums was left to them, which costs some 10 us.  Three parts against two, us:
    // 1024 x 1024 x 1024 37 / 40, 2048 x 1024 x 1024 50 / 49, 4096 x 1024 x 1024 74 / 57, 2048 x 2048 x 2048 115 / 96, 4096 x 4096 x 4096 633 / 395.
    DenseProduct h{};
    const bool halves = planes == 3 && (double)a.M * a.N * a.K >= 3e9 && launchable(dense_halves_groups(a.M, a.N, a.K), 256);
    const DenseTilePlan plan = dense_tile_plan(p.M, p.N, p.K, halves ? 3 : p.segments);         // (one for both: they finish the same blocks)
    if (!dense_tile_launchable(plan, p.M, p.N) || !launchable((x_direct ? 0 : layout_groups(a.M, a.K)) + (w_direct ? 0 : layout_groups(a.N, a.K)), 256))
        return IOLB_EUNSUPPORTED;
    p.splits = plan.splits;
    int* uneven = nullptr;
    DenseHalves hx{static_cast<const float*>(a.x), a.ldx, (int)a.M}, hw{static_cast<const float*>(a.w), a.ldw, (int)a.N};
    if (halves) {
        // (where the three parts go: those are laid out when the product of these is done)
        hx.planes = static_cast<unsigned short*>(xp);
        hw.planes = static_cast<unsigned short*>(wp);
        for (DenseHalves* t : {&hx, &hw}) t->scales = static_cast<DenseScale*>(pieces.take((size_t)t->rows * sizeof(DenseScale)));
        p.uneven = uneven = static_cast<int*>(pieces.take(8));
        p.left = static_cast<int*>(pieces.take((size_t)dense_finish_blocks(plan, p.M, p.N) * 4));
        p.when = 1;
        h = p;
        h.when = 0;
        h.a = hx.planes; h.lda = Kp;
        h.b = hw.planes; h.ldb = Kp;
        h.scales_a = hx.scales; h.values_a = hx.x; h.ld_values_a = hx.ld;
        h.scales_b = hw.scales; h.values_b = hw.x; h.ld_values_b = hw.ld;
        h.values_k = (int)a.K;
        h.segments = 3;                                                    // l h, h l, h h
        h.a_plane[0] = a.M * Kp; h.a_plane[1] = h.a_plane[2] = 0;
        h.b_plane[1] = a.N * Kp; h.b_plane[0] = h.b_plane[2] = 0;
    }
    if (plan.splits > 1) h.partial = p.partial = static_cast<float*>(pieces.take(dense_partial_bytes(plan.splits, a.M, a.N)));
    *need = pieces.used;
    if (!launch) return IOLB_OK;

    const hipStream_t st = call_stream();
    if (halves) {
        DENSE_HIP(launch_dense_halves(hx, hw, (int)a.K, Kp, uneven, st));
        DENSE_HIP(launch_dense_product(h, plan.tile, a.dtype, st));
    }
    DenseLayouts layouts{};
    layouts.uneven = uneven;
    const auto lay = [&](const void* src, int64_t ld, int64_t rows, void* to) {
        DenseLayout& l = layouts.of[layouts.count++];
        l.source = DENSE_FROM_TENSOR; l.planes = planes;
        l.rows = (int)rows; l.cols = (int)a.K;
        l.src = src; l.ld = ld;
        l.rowmajor = to; l.ld_rm = Kp;
    };
    if (!x_direct) lay(a.x, a.ldx, a.M, xp);
    if (!w_direct) lay(a.w, a.ldw, a.N, wp);
    if (layouts.count) DENSE_HIP(launch_dense_layouts(a.dtype, layouts, st));
    DENSE_HIP(launch_dense_product(p, plan.tile, a.dtype, st));
    return IOLB_OK;
}

int check_backward(const iolb_linear_backward_args& a)
{
    if (a.M < 0 || a.N < 0 || a.K < 0) return IOLB_EINVAL;
    if (!known_type(a.dtype) || !known_act(a.act) || !known_act(a.x_act)) return IOLB_EUNSUPPORTED;
    // each of the three is the summed axis of a product, or a dimension of one
    if (a.M > MOST_K || a.N > MOST_K || a.K > MOST) return IOLB_EUNSUPPORTED;
    if ((!a.xq) != (!a.xe) || (!a.zq) != (!a.ze)) return IOLB_EINVAL;
    if (a.M > 0 && a.N > 0) {
        if (!a.dy || (a.M > 1 && a.ldy < a.N)) return IOLB_EINVAL;
        if (a.act != IOLB_ACT_NONE && !a.zq) return IOLB_EINVAL;
        if (a.dx && a.K > 0 && (!a.w || (a.N > 1 && a.ldw < a.K))) return IOLB_EINVAL;
        if (a.dw && a.K > 0 && !a.xq) return IOLB_EINVAL;
    }
    const size_t size = (size_t)size_of(a.dtype);
    for (const void* p : {a.dy, a.w, (const void*)a.dx, (const void*)a.dw, (const void*)a.db, (const void*)a.dz})
        if (!aligned_to(p, size)) return IOLB_EINVAL;
    return IOLB_OK;
}

int run_backward(const iolb_linear_backward_args& a, void* ws, size_t* need, bool launch)
{
    Pieces pieces{static_cast<char*>(ws)};
    const int planes = a.dtype == IOLB_F32 ? 3 : 1;
    // the input's checkpoint is exact in one bf16 part, unless a smooth activation has to be taken of it
    const int planes_x = planes == 3 && a.x_act != IOLB_ACT_NONE && a.x_act != IOLB_ACT_RELU ? 3 : 1;
    const int64_t Mp = up8(a.M), Np = up8(a.N);
    const bool want_dx = a.dx && a.M > 0 && a.K > 0, few = dense_rows_wanted(a.M, a.N, a.K, a.dtype, true), want_dw = a.dw && a.N > 0 && a.K > 0;
    const bool has_z = a.act != IOLB_ACT_NONE;

    // dz = dy act'(z) along the rows for dx (dy itself where that is it), transposed for dW
    // (few rows: dx is taken from dz in the tensor's own type, dense, and from w as it is)
    const bool dy_is_dz = !has_z && (few || direct(a.dy, a.ldy, a.N, a.dtype));
    const bool dz_is_plane = a.dz && !few && direct(a.dz, a.N, a.N, a.dtype);
    const void* dz = a.dy;
    int64_t ld_dz = a.ldy;
    void *dz_to = nullptr, *dz_copy = a.dz, *dzt = nullptr, *wt = nullptr, *xt = nullptr;
    if (want_dx && !dy_is_dz && few) {
        if (!dz_copy) dz_copy = pieces.take((size_t)(a.M * a.N * size_of(a.dtype)));
        ld_dz = a.N;
        dz = dz_copy;
    } else if (want_dx && !dy_is_dz) {
        ld_dz = Np;
        dz = dz_to = dz_is_plane ? a.dz : pieces.take((size_t)planes * a.M * Np * 2);
        if (dz_is_plane) dz_copy = nullptr;
    }
    if (want_dw) {
        dzt = pieces.take((size_t)planes * a.N * Mp * 2);
        xt = pieces.take((size_t)planes_x * a.K * Mp * 2);
    }
    if (want_dx && !few) wt = pieces.take((size_t)planes * a.K * Np * 2);
    const int row_blocks = (int)((a.M + 63) / 64);
    // (up to 64 rows the first stage's sums are the sums)
    const bool one_block = row_blocks == 1;
    float* const sums = static_cast<float*>(a.db && !one_block ? pieces.take((size_t)row_blocks * a.N * 4) : nullptr);

    DenseProduct px{}, pw{};
    DenseTilePlan plan_x{}, plan_w{};
    DenseRowsPlan rows_x{};
    size_t partial_x = 0, partial_w = 0;
    bool outer = false;
    if (want_dx && few) {
        px.M = (int)a.M; px.N = (int)a.K; px.K = (int)a.N;
        px.a = dz; px.lda = ld_dz;
        px.b = a.w; px.ldb = a.ldw;
        rows_x = dense_rows_plan(px.M, px.N, px.K, a.dtype, true, false);
        if (!dense_rows_launchable(rows_x, px.M, px.N, px.K, true)) return IOLB_EUNSUPPORTED;
        px.splits = rows_x.splits; px.per = rows_x.per; px.block_columns = rows_x.block_columns;
        if (rows_x.join) partial_x = dense_partial_bytes(px.splits, px.M, px.N);
    } else if (want_dx) {
        px.M = (int)a.M; px.N = (int)a.K; px.K = (int)Np;
        px.a = dz; px.lda = ld_dz; px.b = wt; px.ldb = Np;
        segments(&px, planes, planes, a.M * Np, a.K * Np);
        plan_x = dense_tile_plan(px.M, px.N, px.K, px.segments);
        if (!dense_tile_launchable(plan_x, px.M, px.N)) return IOLB_EUNSUPPORTED;
        px.splits = plan_x.splits;
        if (px.splits > 1) partial_x = dense_partial_bytes(px.splits, px.M, px.N);
    }
    if (want_dw) {
        pw.M = (int)a.N; pw.N = (int)a.K; pw.K = (int)Mp;
        pw.a = dzt; pw.lda = Mp; pw.b = xt; pw.ldb = Mp;
        segments(&pw, planes, planes_x, a.N * Mp, a.K * Mp);
        outer = a.M > 0 && a.M <= DENSE_OUTER_MOST && a.N <= DENSE_OUTER_ROWS;
        plan_w = dense_tile_plan(pw.M, pw.N, pw.K, pw.segments);
        if (!outer && !dense_tile_launchable(plan_w, pw.M, pw.N)) return IOLB_EUNSUPPORTED;
        pw.splits = outer ? 1 : plan_w.splits;
        if (pw.splits > 1) partial_w = dense_partial_bytes(pw.splits, pw.M, pw.N);
    }
    if (!launchable(layout_groups(a.M, a.N) + (wt ? layout_groups(a.N, a.K) : 0) + (want_dw ? layout_groups(a.M, a.K) : 0), 256)) return IOLB_EUNSUPPORTED;
    // one after the other on the stream: they share the room for partial sums
    px.partial = pw.partial = static_cast<float*>(pieces.take(std::max(partial_x, partial_w)));
    *need = pieces.used;
    if (!launch) return IOLB_OK;

    const hipStream_t st = call_stream();
    DenseLayouts layouts{};
    if (a.M > 0 && a.N > 0 && (dz_to || dzt || dz_copy || a.db)) {
        DenseLayout& l = layouts.of[layouts.count++];
        l.source = DENSE_FROM_GRADIENT; l.planes = planes;
        l.rows = (int)a.M; l.cols = (int)a.N;
        l.src = a.dy; l.ld = a.ldy;
        l.q = has_z ? a.zq : nullptr; l.e = a.ze; l.act = a.act;
        l.rowmajor = dz_to; l.ld_rm = Np;
        l.transposed = dzt; l.ld_tr = Mp;
        l.copy = dz_copy;
        l.colsum = sums; l.total = one_block ? a.db : nullptr;
    }
    if (wt) {
        DenseLayout& l = layouts.of[layouts.count++];
        l.source = DENSE_FROM_TENSOR; l.planes = planes;
        l.rows = (int)a.N; l.cols = (int)a.K;
        l.src = a.w; l.ld = a.ldw;
        l.transposed = wt; l.ld_tr = Np;
    }
    if (want_dw && a.M > 0) {
        DenseLayout& l = layouts.of[layouts.count++];
        l.source = DENSE_FROM_CHECKPOINT; l.planes = planes_x;
        l.rows = (int)a.M; l.cols = (int)a.K;
        l.q = a.xq; l.e = a.xe; l.act = a.x_act;
        l.transposed = xt; l.ld_tr = Mp;
    }
    if (layouts.count) DENSE_HIP(launch_dense_layouts(a.dtype, layouts, st));
    if (a.db && a.N > 0 && !one_block) DENSE_HIP(launch_dense_colsum(sums, row_blocks, (int)a.N, a.db, a.dtype, st));
    const auto finish = [&](void* out, int64_t m, int64_t n) {
        DenseFinish f{};
        f.y = out; f.ldy = n; f.M = (int)m; f.N = (int)n;
        f.act = IOLB_ACT_NONE;
        return f;
    };
    if (want_dx && few) {
        px.f = finish(a.dx, a.M, a.K);
        DENSE_HIP(launch_dense_rows(px, true, rows_x.join, a.dtype, st));
    } else if (want_dx) {
        px.f = finish(a.dx, a.M, a.K);
        DENSE_HIP(launch_dense_product(px, plan_x.tile, a.dtype, st));
    }
    if (want_dw) {
        pw.f = finish(a.dw, a.N, a.K);
        if (outer) DENSE_HIP(launch_dense_outer(pw, planes_x, a.N * Mp, a.K * Mp, a.dtype, st));
        else DENSE_HIP(launch_dense_product(pw, plan_w.tile, a.dtype, st));
    }
    return IOLB_OK;
}

// Nothing the C++ runtime throws crosses the C boundary.
template <class F>
int guarded(F f) noexcept
{
    try {
        return f();
    } catch (...) {
        return note_hip_error(hipErrorOutOfMemory);
    }
}

template <class Args>
int checked_call(const Args* a, void* ws, size_t ws_bytes, int (*check)(const Args&), int (*run)(const Args&, void*, size_t*, bool))
{
    return guarded([&] {
        if (!a) return IOLB_EINVAL;
        const int rc = check(*a);
        if (rc != IOLB_OK) return rc;
        size_t need = 0;
        const int planned = run(*a, nullptr, &need, false);
        if (planned != IOLB_OK) return planned;
        if (need && (!ws || ws_bytes < need || !aligned_to(ws, 256))) return IOLB_EWORKSPACE;
        return run(*a, ws, &need, true);
    });
}

template <class Args>
int needed_bytes(const Args* a, size_t* bytes, int (*check)(const Args&), int (*run)(const Args&, void*, size_t*, bool))
{
    return guarded([&] {
        if (!a || !bytes) return IOLB_EINVAL;
        const int rc = check(*a);
        if (rc != IOLB_OK) return rc;
        return run(*a, nullptr, bytes, false);
    });
}

int check_checkpoint(int64_t rows, int64_t cols, int64_t ld, int dtype, const void* values, const void* q, const void* e)
{
    if (rows < 0 || cols < 0) return IOLB_EINVAL;
    if (!known_type(dtype) || rows > MOST || cols > MOST) return IOLB_EUNSUPPORTED;
    if (rows == 0 || cols == 0) return IOLB_OK;
    if (!values || !q || !e || (rows > 1 && ld < cols) || !aligned_to(values, (size_t)size_of(dtype))) return IOLB_EINVAL;
    return IOLB_OK;
}

}  // namespace

extern "C" {

int iolb_linear_workspace_bytes(const iolb_linear_args* args, size_t* bytes) { return needed_bytes(args, bytes, check_linear, run_linear); }

int iolb_linear(const iolb_linear_args* args, void* workspace, size_t workspace_bytes)
{
    return checked_call(args, workspace, workspace_bytes, check_linear, run_linear);
}

int iolb_linear_backward_workspace_bytes(const iolb_linear_backward_args* args, size_t* bytes)
{
    return needed_bytes(args, bytes, check_backward, run_backward);
}

int iolb_linear_backward(const iolb_linear_backward_args* args, void* workspace, size_t workspace_bytes)
{
    return checked_call(args, workspace, workspace_bytes, check_backward, run_backward);
}

int iolb_checkpoint_pack(const void* x, int64_t ldx, int64_t rows, int64_t cols, int dtype, int8_t* q, uint8_t* e)
{
    return guarded([&] {
        const int rc = check_checkpoint(rows, cols, ldx, dtype, x, q, e);
        if (rc != IOLB_OK || rows == 0 || cols == 0) return rc;
        DENSE_HIP(launch_checkpoint_pack(x, ldx, (int)rows, (int)cols, dtype, q, e, call_stream()));
        return IOLB_OK;
    });
}

int iolb_checkpoint_unpack(const int8_t* q, const uint8_t* e, int64_t rows, int64_t cols, int act, int dtype, void* y, int64_t ldy)
{
    return guarded([&] {
        const int rc = check_checkpoint(rows, cols, ldy, dtype, y, q, e);
        if (rc != IOLB_OK) return rc;
        if (!known_act(act)) return IOLB_EUNSUPPORTED;
        if (rows == 0 || cols == 0) return IOLB_OK;
        DENSE_HIP(launch_checkpoint_unpack(q, e, (int)rows, (int)cols, act, dtype, y, ldy, call_stream()));
        return IOLB_OK;
    });
}

}  // extern "C"
