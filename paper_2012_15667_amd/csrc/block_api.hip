// C entry points of block norms, dropout and layers in 4 bits: argument checks, workspace, launches.
#include <cmath>
#include <initializer_list>

#include "block.h"

namespace {

using namespace iolb;

constexpr int64_t MOST = (int64_t)1 << 30;             // rows and columns
constexpr int64_t MOST_K = (int64_t)1 << 22;           // summed axes: a tile's rows are addressed with 32-bit offsets

bool known_type(int dtype) { return dtype == IOLB_F32 || dtype == IOLB_F16 || dtype == IOLB_BF16; }
bool known_act(int act) { return act >= IOLB_ACT_NONE && act <= IOLB_ACT_GELU_TANH; }
bool known_norm(int kind) { return kind >= IOLB_NORM_NONE && kind <= IOLB_NORM_LAYER; }
size_t size_of(int dtype) { return dtype == IOLB_F32 ? 4 : 2; }
bool aligned_to(const void* p, size_t bytes) { return reinterpret_cast<uintptr_t>(p) % bytes == 0; }
bool all_aligned_to(std::initializer_list<const void*> all, size_t bytes)
{
    for (const void* p : all)
        if (!aligned_to(p, bytes)) return false;
    return true;
}
size_t up256(size_t n) { return (n + 255) & ~(size_t)255; }

#define BLOCK_HIP(call)                                          \
    do {                                                         \
        const hipError_t e__ = (call);                           \
        if (e__ != hipSuccess) return note_hip_error(e__);       \
    } while (0)

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

int check_norm(const iolb_block_norm_args& a)
{
    if (a.M < 0 || a.N < 0) return IOLB_EINVAL;
    if (!known_type(a.dtype) || !known_norm(a.post) || !known_norm(a.pre) || a.M > MOST || a.N > MOST) return IOLB_EUNSUPPORTED;
    if (a.gate && (a.groups < 1 || a.M % a.groups)) return IOLB_EINVAL;
    if (!(a.eps >= 0.f)) return IOLB_EINVAL;
    if (a.M == 0 || a.N == 0) return IOLB_OK;               // (tensors without values may have no address)
    if (!a.h && (a.gate || a.x_out || a.post != IOLB_NORM_NONE || a.scale != 1.f)) return IOLB_EINVAL;
    if (a.post == IOLB_NORM_NONE && (a.post_weight || a.post_bias)) return IOLB_EINVAL;
    if (a.pre == IOLB_NORM_NONE && (a.pre_weight || a.pre_bias || a.y)) return IOLB_EINVAL;
    if (!all_aligned_to({a.x, a.h, a.post_weight, a.post_bias, a.gate, a.pre_weight, a.pre_bias, a.x_out, a.y}, size_of(a.dtype))) return IOLB_EINVAL;
    if (!a.x || (a.h && !a.x_out) || (a.pre != IOLB_NORM_NONE && !a.y)) return IOLB_EINVAL;
    if (a.M > 1 && (a.ldx < a.N || (a.h && (a.ldh < a.N || a.ldo < a.N)) || (a.y && a.ldy < a.N))) return IOLB_EINVAL;
    return IOLB_OK;
}

int check_norm_backward(const iolb_block_norm_backward_args& a)
{
    if (a.M < 0 || a.N < 0) return IOLB_EINVAL;
    if (!known_type(a.dtype) || !known_norm(a.post) || !known_norm(a.pre) || a.M > MOST_K || a.N > MOST_K) return IOLB_EUNSUPPORTED;
    if (a.gate && (a.groups < 1 || a.M % a.groups)) return IOLB_EINVAL;
    if (a.gate && a.groups > MOST_K) return IOLB_EUNSUPPORTED;      // (without rows any number divides them)
    if (!(a.eps >= 0.f)) return IOLB_EINVAL;
    if (a.N && !a.gate && a.dgate) return IOLB_EINVAL;
    if (a.M == 0 || a.N == 0) return IOLB_OK;               // (tensors without values may have no address)
    if (!a.h && (a.gate || a.dh || a.dgate || a.post != IOLB_NORM_NONE || a.scale != 1.f)) return IOLB_EINVAL;
    if (a.post == IOLB_NORM_NONE && (a.post_weight || a.post_bias || a.dpost_weight || a.dpost_bias)) return IOLB_EINVAL;
    if (a.pre == IOLB_NORM_NONE && (a.pre_weight || a.dy)) return IOLB_EINVAL;
    if (!a.dy && (a.dpre_weight || a.dpre_bias)) return IOLB_EINVAL;
    if (!all_aligned_to({a.dy, a.dx_out, a.x, a.h, a.post_weight, a.post_bias, a.gate, a.pre_weight, a.dx, a.dh, a.dgate, a.dpost_weight, a.dpost_bias,
                         a.dpre_weight, a.dpre_bias}, size_of(a.dtype))) return IOLB_EINVAL;
    if ((!a.dy && !a.dx_out) || (a.dy && !a.x)) return IOLB_EINVAL;
    if (a.M > 1 && ((a.dy && (a.lddy < a.N || a.ldx < a.N)) || (a.dx_out && a.lddx < a.N) || (a.h && a.ldh < a.N))) return IOLB_EINVAL;
    return IOLB_OK;
}

int run_norm_backward(const iolb_block_norm_backward_args& a, void* ws, size_t* need, bool launch)
{
    *need = 0;
    if (a.N == 0 || (a.M == 0 && !a.dpost_weight && !a.dpost_bias && !a.dpre_weight && !a.dpre_bias && !a.dgate)) return IOLB_OK;
    BlockNormBackward p{};
    p.dy = a.dy; p.dout = a.dx_out; p.x = a.x; p.h = a.h; p.gate = a.gate;
    p.post_weight = a.post_weight; p.post_bias = a.post_bias; p.pre_weight = a.pre_weight;
    p.dx = a.dx; p.dh = a.dh;
    p.dgate = a.dgate; p.dpost_weight = a.dpost_weight; p.dpost_bias = a.dpost_bias; p.dpre_weight = a.dpre_weight; p.dpre_bias = a.dpre_bias;
    p.lddy = a.lddy; p.lddout = a.lddx; p.ldx = a.ldx; p.ldh = a.ldh;
    p.M = (int)a.M; p.N = (int)a.N;
    p.post = a.post; p.pre = a.pre;
    p.groups = a.gate ? (int)a.groups : 1;
    p.rows_per_group = p.M / p.groups;
    p.scale = a.scale; p.eps = a.eps;
    if (p.M == 0) p.gate = p.post_weight = p.post_bias = nullptr;   // (sums of nothing are 0: no factor of theirs, an infinite one, makes them NaN)
    const NormBackwardPlan plan = block_norm_backward_plan(p, a.dtype);
    if (!plan.launchable) return IOLB_EUNSUPPORTED;
    *need = up256(plan.row_bytes) + up256(plan.column_bytes);
    if (!launch) return IOLB_OK;
    p.rows = static_cast<float*>(plan.row_bytes ? ws : nullptr);
    if (plan.column_bytes) p.columns = reinterpret_cast<float*>(static_cast<char*>(ws) + up256(plan.row_bytes));
    BLOCK_HIP(launch_block_norm_backward(p, plan, a.dtype, call_stream()));
    return IOLB_OK;
}

int check_linear(const iolb_linear_mx4_args& a)
{
    if (a.M < 0 || a.N < 0 || a.K < 0) return IOLB_EINVAL;
    if (!known_type(a.dtype) || !known_act(a.act)) return IOLB_EUNSUPPORTED;
    if (a.M > MOST || a.N > MOST || a.K > MOST_K) return IOLB_EUNSUPPORTED;
    if (a.x && (a.x_codes || a.x_scales)) return IOLB_EINVAL;
    if (!all_aligned_to({a.x, a.bias, a.residual, a.y}, size_of(a.dtype)) || !all_aligned_to({a.x_codes, a.w_codes}, 16) ||
        !all_aligned_to({a.x_scales, a.w_scales}, 4)) return IOLB_EINVAL;
    if (a.M == 0 || a.N == 0) return IOLB_OK;
    if (!a.y || (a.K > 0 && (!a.w_codes || !a.w_scales || (!a.x && (!a.x_codes || !a.x_scales))))) return IOLB_EINVAL;
    if (a.M > 1 && ((a.x && a.ldx < a.K) || a.ldy < a.N || (a.residual && a.ldr < a.N))) return IOLB_EINVAL;
    return IOLB_OK;
}

int run_linear(const iolb_linear_mx4_args& a, void* ws, size_t* need, bool launch)
{
    *need = 0;
    if (a.M == 0 || a.N == 0) return IOLB_OK;
    Mx4Product p{};
    p.M = (int)a.M; p.N = (int)a.N; p.K = (int)a.K;
    p.a = a.x_codes; p.a_scales = a.x_scales;
    p.b = a.w_codes; p.b_scales = a.w_scales;
    p.f = DenseFinish{a.bias, a.residual, a.y, nullptr, nullptr, a.ldr, a.ldy, p.M, p.N, a.act, a.residual_first != 0};
    const bool few = mx4_few_wanted(a.M, a.N, a.K), pack = a.x && a.K > 0 && !mx4_short(a.M, a.N, a.K);
    const DenseTilePlan plan = few ? DenseTilePlan{0, 1} : mx4_tile_plan(p.M, p.N, p.K);
    if (few ? !mx4_few_launchable(p.N) : !dense_tile_launchable(plan, p.M, p.N)) return IOLB_EUNSUPPORTED;
    p.splits = plan.splits;
    const size_t codes = up256((size_t)a.M * mx4_pitch(a.K)), scales = up256((size_t)a.M * mx4_scale_pitch(a.K));
    const size_t partial = plan.splits > 1 ? up256(dense_partial_bytes(plan.splits, a.M, a.N)) : 0;
    *need = (pack ? codes + scales : 0) + partial;
    if (!launch) return IOLB_OK;
    const hipStream_t st = call_stream();
    if (pack) {
        uint8_t* const to = static_cast<uint8_t*>(ws);
        BLOCK_HIP(launch_mx4_pack(a.x, a.ldx, p.M, p.K, a.dtype, to, to + codes, st));
        p.a = to;
        p.a_scales = to + codes;
    }
    if (few && !pack) { p.x = a.x; p.ldx = a.ldx; }
    if (partial) p.partial = reinterpret_cast<float*>(static_cast<char*>(ws) + (pack ? codes + scales : 0));
    BLOCK_HIP(few ? launch_mx4_few(p, a.dtype, st) : launch_mx4_tile(p, plan.tile, a.dtype, st));
    return IOLB_OK;
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

int check_mx4(int64_t rows, int64_t cols, int64_t ld, int dtype, const void* values, const void* codes, const void* scales)
{
    if (rows < 0 || cols < 0) return IOLB_EINVAL;
    if (!known_type(dtype) || rows > MOST || cols > MOST) return IOLB_EUNSUPPORTED;
    if (!aligned_to(values, size_of(dtype)) || !aligned_to(codes, 16) || !aligned_to(scales, 4)) return IOLB_EINVAL;
    if (rows == 0 || cols == 0) return IOLB_OK;
    if (!values || !codes || !scales || (rows > 1 && ld < cols)) return IOLB_EINVAL;
    return IOLB_OK;
}

}  // namespace

extern "C" {

int iolb_block_norm(const iolb_block_norm_args* args)
{
    return guarded([&] {
        if (!args) return IOLB_EINVAL;
        const iolb_block_norm_args& a = *args;
        const int rc = check_norm(a);
        if (rc != IOLB_OK || a.M == 0 || a.N == 0 || (!a.h && !a.y)) return rc;
        BlockNorm p{};
        p.x = a.x; p.h = a.h; p.gate = a.gate;
        p.post_weight = a.post_weight; p.post_bias = a.post_bias; p.pre_weight = a.pre_weight; p.pre_bias = a.pre_bias;
        p.out = a.x_out; p.y = a.y;
        p.ldx = a.ldx; p.ldh = a.ldh; p.ldo = a.ldo; p.ldy = a.ldy;
        p.M = (int)a.M; p.N = (int)a.N;
        p.post = a.post; p.pre = a.pre;
        p.rows_per_group = a.gate ? (int)(a.M / a.groups) : 1;
        p.scale = a.scale; p.eps = a.eps;
        BLOCK_HIP(launch_block_norm(p, a.dtype, call_stream()));
        return IOLB_OK;
    });
}

int iolb_block_norm_backward_workspace_bytes(const iolb_block_norm_backward_args* args, size_t* bytes)
{
    return needed_bytes(args, bytes, check_norm_backward, run_norm_backward);
}

int iolb_block_norm_backward(const iolb_block_norm_backward_args* args, void* workspace, size_t workspace_bytes)
{
    return checked_call(args, workspace, workspace_bytes, check_norm_backward, run_norm_backward);
}

int iolb_dropout(const iolb_dropout_args* args)
{
    return guarded([&] {
        if (!args) return IOLB_EINVAL;
        const iolb_dropout_args& a = *args;
        if (a.rows < 0 || a.cols < 0 || !(a.p >= 0. && a.p <= 1.)) return IOLB_EINVAL;
        if (!known_type(a.dtype) || a.rows > MOST || a.cols > MOST) return IOLB_EUNSUPPORTED;
        if (!a.zq != !a.ze || !all_aligned_to({a.x, a.residual, a.y}, size_of(a.dtype)) || !aligned_to(a.counter, 8)) return IOLB_EINVAL;
        if (a.rows == 0 || a.cols == 0) return IOLB_OK;
        if (!a.x || !a.y) return IOLB_EINVAL;
        if (a.rows > 1 && (a.ldx < a.cols || a.ldy < a.cols || (a.residual && a.ldr < a.cols))) return IOLB_EINVAL;
        Dropout p{};
        p.x = a.x; p.residual = a.residual; p.y = a.y;
        p.zq = a.zq; p.ze = a.ze;
        p.ldx = a.ldx; p.ldr = a.ldr; p.ldy = a.ldy;
        p.rows = (int)a.rows; p.cols = (int)a.cols;
        const long t = std::lrint(a.p * 65536.);
        p.least = a.p < 1. && t > 65535 ? 65535u : (unsigned)t;
        p.scale = p.least < 65536u ? (float)(65536. / (65536. - p.least)) : 0.f;
        p.seed = a.seed; p.offset = a.offset;
        p.counter = reinterpret_cast<const unsigned long long*>(a.counter);
        BLOCK_HIP(launch_dropout(p, a.dtype, call_stream()));
        return IOLB_OK;
    });
}

int iolb_mx4_pack(const void* x, int64_t ldx, int64_t rows, int64_t cols, int dtype, uint8_t* codes, uint8_t* scales)
{
    return guarded([&] {
        const int rc = check_mx4(rows, cols, ldx, dtype, x, codes, scales);
        if (rc != IOLB_OK || rows == 0 || cols == 0) return rc;
        BLOCK_HIP(launch_mx4_pack(x, ldx, (int)rows, (int)cols, dtype, codes, scales, call_stream()));
        return IOLB_OK;
    });
}

int iolb_mx4_unpack(const uint8_t* codes, const uint8_t* scales, int64_t rows, int64_t cols, int dtype, void* y, int64_t ldy)
{
    return guarded([&] {
        const int rc = check_mx4(rows, cols, ldy, dtype, y, codes, scales);
        if (rc != IOLB_OK || rows == 0 || cols == 0) return rc;
        BLOCK_HIP(launch_mx4_unpack(codes, scales, (int)rows, (int)cols, dtype, y, ldy, call_stream()));
        return IOLB_OK;
    });
}

int iolb_linear_mx4_workspace_bytes(const iolb_linear_mx4_args* args, size_t* bytes) { return needed_bytes(args, bytes, check_linear, run_linear); }

int iolb_linear_mx4(const iolb_linear_mx4_args* args, void* workspace, size_t workspace_bytes)
{
    return checked_call(args, workspace, workspace_bytes, check_linear, run_linear);
}

}  // extern "C"
