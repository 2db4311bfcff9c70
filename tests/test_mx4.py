"""Microscaled 4-bit floating point and layers in it, against the definition in 64 bits.

Codes, scales and values are equal to the last bit.  Products of codes are exact; a sum of n of them in fp32 is within (n + 16) 2^-24 of its sum of
magnitudes, the rest as for the dense layers.
"""
import ctypes

import numpy as np
import pytest

from paper_2012_15667_amd import binding as B
from tests.test_dense import ACTS, HALF_ULP, TINY, TYPES, act64, assert_within, make, to64

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def _torch():
    import torch
    return torch


def pack64(x):
    """(codes, scales) of the definition: by the nearest level, ties to the even code."""
    rows, cols = x.shape
    wide = -(-cols // 128) * 128
    v = np.zeros((rows, wide))
    v[:, :cols] = x
    v = v.reshape(rows, -1, 32)
    with np.errstate(invalid="ignore"):
        most = np.abs(v).max(2)
    bad = ~np.isfinite(v).all(2)
    s = np.zeros(most.shape, dtype=int)
    for at in range(255):
        s[(np.where(bad, 0, most) > 7 * 2.0 ** (at - 127)) & (s == at)] = at + 1
    u = np.where(bad[:, :, None], 0, v) / 2.0 ** (s - 127.0)[:, :, None]
    a = np.abs(u)[..., None]
    middles = (LEVELS[1:] + LEVELS[:-1]) / 2
    code = ((a > middles) | ((a == middles) & (np.arange(7) % 2 == 1))).sum(-1)
    code = np.where(bad[:, :, None], 0, code | np.where(np.signbit(u), 8, 0)).reshape(rows, -1)
    return (code[:, 0::2] + 16 * code[:, 1::2]).astype(np.uint8), np.where(bad, 255, s).astype(np.uint8)


def values64(codes, scales, cols):
    code = np.stack([codes & 15, codes >> 4], 2).reshape(codes.shape[0], -1).astype(int)
    v = np.where(code & 8, -1, 1) * LEVELS[code & 7] * 2.0 ** (np.repeat(scales.astype(int), 32, 1) - 127.0)
    return np.where(np.repeat(scales == 255, 32, 1), np.nan, v)[:, :cols]


def arrays(c):
    return c.codes.cpu().numpy(), c.scales.cpu().numpy()


def hard_values(rng, rows, cols, dtype):
    """Blocks of all magnitudes, borders between levels and scales, zeros of both signs, values that are not finite."""
    torch = _torch()
    lo, hi = (-24, 15) if dtype == "float16" else (-149, 127)
    unit = 2.0 ** rng.integers(lo, hi - 3, (rows, -(-cols // 32))).astype(float)
    unit = np.repeat(unit, 32, 1)[:, :cols]
    v = rng.standard_normal((rows, cols)) * unit
    pick = rng.random((rows, cols))
    borders = np.array([0.25, 0.5, 0.75, 1.25, 1.75, 2.5, 3.5, 5, 6, 7, 7.25, 3.75, -0.0, -0.25, -5, -7])
    v = np.where(pick < 0.4, borders[rng.integers(0, len(borders), (rows, cols))] * unit, v)
    v[pick > 0.999] = np.inf
    v[(pick > 0.998) & (pick < 0.999)] = np.nan
    if rows > 4:
        v[0] = 0
        v[1] = -0.0
        v[2] = torch.finfo(getattr(torch, dtype)).max
        v[3] = -np.inf
        v[4] = np.nan
    with np.errstate(over="ignore"):
        return torch.from_numpy(v.astype(np.float32)).to(getattr(torch, dtype))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,gap", [(1, 1, 0), (1, 32, 0), (7, 31, 0), (40, 33, 3), (70, 128, 0), (300, 129, 8), (5, 4100, 0), (3, 2056, 1), (64, 1000, 0)])
def test_codes_scales_and_values(dtype, rows, cols, gap):
    torch = _torch()
    rng = np.random.default_rng(cols)
    wide = hard_values(rng, rows, cols + gap, dtype).cuda()
    x = wide[:, :cols]
    c = B.mx4_pack(x)
    codes, scales = arrays(c)
    want_codes, want_scales = pack64(to64(x))
    assert c.cols == cols and np.array_equal(scales, want_scales)
    assert np.array_equal(codes, want_codes)
    top = float(torch.finfo(x.dtype).max)
    for read in TYPES:
        T = getattr(torch, read)
        with np.errstate(invalid="ignore", over="ignore"):
            want = values64(codes, scales, cols)
            limit = float(torch.finfo(T).max)
            want = torch.from_numpy(np.where(np.isnan(want), want, np.clip(want, -limit, limit))).to(T)
        got = B.mx4_unpack(c, T).cpu()
        assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.equal(got.nan_to_num(nan=0.0), want.nan_to_num(nan=0.0)), read
    del top


@pytest.mark.gpu
def test_nothing_is_off_by_more_than_half_a_step():
    """Below 1 of the unit 0.25, below 4 half a unit, up to 7 one unit."""
    rng = np.random.default_rng(2)
    x, x64 = make(rng, (200, 320), "float32")
    c = B.mx4_pack(x)
    unit = 2.0 ** (np.repeat(c.scales.cpu().numpy().astype(int), 32, 1)[:, :320] - 127.0)
    a, off = np.abs(x64) / unit, np.abs(to64(B.mx4_unpack(c)) - x64) / unit
    assert a.max() <= 7 and np.all(off <= np.where(a < 2, 0.25, np.where(a < 4, 0.5, 1.0)))
    most = np.abs(x64).reshape(200, 10, 32).max(2)
    assert np.all(most > 3.5 * unit[:, ::32][:, :10])


@pytest.mark.gpu
def test_unpack_into_rows_of_a_wider_tensor_and_offsets_beyond_32_bits():
    torch = _torch()
    rng = np.random.default_rng(4)
    x, _ = make(rng, (30, 75), "bfloat16")
    c = B.mx4_pack(x)
    wide = torch.full((30, 90), 7.0, dtype=torch.bfloat16, device="cuda")
    B.mx4_unpack(c, y=wide[:, 9:84])
    assert torch.equal(wide[:, 9:84], B.mx4_unpack(c, torch.bfloat16)) and bool((wide[:, :9] == 7).all()) and bool((wide[:, 84:] == 7).all())
    rows, gap = 1100, 1 << 21
    big = torch.empty(rows * gap, dtype=torch.bfloat16, device="cuda").view(rows, gap)
    x, _ = make(rng, (rows, 64), "bfloat16")
    far = big[:, 128:192]
    far.copy_(x)
    a, b = B.mx4_pack(far), B.mx4_pack(x)
    assert torch.equal(a.codes, b.codes) and torch.equal(a.scales, b.scales)
    w = B.mx4_pack(make(rng, (40, 64), "bfloat16")[0])
    y = big[:, 256:296]
    B.linear_mx4(far, w, y=y)
    assert torch.equal(y, B.linear_mx4(x, w))
    # codes beyond 2^31 bytes: rows at the end of a tall operand
    tall = torch.zeros((36000, 65536), dtype=torch.uint8, device="cuda")
    scales = torch.full((36000, 4096), 127, dtype=torch.uint8, device="cuda")
    few = B.mx4_pack(make(rng, (40, 131072), "bfloat16")[0])
    tall[-40:] = few.codes
    scales[-40:] = few.scales
    y = B.mx4_pack(make(rng, (3, 131072), "bfloat16")[0])
    whole = B.linear_mx4(y, B.Mx4(tall, scales, 131072), dtype=torch.float32)
    assert torch.equal(whole[:, -40:], B.linear_mx4(y, few, dtype=torch.float32)) and bool((whole[:, :-40] == 0).all())
    whole = B.linear_mx4(B.Mx4(tall, scales, 131072), y, dtype=torch.float32)
    assert bool((whole[:-40] == 0).all())
    want = values64(*arrays(few), 131072) @ values64(*arrays(y), 131072).T
    total = np.abs(values64(*arrays(few), 131072)) @ np.abs(values64(*arrays(y), 131072)).T
    assert_within(whole[-40:], want, 131088 * 2.0 ** -24 * total)


def check_linear(rng, M, N, K, dtype, act="none", bias=True, residual=None, gap=0, lead=0, packed=False):
    torch = _torch()

    def wide(rows, cols):
        return make(rng, (rows, cols + gap + lead), dtype)[0][:, lead:lead + cols]
    x = wide(M, K)
    w = B.mx4_pack(make(rng, (N, K), "float32", max(K, 1) ** -0.5)[0])
    b = make(rng, (N,), dtype)[0] if bias else None
    r = wide(M, N) if residual else None
    x4 = B.mx4_pack(x)
    xv, wv = values64(*arrays(x4), K), values64(*arrays(w), K)
    z, total = xv @ wv.T, np.abs(xv) @ np.abs(wv).T
    if bias:
        z, total = z + to64(b), total + np.abs(to64(b))
    if residual == "first":
        z, total = z + to64(r), total + np.abs(to64(r))
    y = act64(z, act)
    if residual == "after":
        y = y + to64(r)
    got = B.linear_mx4(x4 if packed else x, w, b, act=act, residual=r, residual_first=residual == "first", dtype=getattr(torch, dtype) if packed else None)
    bound = 1.13 * (K + 16) * 2.0 ** -24 * total + (0 if act in ("none", "relu") else 1e-6 * np.abs(z) + 1e-7)
    if residual == "after":
        bound = bound + 2.0 ** -24 * (np.abs(y) + np.abs(to64(r)))
    assert_within(got, y, bound + HALF_ULP[dtype] * (np.abs(y) + bound) + TINY[dtype])
    return got


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("packed", [False, True])
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 64, 64), (1, 1000, 512), (2, 7, 5), (3, 33, 40), (5, 100, 257), (16, 48, 96), (17, 130, 129), (33, 70, 500), (20, 200, 4000), (64, 100, 2100), (64, 128, 1000),
                                   (65, 129, 65), (100, 260, 200), (129, 257, 384), (200, 40, 1030), (300, 520, 136)])
def test_linear_sizes(dtype, packed, M, N, K):
    check_linear(np.random.default_rng(M + 7 * N + K), M, N, K, dtype, packed=packed)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("residual", [None, "first", "after"])
@pytest.mark.parametrize("M", [3, 40, 150])
def test_linear_epilogue(dtype, act, residual, M):
    check_linear(np.random.default_rng(M), M, 68, 72, dtype, act=act, residual=residual, bias=residual != "after")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act,residual", [("none", None), ("relu", "first"), ("silu", "after"), ("gelu", "first"), ("gelu_tanh", "after")])
@pytest.mark.parametrize("M,N,K", [(1500, 1030, 200), (65, 129, 2500), (129, 257, 4103), (20, 70, 9000), (4100, 2050, 130)])
def test_linear_epilogue_of_large_products_and_of_long_sums(dtype, act, residual, M, N, K):
    """Beyond what the kernel for few rows takes: blocks of all sizes, K shared by workgroups, stages that end in the middle."""
    check_linear(np.random.default_rng(M), M, N, K, dtype, act=act, residual=residual, bias=residual != "after", gap=3 if act == "silu" else 0)


@pytest.mark.gpu
@pytest.mark.parametrize("M,K", [(1500, 200), (129, 4103), (1500, 256), (1500, 384), (1500, 520)])
def test_large_products_of_values_that_are_not_finite(M, K):
    """A NaN in the last block of a row, and scales at both ends of their range, reach their own rows and columns alone, also where a stage has one word of two."""
    torch = _torch()
    rng = np.random.default_rng(M)
    N = 1030
    x, w = make(rng, (M, K), "bfloat16")[0], make(rng, (N, K), "bfloat16")[0]
    clean = B.linear_mx4(x, B.mx4_pack(w), dtype=None)
    x[7, K - 1] = float("nan")
    w[1029, K - 1] = float("inf")
    x[8] = 0
    x[9] *= 2.0 ** -126
    got = B.linear_mx4(x, B.mx4_pack(w))
    assert bool(torch.isnan(got[7]).all()) and bool(torch.isnan(got[:, 1029]).all()) and bool((got[8, :1029] == 0).all())
    rest = torch.ones((M, N), dtype=torch.bool, device="cuda")
    rest[7:10], rest[:, 1029] = False, False
    assert torch.equal(got[rest], clean[rest])
    assert bool((got[9, :1029].float().abs() < 2.0 ** -110).all())


@pytest.mark.gpu
def test_tensors_larger_than_the_caches():
    """Rows of a large call and of a small one are the same to the last bit: packed, read back, multiplied."""
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    x = torch.randn((9001, 8200), generator=g, device="cuda").bfloat16()
    c = B.mx4_pack(x)
    y = B.mx4_unpack(c, torch.bfloat16)
    w = B.mx4_pack(torch.randn((9000, 200), generator=g, device="cuda"))
    z = B.linear_mx4(x[:, :200], w, act="silu")
    for at in (0, 4000, 8960):
        part = x[at:at + 41]
        few = B.mx4_pack(part)
        assert torch.equal(c.codes[at:at + 41], few.codes) and torch.equal(c.scales[at:at + 41], few.scales)
        assert torch.equal(y[at:at + 41], B.mx4_unpack(few, torch.bfloat16))
        off = (z[at:at + 41].float() - B.linear_mx4(part[:, :200], w, act="silu", dtype=None).float()).abs()
        # sums of 200 products in another order, each within 216 2^-24 of magnitudes that stay below 250 here, through a slope of at most 1.1: 7.1e-3; and a
        # rounding of half a unit in the last place each
        assert bool((off <= 2.0 ** -7 * z[at:at + 41].float().abs() + 2.0 ** -7).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap,lead", [(8, 0), (3, 0), (8, 8), (5, 1), (7, 9)])
@pytest.mark.parametrize("M,N,K", [(2, 40, 64), (70, 140, 128), (33, 20, 61)])
def test_linear_strides_and_alignment(dtype, gap, lead, M, N, K):
    check_linear(np.random.default_rng(gap), M, N, K, dtype, act="silu", residual="after", gap=gap, lead=lead)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_linear_blocks_of_all_sizes_and_long_sums(dtype):
    rng = np.random.default_rng(11)
    check_linear(rng, 4097, 3200, 96, dtype, act="relu")
    check_linear(rng, 2100, 1030, 1500, dtype, act="silu", residual="first")
    check_linear(rng, 130, 200, 9000, dtype, act="gelu_tanh")
    check_linear(rng, 30, 200, 20000, dtype)
    check_linear(rng, 1, 4100, 4097, dtype, act="gelu", residual="after")
    check_linear(rng, 8, 300, 25088, dtype)
    check_linear(rng, 700, 5, 7, dtype)
    check_linear(rng, 513, 130, 1000, dtype, residual="first", packed=True)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [1, 5, 16, 17, 31, 33, 64, 70, 400])
def test_linear_gives_the_same_for_a_tensor_and_for_its_codes(M):
    torch = _torch()
    rng = np.random.default_rng(M)
    for N, K in ((96, 300), (1000, 4096)):
        x, w = make(rng, (M, K), "bfloat16")[0], B.mx4_pack(make(rng, (N, K), "bfloat16")[0])
        a, b = B.linear_mx4(x, w), B.linear_mx4(B.mx4_pack(x), w)
        assert torch.equal(a, b) and a.dtype == torch.bfloat16 and torch.equal(B.linear_mx4(x, w), a)


@pytest.mark.gpu
@pytest.mark.parametrize("packed", [False, True])
def test_nothing_to_sum_for_many_rows(packed):
    torch = _torch()
    M, N = 33000, 70
    x, w = torch.empty((M, 0), dtype=torch.float32, device="cuda"), B.mx4_pack(torch.empty((N, 0), dtype=torch.float32, device="cuda"))
    b, b64 = make(np.random.default_rng(1), (N,), "float32")
    y = B.linear_mx4(B.mx4_pack(x) if packed else x, w, b, act="relu", dtype=torch.float32 if packed else None)
    assert_within(y, np.broadcast_to(np.maximum(b64, 0), (M, N)), np.zeros((M, N)))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(0, 5, 8), (5, 0, 8), (5, 40, 0), (0, 0, 0), (1, 3, 0), (600, 30, 0)])
def test_empty(dtype, M, N, K):
    torch = _torch()
    rng = np.random.default_rng(1)
    T = getattr(torch, dtype)
    x, w = torch.empty((M, K), dtype=T, device="cuda"), B.mx4_pack(torch.empty((N, K), dtype=T, device="cuda"))
    b, b64 = make(rng, (N,), dtype)
    r, r64 = make(rng, (M, N), dtype)
    for y in (B.linear_mx4(x, w, b, act="relu", residual=r), B.linear_mx4(B.mx4_pack(x), w, b, act="relu", residual=r, dtype=T)):
        assert_within(y, np.maximum(np.zeros((M, N)) + b64, 0) + r64, HALF_ULP[dtype] * 2 * (np.abs(b64) + np.abs(r64) + 1))
    assert B.mx4_unpack(w).shape == (N, K)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [1, 6, 30, 200])
def test_linear_of_values_that_are_not_finite(dtype, M):
    """A block that is not finite makes its row's sums NaN, and no other."""
    rng = np.random.default_rng(M)
    N, K = 70, 200
    x, _ = make(rng, (M, K), dtype)
    w, _ = make(rng, (N, K), dtype)
    clean = B.linear_mx4(x, B.mx4_pack(w))
    x[M // 2, 150] = float("inf")
    w[9, 3] = float("nan")
    got = to64(B.linear_mx4(x, B.mx4_pack(w)))
    assert np.isnan(got[M // 2]).all() and np.isnan(got[:, 9]).all()
    rest = np.ones((M, N), dtype=bool)
    rest[M // 2], rest[:, 9] = False, False
    assert np.array_equal(got[rest], to64(clean)[rest])


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 300, 500), (40, 96, 64), (600, 520, 520)])
def test_into_the_residual_and_into_rows_of_a_wider_tensor(M, N, K):
    torch = _torch()
    rng = np.random.default_rng(4)
    x, r = make(rng, (M, K), "bfloat16")[0], make(rng, (M, N), "bfloat16")[0]
    w = B.mx4_pack(make(rng, (N, K), "bfloat16")[0])
    want = B.linear_mx4(x, w, residual=r)
    wide = torch.full((M + 2, N + 24), 7.0, dtype=torch.bfloat16, device="cuda")
    B.linear_mx4(x, w, residual=r, y=wide[1:-1, 8:8 + N])
    assert torch.equal(wide[1:-1, 8:8 + N], want)
    wide[1:-1, 8:8 + N] = 7
    assert bool((wide == 7).all())
    assert B.linear_mx4(x, w, residual=r, y=r) is r and torch.equal(r, want)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(1, 1000, 4096), (12, 200, 900), (70, 200, 9000), (700, 300, 500)])
def test_other_streams_and_graphs(M, N, K):
    torch = _torch()
    rng = np.random.default_rng(M)
    x, w = make(rng, (M, K), "bfloat16")[0], make(rng, (N, K), "bfloat16")[0]
    w4 = B.mx4_pack(w)

    def both():
        return B.linear_mx4(x, w4, act="gelu"), B.mx4_unpack(B.mx4_pack(x))
    want = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = both()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    graphs, held = [], []
    for _ in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            held.append(both())
    for turn in range(3):
        x.copy_(make(rng, (M, K), "bfloat16")[0])
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        want = both()
        assert all(torch.equal(a, b) for h in held for a, b in zip(want, h)), turn


@pytest.mark.gpu
def test_a_backward_pass_through_the_result_is_refused():
    torch = _torch()
    x = torch.ones((4, 64), device="cuda", requires_grad=True)
    w = B.mx4_pack(torch.ones((8, 64), device="cuda"))
    with pytest.raises(RuntimeError, match="linear_mx4"):
        B.linear_mx4(x, w).sum().backward()
    with torch.no_grad():
        assert not B.linear_mx4(x, w).requires_grad


# ---- refusals ---------------------------------------------------------------------------------------------

P = 4096


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), -1), (dict(N=-1), -1), (dict(K=-1), -1), (dict(M=1 << 31), -2), (dict(N=1 << 31), -2), (dict(K=1 << 23), -2), (dict(dtype=3), -2), (dict(act=5), -2),
    (dict(x=None), -1), (dict(x_codes=P, x_scales=P), -1), (dict(x=None, x_codes=P), -1), (dict(x=None, x_codes=P + 8, x_scales=P), -1), (dict(x=None, x_codes=P, x_scales=P + 2), -1),
    (dict(w_codes=None), -1), (dict(w_scales=None), -1), (dict(w_codes=P + 8), -1), (dict(w_scales=P + 1), -1), (dict(y=None), -1), (dict(ldx=2999), -1), (dict(ldy=7), -1),
    (dict(residual=P, ldr=7), -1), (dict(x=P + 2), -1), (dict(y=P + 1), -1), (dict(M=1 << 30, N=1 << 30, ldy=1 << 30), -2), ({}, -4)])
def test_c_linear_refuses_without_touching_the_gpu(change, code):
    a = dict(M=100, N=8, K=3000, dtype=0, act=0, residual_first=0, x=P, ldx=3000, x_codes=None, x_scales=None, w_codes=P, w_scales=P, bias=None, residual=None, y=P, ldr=8, ldy=8)
    a.update(change)
    args = B.LinearMx4Args(*[a[n] for n, _ in B.LinearMx4Args._fields_])
    assert B.lib().iolb_linear_mx4(ctypes.byref(args), None, 0) == code
    need = ctypes.c_size_t(0)
    assert B.lib().iolb_linear_mx4_workspace_bytes(ctypes.byref(args), ctypes.byref(need)) == (code if code != -4 else 0)
    if code == -4:
        assert need.value > 0 and B.lib().iolb_linear_mx4(ctypes.byref(args), P, need.value - 1) == -4
        assert B.lib().iolb_linear_mx4(ctypes.byref(args), P + 128, need.value) == -4
    assert B.lib().iolb_linear_mx4(None, None, 0) == -1


@pytest.mark.parametrize("x,ld,rows,cols,dtype,codes,scales,code", [
    (None, 8, 2, 8, 0, P, P, -1), (P, 8, -1, 8, 0, P, P, -1), (P, 8, 2, -8, 0, P, P, -1), (P, 7, 2, 8, 0, P, P, -1), (P, 8, 2, 8, 5, P, P, -2),
    (P, 8, 1 << 31, 8, 0, P, P, -2), (P, 8, 2, 8, 0, P + 4, P, -1), (P, 8, 2, 8, 0, P, P + 1, -1), (P + 1, 8, 2, 8, 1, P, P, -1), (P, 8, 2, 8, 0, None, P, -1), (P, 8, 2, 8, 0, P, None, -1)])
def test_c_pack_and_unpack_refuse_without_touching_the_gpu(x, ld, rows, cols, dtype, codes, scales, code):
    assert B.lib().iolb_mx4_pack(x, ld, rows, cols, dtype, codes, scales) == code
    assert B.lib().iolb_mx4_unpack(codes, scales, rows, cols, dtype, x, ld) == code


@pytest.mark.gpu
def test_python_refusals():
    torch = _torch()
    x = torch.zeros((4, 64), device="cuda")
    w = B.mx4_pack(torch.zeros((8, 64), device="cuda"))
    b = torch.zeros((8,), device="cuda")
    for error, call in (
            (TypeError, lambda: B.linear_mx4(x, x)), (TypeError, lambda: B.linear_mx4(3, w)), (ValueError, lambda: B.linear_mx4(x[:, :32], w)), (TypeError, lambda: B.linear_mx4(x, w, b.half())),
            (ValueError, lambda: B.linear_mx4(x, w, b[:4])), (ValueError, lambda: B.linear_mx4(x, w, act="tanh")), (ValueError, lambda: B.linear_mx4(x, w, dtype=torch.float16)),
            (TypeError, lambda: B.linear_mx4(x.double(), w)), (TypeError, lambda: B.mx4_pack(x.cpu())), (TypeError, lambda: B.mx4_unpack(x)), (TypeError, lambda: B.mx4_unpack(w, torch.int8)),
            (ValueError, lambda: B.mx4_unpack(B.Mx4(w.codes, w.scales, 300))), (ValueError, lambda: B.mx4_unpack(B.Mx4(w.codes, w.scales[:4], 64))),
            (TypeError, lambda: B.mx4_unpack(B.Mx4(w.codes, w.scales.to(torch.int8), 64))), (TypeError, lambda: B.mx4_unpack(B.Mx4(w.codes, w.scales, 64.0))),
            (ValueError, lambda: B.linear_mx4(x, w, residual=x)), (ValueError, lambda: B.linear_mx4(x, w, y=x))):
        with pytest.raises(error):
            call()


def test_python_refuses_cpu_tensors():
    torch = _torch()
    c = B.Mx4(torch.zeros((4, 64), dtype=torch.uint8), torch.zeros((4, 4), dtype=torch.uint8), 64)
    for call in (lambda: B.mx4_unpack(c), lambda: B.linear_mx4(c, c), lambda: B.mx4_pack(torch.zeros((4, 4)))):
        with pytest.raises(TypeError):
            call()
