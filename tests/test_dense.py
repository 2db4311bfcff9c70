"""Dense layers, 8-bit activation checkpoints and the layers' gradients against the formulas in 64 bits.

Bounds, element by element, before anything was run.  u: half a unit in the last place of the output's type (2^-p for p significant bits:
24, fp16 11, bf16 8; fp16 has 2^-25 below its normal range).  A sum of n products in fp32 is within (n + 16) 2^-24 of the sum
of magnitudes (the parts of an fp32 operand add 3 2^-24 to it: inside the 16).  The activations' formulas hold to 1e-6 |z| + 1e-7,
their slopes to 4e-6; no slope exceeds 1.13.
"""
import ctypes

import numpy as np
import pytest

from paper_2012_15667_amd import binding as B

ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]
TYPES = ["float32", "float16", "bfloat16"]
HALF_ULP = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}
TINY = {"float32": 2.0 ** -149, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -133}


def _torch():
    import torch
    return torch


def _phi(z):
    from scipy.special import ndtr
    return ndtr(z)


def act64(z, name):
    from scipy.special import expit
    with np.errstate(all="ignore"):
        if name == "relu":
            return np.where(z <= 0, 0.0, z)
        if name == "silu":
            y = z * expit(z)
        elif name == "gelu":
            y = z * _phi(z)
        elif name == "gelu_tanh":
            y = z * expit(2 * np.sqrt(2 / np.pi) * (z + 0.044715 * z ** 3))
        else:
            return z
    return np.where(z == -np.inf, 0.0, y)


def slope64(z, name):
    from scipy.special import expit
    if name == "none":
        return np.ones_like(z)
    if name == "relu":
        return (z > 0).astype(float)
    z = np.clip(z, -1e3, 1e3)
    if name == "silu":
        s = expit(z)
        return s * (1 + z * (1 - s))
    if name == "gelu":
        return _phi(z) + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    k = 2 * np.sqrt(2 / np.pi)
    s = expit(k * (z + 0.044715 * z ** 3))
    return s + z * s * (1 - s) * k * (1 + 3 * 0.044715 * z * z)


def pack64(x, dtype):
    """(q, e) of the checkpoint's definition, block by block."""
    lo, hi = (-24, 10) if dtype == "float16" else (-126, 122)
    rows, cols = x.shape
    q = np.zeros((rows, cols), dtype=np.int8)
    e = np.zeros((rows, -(-cols // 32)), dtype=np.uint8)
    for r in range(rows):
        for b in range(e.shape[1]):
            v = x[r, 32 * b:32 * b + 32]
            fine = np.isfinite(v)
            most = np.max(np.abs(v[fine]), initial=0.0)
            ex = lo
            while ex < hi and 127 * 2.0 ** ex < most:
                ex += 1
            top = 63 if ex == hi else 127
            code = np.clip(np.rint(np.where(fine, v, 0) / 2.0 ** ex), -top, top)
            q[r, 32 * b:32 * b + 32] = np.where(fine, code, -128)
            e[r, b] = ex + 127
    return q, e


def values64(q, e):
    v = q.astype(np.float64) * 2.0 ** (np.repeat(e.astype(int), 32, axis=1)[:, :q.shape[1]] - 127.0)
    return np.where(q == -128, np.nan, v)


def to64(t):
    return t.detach().double().cpu().numpy()


def make(rng, shape, dtype, scale=1.0):
    """A GPU tensor of the type and its values in 64 bits."""
    torch = _torch()
    t = torch.from_numpy((rng.standard_normal(shape) * scale).astype(np.float32)).to(getattr(torch, dtype)).cuda()
    return t, to64(t)


def assert_within(got, want, bound):
    got = to64(got)
    assert got.shape == want.shape
    finite = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    assert np.array_equal(got[~finite & ~np.isnan(want)], want[~finite & ~np.isnan(want)])
    off = np.abs(got - want)[finite] - (bound + np.zeros_like(want))[finite]
    assert off.size == 0 or off.max() <= 0, off.max()


def check_linear(rng, M, N, K, dtype, act="none", bias=True, residual=None, checkpoint=False, gap=0, lead=0):
    torch = _torch()

    def wide(rows, cols):
        t, _ = make(rng, (rows, cols + gap + lead), dtype, 1.0)
        return t[:, lead:lead + cols]

    x, w = wide(M, K), wide(N, K)
    w *= 1.0 / max(K, 1) ** 0.5
    x64, w64 = to64(x), to64(w)
    b = make(rng, (N,), dtype)[0] if bias else None
    r = wide(M, N) if residual else None
    z = x64 @ w64.T
    total = np.abs(x64) @ np.abs(w64).T
    if bias:
        z, total = z + to64(b), total + np.abs(to64(b))
    if residual == "first":
        z, total = z + to64(r), total + np.abs(to64(r))
    y = act64(z, act)
    if residual == "after":
        y = y + to64(r)
    off_z = (K + 16) * 2.0 ** -24 * total
    got = B.linear(x, w, b, act=act, residual=r, residual_first=residual == "first", checkpoint=checkpoint)
    if checkpoint:
        got, c = got
        torch.cuda.synchronize()
        q, e = c.q.cpu().numpy(), c.e.cpu().numpy()
        unit = 2.0 ** (np.repeat(e.astype(int), 32, axis=1)[:, :N] - 127.0)
        assert np.all(np.abs(values64(q, e) - z) <= unit / 2 + off_z)
        for n in range(0, N, 32):
            most = np.abs(z[:, n:n + 32]).max(axis=1)
            slack = off_z[:, n:n + 32].max(axis=1)
            u = unit[:, n]
            assert np.all(most <= 127 * u + slack)
            assert np.all((most >= 63.5 * u - slack) | (u == 2.0 ** (-24 if dtype == "float16" else -126)))
    u = HALF_ULP[dtype]
    bound = 1.13 * off_z + (0 if act in ("none", "relu") else 1e-6 * np.abs(z) + 1e-7)
    if residual == "after":
        bound = bound + 2.0 ** -24 * (np.abs(y) + np.abs(to64(r)))
    assert_within(got, y, bound + u * (np.abs(y) + bound) + TINY[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 64, 64), (1, 1000, 512), (2, 7, 5), (3, 33, 40), (5, 100, 257), (16, 48, 96), (17, 130, 72),
                                   (64, 128, 1000), (65, 129, 65), (100, 260, 200), (129, 257, 64), (200, 40, 1030),
                                   (300, 520, 136)])
def test_linear_sizes(dtype, M, N, K):
    check_linear(np.random.default_rng(M + 7 * N + K), M, N, K, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("residual", [None, "first", "after"])
@pytest.mark.parametrize("M", [3, 40, 150])
def test_linear_epilogue(dtype, act, residual, M):
    check_linear(np.random.default_rng(M), M, 68, 72, dtype, act=act, residual=residual, bias=residual != "after")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 32, 64), (2, 5, 16), (20, 33, 64), (70, 100, 128), (150, 257, 72)])
def test_linear_checkpoint_from_the_epilogue(dtype, M, N, K):
    check_linear(np.random.default_rng(N), M, N, K, dtype, act="gelu", residual="first", checkpoint=True)


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
    check_linear(rng, 4097, 3200, 96, dtype, act="relu")              # the largest blocks, ragged
    check_linear(rng, 130, 200, 9000, dtype, act="gelu_tanh")         # K shared by workgroups
    check_linear(rng, 30, 200, 20000, dtype, checkpoint=True)
    check_linear(rng, 513, 130, 1000, dtype, act="silu", residual="first", checkpoint=True)
    check_linear(rng, 2200, 1000, 4600, dtype, act="relu", residual="after", checkpoint=True, gap=3)
    check_linear(rng, 700, 5, 7, dtype)
    check_linear(rng, 700, 300, 3, dtype, checkpoint=True)


@pytest.mark.gpu
def test_linear_fp32_is_as_precise_as_fp32_sums():
    """Relative 2-norm error of sums of 4096 products: fp32 rounding of a random walk is below sqrt(4096) 2^-24 = 3.8e-6."""
    rng = np.random.default_rng(2)
    for M in (4, 50, 500):
        x, x64 = make(rng, (M, 4096), "float32")
        w, w64 = make(rng, (300, 4096), "float32")
        got, want = to64(B.linear(x, w)), x64 @ w64.T
        assert np.linalg.norm(got - want) <= 3.8e-6 * np.linalg.norm(want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(0, 5, 8), (5, 0, 8), (5, 40, 0), (0, 0, 0), (1, 3, 0)])
def test_linear_empty(dtype, M, N, K):
    torch = _torch()
    rng = np.random.default_rng(1)
    T = getattr(torch, dtype)
    x, w = torch.empty((M, K), dtype=T, device="cuda"), torch.empty((N, K), dtype=T, device="cuda")
    b, b64 = make(rng, (N,), dtype)
    r, r64 = make(rng, (M, N), dtype)
    y, c = B.linear(x, w, b, act="relu", residual=r, checkpoint=True)
    assert y.shape == (M, N)
    assert_within(y, np.maximum(np.zeros((M, N)) + b64, 0) + r64, HALF_ULP[dtype] * 2 * (np.abs(b64) + np.abs(r64) + 1))
    assert c.q.shape == (M, N)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [2, 30, 140, 600])
def test_linear_of_values_that_are_not_finite(dtype, M):
    """Infinities and NaN go where the formula takes them and nowhere else; 0 inf is NaN; the largest finite values stay finite."""
    torch = _torch()
    rng = np.random.default_rng(M)
    N, K = 70, 72
    x, _ = make(rng, (M, K), dtype)
    w, _ = make(rng, (N, K), dtype)
    w[:, 5] = torch.where(torch.arange(N, device="cuda") % 3 == 0, 0.0, 1.5).to(w.dtype)
    w[7, 6] = -1.0
    x[0, 5] = float("inf")
    x[1, 6] = float("nan")
    w[9, 40] = float("-inf")
    x[1, 40] = 2.0
    with np.errstate(all="ignore"):
        want = to64(x) @ to64(w).T
    # numpy's product may stop at NaN in another way: the rows and columns without one are compared in full
    got = to64(B.linear(x, w))
    assert np.isnan(got[0, 0]) and np.isnan(got[0, 3]) and np.isnan(got[1]).all()
    n = np.arange(N)
    assert np.all(got[0, (n % 3 != 0) & (n != 9)] == np.inf)
    clean = np.ones((M, N), dtype=bool)
    clean[:2] = False
    clean[:, 9] = False
    total = np.abs(np.where(np.isfinite(to64(x)), to64(x), 0)) @ np.abs(np.where(np.isfinite(to64(w)), to64(w), 0)).T
    off = np.abs(got[clean] - want[clean])
    assert off.size == 0 or np.all(off <= ((K + 16) * 2.0 ** -24 * total + HALF_ULP[dtype] * 2 * (np.abs(want) + 1))[clean])
    assert np.all(np.isinf(got[2:, 9]) | np.isnan(got[2:, 9]))
    top = torch.finfo(x.dtype).max
    big = torch.full((M, 8), top, dtype=x.dtype, device="cuda")
    one = torch.zeros((N, 8), dtype=x.dtype, device="cuda")
    one[:, 0] = 1.0
    assert bool((B.linear(big, one) == top).all())
    low = torch.full((M, N), -top, dtype=x.dtype, device="cuda")         # a residual of the type's lowest value, as a mask would be
    y = B.linear(torch.zeros_like(big), one, residual=low, residual_first=True, act="gelu")
    assert bool((y == 0).all())
    y = B.linear(torch.zeros_like(big), one, residual=low * float("inf"), residual_first=True, act="silu")
    assert bool((y == 0).all())


@pytest.mark.gpu
def test_linear_into_the_residual_and_into_rows_of_a_wider_tensor():
    torch = _torch()
    rng = np.random.default_rng(4)
    x, _ = make(rng, (70, 64), "bfloat16")
    w, _ = make(rng, (96, 64), "bfloat16")
    r, _ = make(rng, (70, 96), "bfloat16")
    want = B.linear(x, w, residual=r)
    wide = torch.full((70, 120), 7.0, dtype=torch.bfloat16, device="cuda")
    B.linear(x, w, residual=r, y=wide[:, 8:104])
    assert torch.equal(wide[:, 8:104], want) and bool((wide[:, :8] == 7).all()) and bool((wide[:, 104:] == 7).all())
    assert B.linear(x, w, residual=r, y=r) is r and torch.equal(r, want)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    """Rows 2^21 values apart: the last ones start beyond 2^31 values."""
    torch = _torch()
    rng = np.random.default_rng(6)
    rows, gap = 1100, 1 << 21
    big = torch.empty(rows * gap, dtype=torch.bfloat16, device="cuda").view(rows, gap)
    x = big[:, 128:192]
    x.copy_(make(rng, (rows, 64), "bfloat16")[0])
    w, _ = make(rng, (40, 64), "bfloat16")
    want = B.linear(x.contiguous(), w)
    y = big[:, 256:296]
    B.linear(x, w, y=y)
    assert torch.equal(y, want)
    assert torch.equal(B.linear(w, x), B.linear(w, x.contiguous()))
    a, b = B.checkpoint_pack(x), B.checkpoint_pack(x.contiguous())
    assert torch.equal(a.q, b.q) and torch.equal(a.e, b.e)


# ---- checkpoints ------------------------------------------------------------------------------------------

def hard_values(rng, rows, cols, dtype):
    """Blocks of all scales: subnormal to the type's largest, zeros, powers of two and their neighbours, ties, NaN, infinities."""
    torch = _torch()
    lo, hi = (-24, 16) if dtype == "float16" else (-149, 128)
    v = rng.standard_normal((rows, cols)) * 2.0 ** rng.integers(lo, hi, (rows, 1)).astype(float)
    v *= 2.0 ** -rng.integers(0, 12, (rows, cols)).astype(float)
    pick = rng.random((rows, cols))
    v[pick < 0.05] = 0
    v[(pick > 0.05) & (pick < 0.08)] = 63.5
    v[(pick > 0.08) & (pick < 0.10)] = 127.0
    v[(pick > 0.10) & (pick < 0.11)] = 126.5
    v[(pick > 0.11) & (pick < 0.115)] = np.inf
    v[(pick > 0.115) & (pick < 0.12)] = -np.inf
    v[(pick > 0.12) & (pick < 0.125)] = np.nan
    if rows > 4:
        v[0] = 0
        v[1] = np.nan
        v[2] = torch.finfo(getattr(torch, dtype)).max
        v[3] = -np.inf
    with np.errstate(over="ignore"):
        t = torch.from_numpy(v.astype(np.float32)).to(getattr(torch, dtype))
    return t


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,cols,gap", [(1, 1, 0), (1, 32, 0), (7, 31, 0), (40, 33, 3), (70, 100, 0), (300, 64, 8), (5, 4100, 0), (3, 2056, 1)])
def test_checkpoint_codes_and_values(dtype, rows, cols, gap):
    torch = _torch()
    t = hard_values(np.random.default_rng(rows + cols), rows, cols, dtype)
    wide = torch.empty((rows, cols + gap), dtype=t.dtype, device="cuda")
    wide[:, :cols] = t.cuda()
    c = B.checkpoint_pack(wide[:, :cols])
    q, e = pack64(to64(t), dtype)
    assert np.array_equal(c.q.cpu().numpy(), q) and np.array_equal(c.e.cpu().numpy(), e)
    want = values64(q, e)
    for out in TYPES if dtype != "float16" else ["float16", "float32", "bfloat16"]:
        if out == "float16" and dtype != "float16":
            continue                                              # another type's values may be beyond fp16
        assert_within(B.checkpoint_unpack(c, getattr(torch, out)), want, 0.0)
    y = torch.full((rows, cols + 5), 3.0, dtype=t.dtype, device="cuda")
    B.checkpoint_unpack(c, y=y[:, 2:2 + cols])
    assert_within(y[:, 2:2 + cols], want, 0.0)
    assert bool((y[:, :2] == 3).all()) and bool((y[:, 2 + cols:] == 3).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
def test_checkpoint_read_through_an_activation(dtype, act):
    rng = np.random.default_rng(3)
    t, _ = make(rng, (40, 100), dtype, 3.0)
    c = B.checkpoint_pack(t)
    v = values64(c.q.cpu().numpy(), c.e.cpu().numpy())
    want = act64(v, act)
    slack = 0 if act in ("none", "relu") else 1e-6 * np.abs(v) + 1e-7
    assert_within(B.checkpoint_unpack(c, getattr(_torch(), dtype), act=act), want, slack + HALF_ULP[dtype] * (np.abs(want) + slack) + TINY[dtype])


# ---- gradients ---------------------------------------------------------------------------------------------

def check_backward(rng, M, N, K, dtype, act="none", x_act="none", gap=0, **want):
    w = make(rng, (N, K + gap), dtype, 1.0 / max(K, 1) ** 0.5)[0][:, :K]
    dy = make(rng, (M, N + gap), dtype)[0][:, :N]
    x = B.checkpoint_pack(make(rng, (M, K), dtype)[0])
    z = B.checkpoint_pack(make(rng, (M, N), dtype, 2.0)[0])
    g = B.linear_backward(dy, w, x, z if act != "none" else None, act=act, x_act=x_act, want_dz=True, **want)
    x64 = act64(values64(x.q.cpu().numpy(), x.e.cpu().numpy()), x_act)
    z64 = values64(z.q.cpu().numpy(), z.e.cpu().numpy())
    dy64, w64 = to64(dy), to64(w)
    dz = dy64 * slope64(z64, act)
    u = HALF_ULP[dtype]
    smooth, smooth_x = act not in ("none", "relu"), x_act not in ("none", "relu")
    off = (4e-6 * np.abs(dy64) if smooth else 0 * dz)                          # of dz before it is rounded
    off_r = off + (u * (np.abs(dz) + off) + TINY[dtype] if smooth and dtype != "float32" else 0)
    off_x = (1e-6 * np.abs(x64) + 1e-7 + (u * np.abs(x64) + TINY[dtype] if dtype != "float32" else 0) if smooth_x else 0 * x64)

    def bound(a, da, b, db, n, want):
        s = (n + 16) * 2.0 ** -24 * (np.abs(a) @ np.abs(b)) + da @ (np.abs(b) + db) + np.abs(a) @ db
        return s + u * (np.abs(want) + s) + TINY[dtype]

    if g.dx is not None:
        dx = dz @ w64
        assert_within(g.dx, dx, bound(dz, off_r, w64, 0 * w64, N, dx))
    if g.dw is not None:
        dw = dz.T @ x64
        assert_within(g.dw, dw, bound(dz.T, off_r.T, x64, off_x, M, dw))
    if g.db is not None:
        db = dz.sum(0)
        s = (M + 16) * 2.0 ** -24 * np.abs(dz).sum(0) + off.sum(0)
        assert_within(g.db, db, s + u * (np.abs(db) + s) + TINY[dtype])
    assert_within(g.dz, dz, off + u * (np.abs(dz) + off) + TINY[dtype])
    return g


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 64, 64), (2, 7, 5), (3, 33, 40), (16, 48, 96), (17, 130, 72), (64, 128, 1000), (65, 129, 65),
                                   (100, 260, 200), (300, 40, 130), (1000, 72, 136)])
def test_backward_sizes(dtype, M, N, K):
    check_backward(np.random.default_rng(M + 7 * N + K), M, N, K, dtype, act="gelu")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("x_act", ["none", "relu", "silu"])
@pytest.mark.parametrize("M", [5, 70])
def test_backward_activations(dtype, act, x_act, M):
    check_backward(np.random.default_rng(M), M, 68, 72, dtype, act=act, x_act=x_act, gap=8 if M == 5 else 3)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dx,dw,db", [(True, False, False), (False, True, False), (False, False, True), (False, False, False)])
def test_backward_of_what_is_wanted_only(dtype, dx, dw, db):
    g = check_backward(np.random.default_rng(1), 20, 72, 40, dtype, act="relu", want_dx=dx, want_dw=dw, want_db=db)
    assert (g.dx is None, g.dw is None, g.db is None) == (not dx, not dw, not db)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_backward_blocks_of_all_sizes(dtype):
    rng = np.random.default_rng(8)
    check_backward(rng, 600, 77, 5, dtype, act="gelu", x_act="silu")
    check_backward(rng, 600, 5, 77, dtype, act="relu")
    check_backward(rng, 100, 2100, 2049, dtype, act="silu", gap=1)
    check_backward(rng, 33, 8, 2, dtype, act="gelu")
    check_backward(rng, 3200, 4097, 96, dtype, act="silu")
    check_backward(rng, 9000, 130, 70, dtype, act="gelu_tanh")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,K", [(0, 5, 8), (5, 0, 8), (5, 40, 0), (0, 0, 0)])
def test_backward_empty(dtype, M, N, K):
    torch = _torch()
    T = getattr(torch, dtype)
    c = B.checkpoint_pack(torch.zeros((M, K), dtype=T, device="cuda"))
    g = B.linear_backward(torch.ones((M, N), dtype=T, device="cuda"), torch.ones((N, K), dtype=T, device="cuda"), c, want_dz=True)
    assert g.dx.shape == (M, K) and g.dw.shape == (N, K) and g.db.shape == (N,)
    assert bool((g.dx == float(N)).all()) and bool((g.dw == 0).all()) and bool((g.db == float(M)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_backward_where_relu_stops_what_is_not_finite(dtype):
    """dy that relu stops is not looked at: infinities and NaN there leave every gradient as it is."""
    torch = _torch()
    rng = np.random.default_rng(5)
    dy, _ = make(rng, (70, 68), dtype)
    w, _ = make(rng, (68, 72), dtype)
    x, z = (B.checkpoint_pack(make(rng, s, dtype)[0]) for s in ((70, 72), (70, 68)))
    stopped = B.checkpoint_unpack(z) <= 0
    a = B.linear_backward(torch.where(stopped, 0.0, dy.float()).to(dy.dtype), w, x, z, act="relu")
    for bad in (float("nan"), float("inf"), float(torch.finfo(dy.dtype).min)):
        b = B.linear_backward(torch.where(stopped, bad, dy.float()).to(dy.dtype), w, x, z, act="relu")
        assert all(torch.equal(a[i], b[i]) for i in range(3))
    # and what it lets through goes on
    z.q[3, 4] = 127
    dy[3, 4] = float("inf")
    g = B.linear_backward(dy, w, x, z, act="relu")
    assert not bool(torch.isfinite(g.dx[3]).any()) and not bool(torch.isfinite(g.db[4])) and bool(torch.isfinite(g.dx[4]).all())


@pytest.mark.gpu
@pytest.mark.parametrize("act", ["silu", "gelu", "gelu_tanh"])
def test_gradients_against_differences(act):
    """Central differences of sum(linear * c) at checkpointed values, fp32.  The loss is formed in 64 bits from the operator's
    outputs, each within 2e-6 of its sum of magnitudes; a step of 2^-4 then leaves 2e-6 L / 2^-4 of noise (L: the loss's
    magnitudes) and (2^-4)^2 / 6 times a third derivative, below 2 for these activations."""
    torch = _torch()
    rng = np.random.default_rng(9)
    M, N, K = 4, 12, 8
    h = 2.0 ** -4
    x8 = B.checkpoint_pack(make(rng, (M, K), "float32")[0])
    x = B.checkpoint_unpack(x8)
    w, _ = make(rng, (N, K), "float32", 0.5)
    b, _ = make(rng, (N,), "float32")
    c, c64 = make(rng, (M, N), "float32")
    # z in full precision would be the derivative's own point: checkpoint z block by block at values it holds exactly
    y, z8 = B.linear(x, w, b, act=act, checkpoint=True)
    z_off = to64(B.linear(x, w, b)) - to64(B.checkpoint_unpack(z8))
    r = torch.from_numpy(-z_off.astype(np.float32)).cuda()              # shifts z onto its checkpoint
    g = B.linear_backward(c, w, x8, z8, act=act, want_dz=True)

    def loss(x, w, b, r):
        return float((to64(B.linear(x, w, b, act=act, residual=r, residual_first=True)) * c64).sum())

    magnitude = float((np.abs(c64) * (np.abs(to64(x)) @ np.abs(to64(w)).T + np.abs(to64(b)) + 1)).sum())
    for name, t, grad in (("dx", x, g.dx), ("dw", w, g.dw), ("db", b, g.db), ("dz", r, g.dz)):
        flat, gf = t.view(-1), to64(grad).reshape(-1)
        third = 2 * float(np.abs(c64).sum()) * max(1.0, float(np.abs(to64(x)).max()), float(np.abs(to64(w)).max())) ** 3
        for i in range(flat.numel()):
            keep = flat[i].item()
            flat[i] = keep + h
            up = loss(x, w, b, r)
            flat[i] = keep - h
            down = loss(x, w, b, r)
            flat[i] = keep
            assert abs((up - down) / (2 * h) - gf[i]) <= 2e-6 * magnitude / h + third * h * h / 6, (name, i)


# ---- streams, graphs, refusals -------------------------------------------------------------------------------

def _step(x, w, b, r):
    x8 = B.checkpoint_pack(x)
    y, z8 = B.linear(x, w, b, act="gelu", residual=r, checkpoint=True)
    g = B.linear_backward(y, w, x8, z8, act="gelu")
    return [y, z8.q, z8.e, x8.q, x8.e, g.dx, g.dw, g.db]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [3, 50, 260])
def test_other_streams_and_graphs(dtype, M):
    torch = _torch()
    rng = np.random.default_rng(7)
    x, w, b, r = (make(rng, s, dtype)[0] for s in ((M, 130), (200, 130), (200,), (M, 200)))
    want = _step(x, w, b, r)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = _step(x, w, b, r)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = _step(x, w, b, r)
    for i in range(3):
        x.copy_(make(rng, (M, 130), dtype)[0])
        want = _step(x, w, b, r)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want)), i


def test_c_calls_refuse_without_touching_the_gpu():
    """Codes of arguments that no launch follows (addresses here are never read)."""
    L = B.lib()
    need = ctypes.c_size_t(0)
    p = 4096

    def linear(**k):
        a = dict(M=4, N=8, K=16, dtype=0, act=0, residual_first=0, x=p, w=p, bias=None, residual=None, y=p, ldx=16, ldw=16, ldr=8, ldy=8,
                 zq=None, ze=None)
        a.update(k)
        return L.iolb_linear(ctypes.byref(B.LinearArgs(**a)), None, 0)

    assert L.iolb_linear(None, None, 0) == -1
    assert L.iolb_linear_workspace_bytes(None, ctypes.byref(need)) == -1
    for bad in (dict(M=-1), dict(N=-1), dict(K=-1), dict(x=None), dict(w=None), dict(y=None), dict(ldx=15), dict(ldw=15), dict(ldy=7),
                dict(residual=p, ldr=7), dict(zq=p), dict(ze=p), dict(x=p + 2), dict(y=p + 1)):
        assert linear(**bad) == -1, bad
    for bad in (dict(dtype=3), dict(dtype=-1), dict(act=5), dict(act=-1), dict(K=1 << 23, ldx=1 << 23, ldw=1 << 23), dict(M=1 << 31)):
        assert linear(**bad) == -2, bad
    assert linear(M=0, y=None) == 0 and linear(N=0, w=None) == 0
    assert linear(M=1000) == -4                                  # parts of fp32 operands need a workspace

    def back(**k):
        a = dict(M=4, N=8, K=16, dtype=2, act=1, x_act=0, dy=p, w=p, ldy=8, ldw=16, xq=p, xe=p, zq=p, ze=p, dx=p, dw=p, db=p, dz=None)
        a.update(k)
        return L.iolb_linear_backward(ctypes.byref(B.LinearBackwardArgs(**a)), None, 0)

    assert L.iolb_linear_backward(None, None, 0) == -1
    for bad in (dict(M=-1), dict(dy=None), dict(w=None), dict(xq=None), dict(zq=None, ze=None), dict(ze=None), dict(xq=None, xe=None),
                dict(ldy=7), dict(ldw=15), dict(dx=p + 1)):
        assert back(**bad) == -1, bad
    for bad in (dict(dtype=9), dict(act=9), dict(x_act=9), dict(M=1 << 23)):
        assert back(**bad) == -2, bad
    assert back(M=1000) == -4
    assert L.iolb_checkpoint_pack(None, 4, 4, 4, 0, p, p) == -1
    assert L.iolb_checkpoint_pack(p, 3, 4, 4, 0, p, p) == -1
    assert L.iolb_checkpoint_pack(p, 4, 4, 4, 7, p, p) == -2
    assert L.iolb_checkpoint_pack(p, 4, -4, 4, 0, p, p) == -1
    assert L.iolb_checkpoint_pack(None, 4, 0, 4, 0, None, None) == 0
    assert L.iolb_checkpoint_unpack(p, p, 4, 4, 9, 0, p, 4) == -2
    assert L.iolb_checkpoint_unpack(p, None, 4, 4, 0, 0, p, 4) == -1


def test_python_refuses_cpu_tensors_and_unknown_names():
    torch = _torch()
    x = torch.zeros((2, 4))
    with pytest.raises(TypeError):
        B.linear(x, x)
    with pytest.raises(TypeError):
        B.linear(x.double(), x.double())
    with pytest.raises(TypeError):
        B.checkpoint_pack(x)
    with pytest.raises(TypeError):
        B.linear(None, x)


@pytest.mark.gpu
def test_python_refusals():
    torch = _torch()
    x, w = torch.zeros((2, 8), device="cuda"), torch.zeros((4, 8), device="cuda")
    for bad, kind in ((lambda: B.linear(x, w.half()), TypeError), (lambda: B.linear(x, torch.zeros((4, 9), device="cuda")), ValueError),
                      (lambda: B.linear(x, w, act="tanh"), ValueError), (lambda: B.linear(x, w, x[0]), ValueError),
                      (lambda: B.linear(x, w, residual=x), ValueError), (lambda: B.linear(x.t().contiguous(), w), ValueError),
                      (lambda: B.linear(torch.zeros((8, 2), device="cuda").t(), w), TypeError), (lambda: B.linear(x[0], w), TypeError),
                      (lambda: B.linear(x[:1].expand(2, 8), w), TypeError), (lambda: B.linear(x, w, y=x), ValueError),
                      (lambda: B.linear_backward(torch.zeros((2, 4), device="cuda"), w), ValueError),
                      (lambda: B.linear_backward(torch.zeros((2, 4), device="cuda"), w, x), TypeError),
                      (lambda: B.linear_backward(torch.zeros((2, 4), device="cuda"), w, B.checkpoint_pack(w)), ValueError),
                      (lambda: B.linear_backward(torch.zeros((2, 4), device="cuda"), w, B.checkpoint_pack(x), act="relu"), ValueError),
                      (lambda: B.checkpoint_unpack(x), TypeError),
                      (lambda: B.checkpoint_unpack(B.checkpoint_pack(x), torch.float64), TypeError)):
        with pytest.raises(kind):
            bad()


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(100, 70, 72), (300, 260, 1000), (2100, 1030, 5000)])
def test_linear_fp32_rows_of_uneven_magnitude(M, N, K):
    """Rows whose values differ by many powers of two, in x and in w, at every scale of the type, with weights that are zero where
    the large ones are: every output keeps the bound of fp32 sums, (K + 16) 2^-24 of its own sum of magnitudes, or of what 2^-40 of a
    row's largest value amounts to in rows of ordinary spread (at most one in 64 of the non-zero values below 2^-20 of the largest)."""
    torch = _torch()
    rng = np.random.default_rng(K)
    x = rng.standard_normal((M, K))
    w = rng.standard_normal((N, K))
    x *= 2.0 ** rng.integers(-40, 40, (M, 1))                       # a scale for each row
    x[0] *= 1e-30
    x[1] *= 1e25
    x[2, 3] = 2.0 ** 70                                              # one value far beyond its row
    x[3, ::2] *= 2.0 ** -60
    x[4] = 0
    x[4, 5] = 3.0
    w[:, 3] = 0
    w[0] = 0
    w[0, 7] = 1.0                                                    # picks one value of x
    w[1, 1:] *= 2.0 ** -50
    x, w = (torch.from_numpy(v.astype(np.float32)).cuda() for v in (x, w))
    x64, w64 = to64(x), to64(w)
    want, total = x64 @ w64.T, np.abs(x64) @ np.abs(w64).T

    def marked(v):
        a = np.abs(v)
        return ((a > 0) & (a < 2.0 ** -20 * a.max(1)[:, None])).sum(1) > (a > 0).sum(1) // 64

    assert marked(x64)[2] and not marked(x64)[5]
    # below 2^-110 three bf16 parts hold a value to 2^-133
    tiny = 2.0 ** -132 * (np.abs(w64).sum(1)[None] + np.abs(x64).sum(1)[:, None])
    assert_within(B.linear(x, w), want, (K + 16) * 2.0 ** -24 * total + tiny + TINY["float32"])
    # the same without the rows that two parts do not hold
    even, kept = ~marked(x64), ~marked(w64)
    x, w = (t[torch.from_numpy(k).cuda()].contiguous() for t, k in ((x, even), (w, kept)))
    x64, w64, want, total = x64[even], w64[kept], want[even][:, kept], total[even][:, kept]
    loose = 2.0 ** -39 * (np.abs(x64).max(1)[:, None] * np.abs(w64).sum(1)[None] + np.abs(x64).sum(1)[:, None] * np.abs(w64).max(1)[None])
    assert_within(B.linear(x, w), want, (K + 16) * 2.0 ** -24 * total + loose + TINY["float32"])


@pytest.mark.gpu
def test_large_fp32_products_of_values_that_are_not_finite():
    """Two fp16 parts: infinities and NaN give what fp32 arithmetic gives in their rows and columns, and change nothing elsewhere."""
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.randn((2200, 4600), generator=g, device="cuda")
    w = torch.randn((1000, 4600), generator=g, device="cuda")
    w[:, 9] = torch.where(torch.arange(1000, device="cuda") % 2 == 0, 0.0, -2.0)
    clean = B.linear(x, w)
    x[5, 9] = float("inf")
    x[300, 77] = float("nan")
    w[44, 3] = float("-inf")
    y = B.linear(x, w)
    assert bool(torch.isnan(y[5, 0::2][torch.arange(500, device="cuda") != 22]).all()) and bool((y[5, 1::2] == float("-inf")).all())
    assert bool(torch.isnan(y[300]).all()) and bool(torch.isinf(y[6:300, 44]).all())
    rows = torch.ones(2200, dtype=torch.bool, device="cuda")
    rows[[5, 300]] = False
    columns = torch.ones(1000, dtype=torch.bool, device="cuda")
    columns[44] = False
    assert torch.equal(y[rows][:, columns], clean[rows][:, columns])
    # the largest finite values, and sums beyond the type
    x[:] = torch.finfo(torch.float32).max
    w[:] = 0
    w[:, 0] = 1
    w[3, 1] = 1
    y = B.linear(x, w)
    assert bool((y[:, :3] == x[0, 0]).all()) and bool((y[:, 3] == float("inf")).all())


@pytest.mark.gpu
def test_linear_fp32_of_some_hundred_rows():
    """65 to 512 rows with so many products that a wave takes two groups of columns: ragged extents, each epilogue, shared K."""
    rng = np.random.default_rng(21)
    check_linear(rng, 70, 8011, 7205, "float32", act="gelu", residual="first", checkpoint=True, gap=3)
    check_linear(rng, 129, 260, 120003, "float32", act="relu", residual="after")
    check_linear(rng, 511, 16001, 490, "float32", lead=1)


@pytest.mark.gpu
def test_linear_fp32_of_some_hundred_rows_not_finite():
    torch = _torch()
    x, w = torch.ones(100, 8008, device="cuda"), torch.ones(5001, 8008, device="cuda")
    w[1::2] = -1
    x[7, 8001] = float("inf")
    w[4990, 3] = float("nan")
    w[4999, 5] = float("-inf")
    x[9, 5] = 0
    y = B.linear(x, w)
    plain = torch.arange(5001, device="cuda")
    even, odd = plain % 2 == 0, plain % 2 == 1
    even[4990] = odd[4999] = False
    assert bool((y[7, even] == float("inf")).all()) and bool((y[7, odd] == float("-inf")).all())
    assert bool(torch.isnan(y[:, 4990]).all()) and bool(torch.isnan(y[9, 4999]))
    others = torch.arange(100, device="cuda")
    others = others[(others != 7) & (others != 9)]
    assert bool((y[others][:, 4999] == float("-inf")).all())
    assert bool((y[others][:, even] == 8008).all()) and bool((y[others][:, odd] == -8008).all())
    assert bool((y[9, even] == 8007).all())
