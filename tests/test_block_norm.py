"""Norms before and after a block with gate and residual scale, and their gradients, against the formulas in 64 bits.

Bounds, element by element, before anything was run.  u: half a unit in the last place of the type.  A row's sums run over at most N / 64 + 8 values
one after another (64 threads, eight values at a time, then a tree), longer ones in more threads: within e = (N / 64 + 16) 2^-24 of their sum of magnitudes.  So
1 / sqrt(mean square) is within e / 2 + 2^-23 of itself, a mean within e mean|v|, and a normalised value within 2 e (|hat| + mean|v| r).
"""
import ctypes

import numpy as np
import pytest

from paper_2012_15667_amd import binding as B
from tests.test_dense import HALF_ULP, TINY, TYPES, assert_within, make, to64

EPS = 1e-5
SIZES = [(1, 1), (3, 7), (1, 64), (5, 65), (70, 33), (4, 1001), (2, 4096), (130, 520), (3, 2056), (37, 264), (5, 8200), (2, 16384), (2, 20001)]


def _torch():
    import torch
    return torch


def hat64(v, kind):
    """(normalised, 1 / root, mean magnitude times that)"""
    if kind == "none":
        return v, np.ones((v.shape[0], 1)), np.zeros((v.shape[0], 1))
    c = v - v.mean(1, keepdims=True) if kind == "layer" else v
    r = 1 / np.sqrt((c * c).mean(1, keepdims=True) + np.float64(np.float32(EPS)))
    return c * r, r, np.abs(v).mean(1, keepdims=True) * r * (kind == "layer")


def affine64(hat, w, b):
    y = hat if w is None else hat * to64(w)
    return y if b is None else y + to64(b)


def rows_of_gate(gate, M):
    if gate is None:
        return np.ones((1, 1))
    g = to64(gate)
    return g[None] if g.ndim == 1 else np.repeat(g, M // g.shape[0], 0)


def tensors(rng, M, N, dtype, post, pre, gate, bias, gap, lead=0):
    def wide():
        return make(rng, (M, N + gap + lead), dtype)[0][:, lead:lead + N]

    def column(there, level):
        return (make(rng, (N,), dtype, 0.3)[0] + level).to(getattr(_torch(), dtype)) if there else None
    g = None
    if gate == "columns":
        g = make(rng, (N,), dtype)[0]
    elif gate:
        g = make(rng, (gate, N), dtype)[0]
    h = wide()
    h += 0.5
    return wide(), h, dict(post=post, pre=pre, gate=g, scale=0.75, eps=EPS,
                           post_weight=column(post != "none", 1.0), post_bias=column(post != "none" and bias, 0.0),
                           pre_weight=column(pre != "none", 1.0), pre_bias=column(pre != "none" and bias, 0.0))


def check_forward(rng, M, N, dtype, post, pre, gate, bias=True, gap=0, lead=0):
    x, h, k = tensors(rng, M, N, dtype, post, pre, gate, bias, gap, lead)
    u, e = HALF_ULP[dtype], (N / 64 + 16) * 2.0 ** -24
    got = B.block_norm(x, h, **k)
    hat, _, off_mean = hat64(to64(h), post)
    p = affine64(hat, k["post_weight"], k["post_bias"])
    g = rows_of_gate(k["gate"], M)
    want = 0.75 * to64(x) + g * p
    w = 1 if k["post_weight"] is None else np.abs(to64(k["post_weight"]))
    off = np.abs(g) * (w * 2 * e * (np.abs(hat) + off_mean) + 2.0 ** -22 * (np.abs(p) + w * np.abs(hat))) + 2.0 ** -22 * (np.abs(to64(x)) + np.abs(want))
    assert_within(got.x, want, off + u * (np.abs(want) + off) + TINY[dtype])
    if pre == "none":
        assert got.y is None
        return
    check_norm_alone(got.y, got.x, dtype, pre, k, e)


def check_norm_alone(y, x, dtype, pre, k, e):
    hat, _, off_mean = hat64(to64(x), pre)
    want = affine64(hat, k["pre_weight"], k["pre_bias"])
    w = 1 if k["pre_weight"] is None else np.abs(to64(k["pre_weight"]))
    off = w * 2 * e * (np.abs(hat) + off_mean) + 2.0 ** -22 * (np.abs(want) + w * np.abs(hat))
    assert_within(y, want, off + HALF_ULP[dtype] * (np.abs(want) + off) + TINY[dtype])


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_forward_sizes(dtype, M, N, kind):
    check_forward(np.random.default_rng(M + N), M, N, dtype, kind, kind, "columns")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("post,pre", [("none", "rms"), ("none", "layer"), ("rms", "none"), ("layer", "rms"), ("none", "none")])
@pytest.mark.parametrize("gate", [None, "columns", 1, 3, 12])
@pytest.mark.parametrize("bias", [False, True])
def test_forward_kinds(dtype, post, pre, gate, bias):
    check_forward(np.random.default_rng(5), 12, 328, dtype, post, pre, gate, bias)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap,lead", [(8, 0), (3, 0), (5, 1), (0, 7), (7, 9)])
@pytest.mark.parametrize("M,N", [(3, 40), (40, 1000), (9, 4097)])
def test_forward_strides_and_alignment(dtype, gap, lead, M, N):
    check_forward(np.random.default_rng(gap), M, N, dtype, "layer", "rms", "columns", True, gap, lead)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N", [(3000, 128), (2100, 2048), (1100, 4096), (1500, 1000)])
def test_forward_many_rows(M, N):
    check_forward(np.random.default_rng(M), M, N, "bfloat16", "rms", "layer", 4 if M % 4 == 0 else None)
    check_forward(np.random.default_rng(M), M, N, "float32", "layer", "rms", None)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N", [(4, 100), (3, 4096), (2, 20001)])
def test_norm_alone_and_in_place(dtype, M, N):
    torch = _torch()
    rng = np.random.default_rng(3)
    x, h, k = tensors(rng, M, N, dtype, "rms", "layer", None, True, 0)
    alone = B.block_norm(x, pre="layer", pre_weight=k["pre_weight"], pre_bias=k["pre_bias"], eps=EPS)
    assert alone.x is None
    check_norm_alone(alone.y, x, dtype, "layer", k, (N / 64 + 16) * 2.0 ** -24)
    want = B.block_norm(x, h, **k)
    wide = torch.full((M, N + 24), 7.0, dtype=x.dtype, device="cuda")
    again = x.clone()
    got = B.block_norm(again, h, x_out=again, y=wide[:, 8:8 + N], **k)
    assert got.x is again and torch.equal(again, want.x) and torch.equal(wide[:, 8:8 + N], want.y)
    assert bool((wide[:, :8] == 7).all()) and bool((wide[:, 8 + N:] == 7).all())
    assert torch.equal(B.block_norm(want.x, pre="layer", pre_weight=k["pre_weight"], pre_bias=k["pre_bias"], eps=EPS).y, want.y)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
def test_rows_of_zeros_equal_rows_and_rows_that_are_not_finite(dtype):
    """A row that is constant has no variance: its normalised values are 0 to rounding, with eps under the root.  NaN stays in its row."""
    torch = _torch()
    rng = np.random.default_rng(9)
    x, h, k = tensors(rng, 6, 200, dtype, "layer", "rms", "columns", True, 0)
    h[0] = 0
    h[1] = 4.0
    x[0] = 0
    clean = B.block_norm(x, h, **k)
    assert bool(torch.isfinite(clean.x).all()) and bool(torch.isfinite(clean.y).all())
    want = 0.75 * to64(x)[:2] + to64(k["gate"]) * to64(k["post_bias"])
    assert_within(clean.x[:2], want, 3 * HALF_ULP[dtype] * (np.abs(want) + 1))
    h[3, 5] = float("nan")
    x[4, 7] = float("inf")
    got = B.block_norm(x, h, **k)
    assert bool(torch.isnan(got.x[3]).all()) and bool(torch.isnan(got.y[3]).all())
    assert float(got.x[4, 7]) == float("inf") and bool(torch.isnan(got.y[4, 7]))
    for t, c in zip(got, clean):
        assert torch.equal(t[[0, 1, 2, 5]], c[[0, 1, 2, 5]])


@pytest.mark.gpu
@pytest.mark.parametrize("M,N", [(0, 8), (5, 0), (0, 0)])
def test_empty(M, N):
    torch = _torch()
    x = torch.empty((M, N), device="cuda")
    w = torch.ones((N,), device="cuda")
    got = B.block_norm(x, x.clone(), post="rms", post_weight=w, gate=w, pre="layer", pre_weight=w, pre_bias=w)
    assert got.x.shape == got.y.shape == (M, N)
    g = B.block_norm_backward(x, x, x, x, post="rms", post_weight=w, gate=w, pre="layer", pre_weight=w, pre_bias=w)
    assert g.dx.shape == g.dh.shape == (M, N)
    for t in (g.dgate, g.dpost_weight, g.dpre_weight, g.dpre_bias):
        assert t.shape == (N,) and bool((t == 0).all())


# ---- gradients -------------------------------------------------------------------------------------------

def through64(t, hat, r, kind):
    if kind == "none":
        return t
    return r * (t - hat * (t * hat).mean(1, keepdims=True) - (t.mean(1, keepdims=True) if kind == "layer" else 0))


def spread64(t, hat, r, kind):
    """The magnitudes that through64 adds."""
    t, hat = np.abs(t), np.abs(hat)
    if kind == "none":
        return t
    return r * (t + hat * (t * hat).mean(1, keepdims=True) + t.mean(1, keepdims=True))


def check_backward(rng, M, N, dtype, post, pre, gate, bias=True, gap=0, lead=0, dout=True, dy=True, scale=0.02):
    x, h, k = tensors(rng, M, N, dtype, post, pre, gate, bias, gap, lead)
    tx, th = to64(x), to64(h)
    gx = make(rng, (M, N + gap + lead), dtype, scale)[0][:, lead:lead + N] if dout else None
    gy = make(rng, (M, N + gap + lead), dtype, scale)[0][:, lead:lead + N] if dy and pre != "none" else None
    got = B.block_norm_backward(gy, gx, x, h, **k)
    u, e = HALF_ULP[dtype], (N / 64 + 16) * 2.0 ** -24
    es = (M / 8 + 64) * 2.0 ** -24                  # column sums: at most this long a chain
    d, off_d = np.zeros((M, N)), np.zeros((M, N))
    if dout:
        d = d + to64(gx)
        off_d = off_d + 2.0 ** -22 * np.abs(d)
    if gy is not None:
        hat, r, mean = hat64(tx, pre)
        y = to64(gy)
        t = y * (1 if k["pre_weight"] is None else to64(k["pre_weight"]))
        d = d + through64(t, hat, r, pre)
        off_hat = 2 * e * (np.abs(hat) + mean)
        off_d = off_d + 8 * e * (1 + mean) * spread64(t, hat, r, pre)

        def column(got, terms, offs):
            want = terms.sum(0)
            off = offs.sum(0) + es * (np.abs(terms) + offs).sum(0)
            assert_within(got, want, off + u * (np.abs(want) + off) + TINY[dtype])
        if k["pre_weight"] is not None:
            column(got.dpre_weight, y * hat, np.abs(y) * off_hat)
        if k["pre_bias"] is not None:
            column(got.dpre_bias, y, 0 * y)

    def near(got, want, off):
        assert_within(got, want, off + u * (np.abs(want) + off) + TINY[dtype])
    near(got.dx, 0.75 * d, off_d + 2.0 ** -22 * np.abs(d))
    hat, r, mean = hat64(th, post)
    off_hat = 2 * e * (np.abs(hat) + mean)
    g = rows_of_gate(k["gate"], M)
    wp = 1 if k["post_weight"] is None else to64(k["post_weight"])
    t, off_t = d * g * wp, off_d * np.abs(g * wp)
    near(got.dh, through64(t, hat, r, post), spread64(off_t, hat, r, post) + 8 * e * (1 + mean) * spread64(np.abs(t) + off_t, hat, r, post))
    # sums of d hat and of d, each taken in 32 bits, then joined with weight, bias and gate
    one, off_one = d * hat, off_d * np.abs(hat) + (np.abs(d) + off_d) * off_hat
    groups = gate if isinstance(gate, int) else 1

    def by_group(v):
        return v.reshape(groups, M // groups, N).sum(1)
    off1, off0 = by_group(off_one + es * np.abs(one)), by_group(off_d + es * np.abs(d))
    s1, s0 = by_group(one), by_group(d)
    bp = 0 if k["post_bias"] is None else to64(k["post_bias"])
    if gate:
        want = wp * s1 + bp * s0
        off = np.abs(wp) * off1 + np.abs(bp) * off0 + 2.0 ** -22 * (np.abs(wp * s1) + np.abs(bp * s0))
        near(got.dgate, want.reshape(tuple(k["gate"].shape)), off.reshape(tuple(k["gate"].shape)))
    gg = np.ones((1, 1)) if k["gate"] is None else to64(k["gate"]).reshape(groups, N)
    eg = (groups + 16) * 2.0 ** -24
    if k["post_weight"] is not None:
        near(got.dpost_weight, (gg * s1).sum(0), (np.abs(gg) * off1 + eg * np.abs(gg * s1)).sum(0))
    if k["post_bias"] is not None:
        near(got.dpost_bias, (gg * s0).sum(0), (np.abs(gg) * off0 + eg * np.abs(gg * s0)).sum(0))
    assert (got.dgate is None) == (gate is None) and (got.dpost_bias is None) == (k["post_bias"] is None)
    again = B.block_norm_backward(gy, gx, x, h, **k)
    for a, b in zip(got, again):
        assert (a is None and b is None) or _torch().equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N", SIZES)
@pytest.mark.parametrize("kind", ["rms", "layer"])
def test_backward_sizes(dtype, M, N, kind):
    check_backward(np.random.default_rng(M + N), M, N, dtype, kind, kind, "columns")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("post,pre", [("none", "rms"), ("none", "layer"), ("rms", "none"), ("layer", "rms"), ("none", "none")])
@pytest.mark.parametrize("gate", [None, "columns", 1, 3, 12])
@pytest.mark.parametrize("bias", [False, True])
def test_backward_kinds(dtype, post, pre, gate, bias):
    check_backward(np.random.default_rng(5), 12, 328, dtype, post, pre, gate, bias)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("gap,lead", [(8, 0), (3, 0), (5, 1), (7, 9)])
@pytest.mark.parametrize("M,N", [(3, 40), (40, 1000), (9, 4097)])
def test_backward_strides_and_alignment(dtype, gap, lead, M, N):
    check_backward(np.random.default_rng(gap), M, N, dtype, "layer", "rms", "columns", True, gap, lead)


@pytest.mark.gpu
@pytest.mark.parametrize("dout,dy", [(False, True), (True, False)])
@pytest.mark.parametrize("post,pre", [("rms", "rms"), ("none", "layer"), ("layer", "layer")])
def test_backward_of_one_gradient_alone(dout, dy, post, pre):
    check_backward(np.random.default_rng(2), 20, 136, "float32", post, pre, 5, dout=dout, dy=dy)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,M,N,gate", [("bfloat16", 3000, 128, 30), ("bfloat16", 2100, 2048, None), ("float32", 1500, 1000, "columns"),
                                            ("float16", 1024, 4096, 2), ("bfloat16", 600, 64, 600), ("float32", 520, 9000, 40)])
def test_backward_many_rows(dtype, M, N, gate):
    check_backward(np.random.default_rng(M), M, N, dtype, "layer", "rms", gate)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,M,N,gate,bias", [("bfloat16", 600, 9001, 40, False), ("float16", 520, 8201, None, True), ("float32", 300, 16383, "columns", True)])
def test_backward_many_wide_rows(dtype, M, N, gate, bias):
    check_backward(np.random.default_rng(N), M, N, dtype, "rms", "layer", gate, bias)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("dout,dy,post,pre", [(False, True, "rms", "rms"), (True, False, "layer", "layer"), (True, True, "none", "layer"), (True, True, "rms", "none")])
def test_backward_wide_rows_of_each_kind(dtype, dout, dy, post, pre):
    check_backward(np.random.default_rng(4), 6, 8195, dtype, post, pre, 3, True, dout=dout, dy=dy and pre != "none")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("last", range(1, 8))
@pytest.mark.parametrize("whole", [0, 8, 128, 520, 1032, 2056, 4104, 8200])
def test_rows_that_end_within_a_piece(dtype, last, whole):
    rng = np.random.default_rng(whole + last)
    check_forward(rng, 5, whole + last, dtype, "layer", "rms", "columns", True)
    check_backward(rng, 5, whole + last, dtype, "layer", "rms", "columns", True)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M,N,gate", [(1, 129, "columns"), (700, 200, 7), (2100, 256, None), (16500, 136, 50)])
def test_rows_of_two_pieces_to_a_lane(dtype, M, N, gate):
    check_forward(np.random.default_rng(M), M, N, dtype, "rms", "layer", gate, True)
    check_backward(np.random.default_rng(M), M, N, dtype, "rms", "layer", gate, True)


@pytest.mark.gpu
def test_backward_without_a_block_and_of_what_is_wanted_only():
    torch = _torch()
    rng = np.random.default_rng(8)
    x, h, k = tensors(rng, 30, 100, "float32", "rms", "layer", 3, True, 0)
    dy, dout = make(rng, (30, 100), "float32")[0], make(rng, (30, 100), "float32")[0]
    pre = dict(pre="layer", pre_weight=k["pre_weight"], pre_bias=k["pre_bias"], eps=EPS)
    full = B.block_norm_backward(dy, dout, x, h, **k)
    alone = B.block_norm_backward(dy, dout, x, **pre)
    assert alone.dh is None and alone.dgate is None
    # the same 30 terms of a column, added in another order where the rows of a gate are summed first: each sum is within 46 2^-24 of their magnitudes,
    # and rounded once more
    hat = np.abs(hat64(to64(x), "layer")[0])
    for a, b, terms in ((alone.dpre_weight, full.dpre_weight, np.abs(to64(dy)) * hat), (alone.dpre_bias, full.dpre_bias, np.abs(to64(dy)))):
        assert_within(a, to64(b), 2 * 47 * 2.0 ** -24 * terms.sum(0))
    assert torch.equal(0.75 * alone.dx, full.dx)
    only = B.block_norm_backward(dy, dout, x, h, want_weights=False, **k)
    assert torch.equal(only.dx, full.dx) and torch.equal(only.dh, full.dh) and all(t is None for t in only[2:])
    only = B.block_norm_backward(dy, dout, x, h, want_dx=False, **k)
    assert only.dx is None and only.dh is None and all(torch.equal(a, b) for a, b in zip(only[2:], full[2:]))


@pytest.mark.gpu
@pytest.mark.parametrize("post,pre", [("rms", "layer"), ("layer", "rms"), ("none", "layer")])
def test_gradients_against_differences(post, pre):
    """Central differences in 64 bits of the formula, step 1e-4 of values of order 1: their error is of order (1e-4)^2 of the third derivative and
    1e-16 / 1e-4 of the loss, together below 1e-6 of the largest gradient; the kernels' sums, 40 rows of 24 columns, below 300 2^-24 = 2e-5 of it."""
    torch = _torch()
    rng = np.random.default_rng(12)
    M, N = 40, 24
    x, h, k = tensors(rng, M, N, "float32", post, pre, 5, True, 0)
    dy, dout = make(rng, (M, N), "float32")[0], make(rng, (M, N), "float32")[0]
    out = B.block_norm(x, h, **k).x
    g = B.block_norm_backward(dy, dout, out, h, **k)
    at = {n: to64(t) for n, t in (("x", x), ("h", h), ("gate", k["gate"]), ("wp", k["post_weight"]), ("bp", k["post_bias"]),
                                  ("w", k["pre_weight"]), ("b", k["pre_bias"])) if t is not None}

    def loss(v):
        p = hat64(v["h"], post)[0] * v.get("wp", 1.0) + v.get("bp", 0.0)
        s = 0.75 * v["x"] + np.repeat(v["gate"], M // 5, 0) * p
        y = hat64(s, pre)[0] * v["w"] + v["b"]
        return float((to64(dy) * y).sum() + (to64(dout) * s).sum())
    for name, got in (("x", g.dx), ("h", g.dh), ("gate", g.dgate), ("wp", g.dpost_weight), ("bp", g.dpost_bias), ("w", g.dpre_weight), ("b", g.dpre_bias)):
        if got is None:
            assert name not in at
            continue
        got = to64(got)
        largest = np.abs(got).max()
        for i in rng.integers(0, got.size, 6):
            ends = []
            for step in (1e-4, -1e-4):
                v = dict(at)
                v[name] = at[name].copy()
                v[name].flat[i] += step
                ends.append(loss(v))
            assert abs((ends[0] - ends[1]) / 2e-4 - got.flat[i]) <= 4e-5 * max(largest, 1.0), (name, i)
    del torch


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,M,N", [("bfloat16", 700, 512), ("float32", 4, 1000), ("float16", 64, 8200)])
def test_other_streams_and_graphs(dtype, M, N):
    """The same bits on another stream and from every replay of a graph, with data that changes between them."""
    torch = _torch()
    rng = np.random.default_rng(M)
    x, h, k = tensors(rng, M, N, dtype, "rms", "layer", 4, True, 0)
    dy, dout = make(rng, (M, N), dtype)[0], make(rng, (M, N), dtype)[0]

    def both():
        n = B.block_norm(x, h, **k)
        return (*n, *B.block_norm_backward(dy, dout, n.x, h, **k))
    want = both()
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        other = both()
    torch.cuda.current_stream().wait_stream(s)
    assert all(torch.equal(a, b) for a, b in zip(want, other))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for turn in range(3):
        x.copy_(make(rng, (M, N), dtype)[0])
        dy.copy_(make(rng, (M, N), dtype)[0])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(both(), held)), turn


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,M,N", [("bfloat16", 9000, 4096), ("float32", 20000, 520), ("float16", 4100, 8200)])
def test_tensors_larger_than_the_caches(dtype, M, N):
    """Rows of a large call and of a small one are the same to the last bit."""
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    T = getattr(torch, dtype)
    x, h, dy, dout = (torch.randn((M, N), generator=g, device="cuda").to(T) for _ in range(4))
    w = torch.randn((N,), generator=g, device="cuda").to(T)
    k = dict(post="rms", post_weight=w, gate=w, scale=0.5, pre="layer", pre_weight=w, pre_bias=w)
    n = B.block_norm(x, h, **k)
    b = B.block_norm_backward(dy, dout, n.x, h, **k)
    for at in (0, M // 2, M - 30):
        s = slice(at, at + 30)
        few = B.block_norm(x[s], h[s], **k)
        assert torch.equal(n.x[s], few.x) and torch.equal(n.y[s], few.y)
        back = B.block_norm_backward(dy[s], dout[s], few.x, h[s], **k)
        assert torch.equal(b.dx[s], back.dx) and torch.equal(b.dh[s], back.dh)


@pytest.mark.gpu
def test_offsets_beyond_32_bits():
    torch = _torch()
    rng = np.random.default_rng(6)
    rows, gap = 1100, 1 << 21
    big = torch.empty(rows * gap, dtype=torch.bfloat16, device="cuda").view(rows, gap)
    x, h, k = tensors(rng, rows, 72, "bfloat16", "rms", "rms", None, True, 0)
    far = [big[:, 128 * i:128 * i + 72] for i in range(4)]
    far[0].copy_(x)
    far[1].copy_(h)
    want = B.block_norm(x, h, **k)
    B.block_norm(far[0], far[1], x_out=far[2], y=far[3], **k)
    assert torch.equal(far[2], want.x) and torch.equal(far[3], want.y)
    a, b = (B.block_norm_backward(t[3], t[0], t[2], t[1], **k) for t in ((x, h, want.x, want.y), far))
    assert all((p is None and q is None) or torch.equal(p, q) for p, q in zip(a, b))


@pytest.mark.gpu
def test_a_backward_pass_through_the_results_is_refused():
    torch = _torch()
    x, h, k = tensors(np.random.default_rng(1), 4, 40, "float32", "rms", "rms", "columns", False, 0)
    for t in (x, h, k["gate"], k["pre_weight"]):
        t.requires_grad_()
        got = B.block_norm(x, h, **k)
        for y in got:
            with pytest.raises(RuntimeError, match="block_norm_backward"):
                y.sum().backward()
        with torch.no_grad():
            assert not B.block_norm(x, h, **k).y.requires_grad
        t.requires_grad_(False)
    with pytest.raises(RuntimeError):
        B.block_norm(x, h, y=torch.empty_like(x).requires_grad_(), **k)
    with pytest.raises(RuntimeError):
        B.block_norm(x.requires_grad_(), h, x_out=x, **k)


# ---- refusals ---------------------------------------------------------------------------------------------

P = 4096                                            # an address that is aligned and never read


def _forward_args(**change):
    a = dict(M=4, N=8, groups=1, dtype=0, post=1, pre=1, scale=1.0, eps=1e-6, x=P, h=P, post_weight=P, post_bias=None, gate=P, pre_weight=P, pre_bias=None,
             x_out=P, y=P, ldx=8, ldh=8, ldo=8, ldy=8)
    a.update(change)
    return B.BlockNormArgs(*[a[n] for n, _ in B.BlockNormArgs._fields_])


def _backward_args(**change):
    a = dict(M=4, N=8, groups=1, dtype=0, post=1, pre=1, scale=1.0, eps=1e-6, dy=P, dx_out=P, x=P, h=P, post_weight=P, post_bias=None, gate=P, pre_weight=P,
             lddy=8, lddx=8, ldx=8, ldh=8, dx=P, dh=P, dgate=P, dpost_weight=P, dpost_bias=P, dpre_weight=P, dpre_bias=P)
    a.update(change)
    return B.BlockNormBackwardArgs(*[a[n] for n, _ in B.BlockNormBackwardArgs._fields_])


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), -1), (dict(N=-1), -1), (dict(M=1 << 31), -2), (dict(N=1 << 31), -2), (dict(dtype=3), -2), (dict(post=3), -2), (dict(pre=-1), -2),
    (dict(groups=0), -1), (dict(groups=3), -1), (dict(x=None), -1), (dict(x_out=None), -1), (dict(y=None), -1), (dict(h=None), -1),
    (dict(h=None, gate=None, x_out=None, post=0, post_weight=None, scale=2.0), -1), (dict(post=0), -1), (dict(pre=0), -1),
    (dict(ldx=7), -1), (dict(ldh=7), -1), (dict(ldo=7), -1), (dict(ldy=7), -1), (dict(x=P + 2), -1), (dict(gate=P + 1), -1), (dict(eps=-1.0), -1),
    (dict(eps=float("nan")), -1)])
def test_c_forward_refuses_without_touching_the_gpu(change, code):
    assert B.lib().iolb_block_norm(ctypes.byref(_forward_args(**change))) == code
    assert B.lib().iolb_block_norm(None) == -1


@pytest.mark.parametrize("change,code", [
    (dict(M=-1), -1), (dict(M=1 << 23), -2), (dict(N=1 << 23), -2), (dict(dtype=-1), -2), (dict(post=9), -2), (dict(groups=3), -1), (dict(groups=0), -1),
    (dict(dy=None, dx_out=None, dpre_weight=None, dpre_bias=None), -1), (dict(dy=None), -1), (dict(x=None), -1), (dict(h=None), -1), (dict(gate=None), -1),
    (dict(post=0), -1), (dict(pre=0), -1), (dict(lddy=7), -1), (dict(lddx=7), -1), (dict(ldx=7), -1), (dict(ldh=7), -1), (dict(dgate=P + 2), -1), ({}, -4)])
def test_c_backward_refuses_without_touching_the_gpu(change, code):
    assert B.lib().iolb_block_norm_backward(ctypes.byref(_backward_args(**change)), None, 0) == code


def test_backward_workspace():
    L, need = B.lib(), ctypes.c_size_t(0)
    assert L.iolb_block_norm_backward_workspace_bytes(ctypes.byref(_backward_args()), ctypes.byref(need)) == 0 and need.value > 0
    assert L.iolb_block_norm_backward(ctypes.byref(_backward_args()), P, need.value - 1) == -4
    assert L.iolb_block_norm_backward(ctypes.byref(_backward_args()), P + 8, need.value) == -4
    assert L.iolb_block_norm_backward_workspace_bytes(None, ctypes.byref(need)) == -1
    assert L.iolb_block_norm_backward_workspace_bytes(ctypes.byref(_backward_args()), None) == -1
    for M, N, groups in ((1 << 22, 1 << 22, 1 << 22), (1 << 22, 1 << 22, 1)):
        code = L.iolb_block_norm_backward_workspace_bytes(ctypes.byref(_backward_args(M=M, N=N, groups=groups, lddy=N, lddx=N, ldx=N, ldh=N)), ctypes.byref(need))
        assert code == (-2 if groups > 1 else 0)


@pytest.mark.parametrize("groups", [(1 << 22) + 1, 1 << 31, 1 << 32, 1 << 62])
def test_backward_of_no_rows_refuses_more_groups_than_it_counts(groups):
    need = ctypes.c_size_t(0)
    args = _backward_args(M=0, groups=groups)
    assert B.lib().iolb_block_norm_backward_workspace_bytes(ctypes.byref(args), ctypes.byref(need)) == -2
    assert B.lib().iolb_block_norm_backward(ctypes.byref(args), P, 1 << 40) == -2


def test_python_refuses_cpu_tensors_and_unknown_names():
    torch = _torch()
    x = torch.zeros((4, 8))
    for call in (lambda: B.block_norm(x), lambda: B.block_norm_backward(x, x, x), lambda: B.block_norm(3)):
        with pytest.raises(TypeError):
            call()


@pytest.mark.gpu
def test_python_refusals():
    torch = _torch()
    x, w = torch.zeros((4, 8), device="cuda"), torch.zeros((8,), device="cuda")
    for error, call in (
            (ValueError, lambda: B.block_norm(x, pre="batch")), (ValueError, lambda: B.block_norm(x, x, post="x")), (ValueError, lambda: B.block_norm(x, pre="none")),
            (ValueError, lambda: B.block_norm(x, gate=w)), (ValueError, lambda: B.block_norm(x, scale=2.0)), (ValueError, lambda: B.block_norm(x, x_out=x)),
            (ValueError, lambda: B.block_norm(x, x, post="none", post_weight=w)), (ValueError, lambda: B.block_norm(x, x, pre="none", pre_bias=w)),
            (ValueError, lambda: B.block_norm(x, x, gate=torch.zeros((3, 8), device="cuda"))), (ValueError, lambda: B.block_norm(x, x, gate=w[:4])),
            (ValueError, lambda: B.block_norm(x, x[:3])), (TypeError, lambda: B.block_norm(x, x.half())), (TypeError, lambda: B.block_norm(x.t())),
            (TypeError, lambda: B.block_norm(x, pre_weight=w.half())), (TypeError, lambda: B.block_norm(x.double())),
            (ValueError, lambda: B.block_norm_backward(None, None, x)), (ValueError, lambda: B.block_norm_backward(x, x, x, pre="none")),
            (ValueError, lambda: B.block_norm_backward(x[:2], x, x))):
        with pytest.raises(error):
            call()
