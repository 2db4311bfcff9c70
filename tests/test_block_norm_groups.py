"""Gradients of block norms whose gate has a row for every row of x, or for nearly as many: more groups than one launch counts."""
import ctypes

import numpy as np
import pytest

from paper_2012_15667_amd import binding as B
from tests.test_block_norm import EPS, P, _backward_args, check_backward
from tests.test_dense import HALF_ULP, TINY

OUTPUTS = ["dx", "dh", "dgate", "dpost_weight", "dpost_bias", "dpre_weight", "dpre_bias"]


def _torch():
    import torch
    return torch


def _need(**change):
    need = ctypes.c_size_t(0)
    N = change["N"]
    code = B.lib().iolb_block_norm_backward_workspace_bytes(ctypes.byref(_backward_args(lddy=N, lddx=N, ldx=N, ldh=N, **change)), ctypes.byref(need))
    return code, need.value


@pytest.mark.parametrize("M,N", [(16384, 4080), (16384, 4096), (8192, 8192), (65536, 1024), (65536, 8208), (1 << 20, 4096), (1 << 22, 64), (1 << 22, 1)])
def test_a_gate_for_every_row_is_taken(M, N):
    """Four sums a column and piece; a piece has rows of one group alone, and rows beyond 8192 values leave eight numbers each."""
    code, need = _need(M=M, N=N, groups=M)
    assert code == 0
    columns, rows = 16 * M * (-(-N // 8) * 8), 32 * M if N > 8192 else 0
    assert need == columns + rows


@pytest.mark.parametrize("M,N,groups", [(16384, 4096, 16384), (1 << 22, 1 << 22, 1 << 22), (1 << 22, 8192, 1 << 22), (1 << 22, 20000, 1 << 20)])
def test_gradients_of_rows_alone_need_nothing_however_many_groups(M, N, groups):
    none = {n: None for n in OUTPUTS[2:]}
    assert _need(M=M, N=N, groups=groups, **none) == (0, 0)


def test_more_sums_than_are_counted_are_refused():
    """2^32 blocks of 16 columns and a group, whose sums alone would be 2^40 bytes."""
    assert _need(M=1 << 22, N=1 << 14, groups=1 << 22)[0] == -2
    assert _need(M=1 << 22, N=(1 << 14) - 16, groups=1 << 22)[0] == 0


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,M,N,groups", [("bfloat16", 270000, 50, 270000), ("float32", 420020, 70, 210010), ("float16", 1100000, 3, 1100000)])
def test_more_groups_than_a_launch_takes(dtype, M, N, groups):
    check_backward(np.random.default_rng(N), M, N, dtype, "rms", "layer", groups)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,M,N", [("bfloat16", 16384, 4096), ("float16", 8200, 8201), ("bfloat16", 8200, 16500)])
def test_wide_gates_for_every_row(dtype, M, N):
    """post(h) = h r, r = 1 / sqrt(mean of h^2 + eps), without a second norm: d is dx_out itself.  A row's gate gets w d hat + b d, w and b the sums over the rows of
    gate d hat and gate d.  Bounds as in test_block_norm.py: hat within 2 e |hat|, three roundings to 32 bits (2^-22 holds them), sums over M groups
    one after the other in 64 threads and then a tree, within (M / 64 + 80) 2^-24 of their magnitudes; one rounding to the type."""
    torch = _torch()
    g = torch.Generator(device="cuda")
    g.manual_seed(N)
    T = getattr(torch, dtype)

    def draw(*shape, by=1.0):
        return (by * torch.randn(shape, generator=g, device="cuda")).to(T)
    x, h, d, gate = draw(M, N), draw(M, N), draw(M, N, by=0.02), draw(M, N)
    w, b = draw(N), draw(N)
    got = B.block_norm_backward(None, d, x, h, post="rms", post_weight=w, post_bias=b, gate=gate, pre="none", eps=EPS)
    u, e, es = HALF_ULP[dtype], (N / 64 + 16) * 2.0 ** -24, (M / 64 + 80) * 2.0 ** -24
    assert torch.equal(got.dx, d)
    sums = torch.zeros((4, N), dtype=torch.float64, device="cuda")
    for at in range(0, M, 1024):
        s = slice(at, at + 1024)
        h64, d64, g64 = h[s].double(), d[s].double(), gate[s].double()
        hat = h64 / (h64.square().mean(1, keepdim=True) + float(np.float32(EPS))).sqrt()
        one, zero = w.double() * d64 * hat, b.double() * d64
        off = (2 * e + 2.0 ** -22) * one.abs() + 2.0 ** -22 * zero.abs()
        assert bool(((got.dgate[s].double() - one - zero).abs() <= off + u * ((one + zero).abs() + off) + TINY[dtype]).all()), at
        for k, t in enumerate((g64 * d64 * hat, g64 * d64)):
            sums[2 * k] += t.sum(0)
            sums[2 * k + 1] += t.abs().sum(0)
    for t, want, magnitudes in ((got.dpost_weight, sums[0], sums[1]), (got.dpost_bias, sums[2], sums[3])):
        off = (2 * e + 2.0 ** -22 + es) * magnitudes
        assert bool(((t.double() - want).abs() <= off + u * (want.abs() + off) + TINY[dtype]).all())
