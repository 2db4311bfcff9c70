"""Gradients of block norms over no rows: sums of nothing, which are zero whatever stands in the weights and the gate."""
import ctypes

import pytest

from paper_2012_15667_amd import binding as B
from tests.test_block_norm import P, _backward_args


def _torch():
    import torch
    return torch


def _need(**change):
    need = ctypes.c_size_t(0)
    N = change["N"]
    code = B.lib().iolb_block_norm_backward_workspace_bytes(ctypes.byref(_backward_args(lddy=N, lddx=N, ldx=N, ldh=N, **change)), ctypes.byref(need))
    return code, need.value


@pytest.mark.parametrize("M", [0, 8])
def test_gradients_of_a_gate_that_is_not_there_are_refused(M):
    assert _need(M=M, N=8, groups=4, gate=None)[0] == -1
    assert B.lib().iolb_block_norm_backward(ctypes.byref(_backward_args(M=M, groups=4, gate=None)), P, 1 << 20) == -1


@pytest.mark.gpu
@pytest.mark.parametrize("N", [8, 700, 9000, 20000])
@pytest.mark.parametrize("groups", [None, 1, 2, 5, 70])
@pytest.mark.parametrize("value", [float("inf"), float("nan"), -float("inf")])
def test_sums_over_no_rows_are_zero_whatever_the_weights(N, groups, value):
    torch = _torch()
    x = torch.empty((0, N), device="cuda")
    w = torch.full((N,), value, device="cuda")
    gate = torch.full((N,) if groups is None else (groups, N), value, device="cuda")
    got = B.block_norm_backward(x, x, x, x, post="rms", post_weight=w, post_bias=w, gate=gate, pre="layer", pre_weight=w, pre_bias=w)
    assert got.dgate.shape == gate.shape
    for t in got[2:]:
        assert bool((t == 0).all())
