"""Extents at which a launch would count 2^32 threads or more along an axis, which the runtime refuses: refused with the plan.
Only sizes are asked for here: nothing is launched, and no address is read."""
import ctypes

import pytest

from paper_2012_15667_amd import binding as B

P = 4096


def _linear(M, N, K, dtype, ld=None):
    a = B.LinearArgs(M, N, K, dtype, 0, 0, P, P, None, None, P, ld or K, ld or K, 0, N, None, None)
    need = ctypes.c_size_t(0)
    return B.lib().iolb_linear_workspace_bytes(ctypes.byref(a), ctypes.byref(need)), need.value


def _backward(M, N, K, dtype):
    a = B.LinearBackwardArgs(M, N, K, dtype, 0, 0, P, P, N, K, P, P, None, None, P, P, P, None)
    need = ctypes.c_size_t(0)
    return B.lib().iolb_linear_backward_workspace_bytes(ctypes.byref(a), ctypes.byref(need)), need.value


@pytest.mark.parametrize("M,N,K,dtype", [(1, 1 << 27, 8, 1), (16, (1 << 27) - 14, 8, 0), (1, 1 << 30, 64, 2),        # sixteen columns to 512 threads
                                         (17, 1 << 30, 8, 0),                                                   # 128 columns to 512
                                         (1 << 30, 1, 1, 0), (1 << 30, 1 << 30, 1, 0), (20, 1 << 30, 9, 1),          # rows laid out 64 to 256
                                         (1 << 20, 1 << 20, 64, 1)])                                            # blocks of sums
def test_linear_refuses_launches_too_large(M, N, K, dtype):
    assert _linear(M, N, K, dtype) [0] == -2


@pytest.mark.parametrize("M,N,K,dtype", [(5, 5, 1 << 30, 0), (100, 4, 1 << 30, 1)])
def test_backward_refuses_launches_too_large(M, N, K, dtype):
    assert _backward(M, N, K, dtype) [0] == -2


def test_what_a_launch_can_count_is_planned():
    for M, N, K, dtype, wanted in ((16, (1 << 27) - 32, 8, 0, False), (17, 1 << 26, 8, 0, False), (1000, 1 << 26, 9, 1, True),
                                   (1 << 26, 100, 7, 0, True)):
        code, need = _linear(M, N, K, dtype)
        assert code == 0 and (need > 0) == wanted, (M, N, K, dtype)
    code, need = _backward(5, 5, 1 << 26, 0)
    assert code == 0 and need > 0
