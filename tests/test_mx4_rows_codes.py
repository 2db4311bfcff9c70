"""Layers of few rows bring x into 4 bits where they multiply it: the same codes and scales as mx4_pack gives, to the last bit, for all values."""
import numpy as np
import pytest

from paper_2012_15667_amd import binding as B
from tests.test_dense import TYPES, to64
from tests.test_mx4 import hard_values, pack64, values64

pytestmark = pytest.mark.gpu


def _identity(K, power):
    """2^power times the unit matrix, in 4 bits."""
    import torch
    w = B.mx4_pack(torch.eye(K, device="cuda") * 2.0 ** power)
    assert torch.equal(B.mx4_unpack(w), torch.eye(K, device="cuda") * 2.0 ** power)
    return w


def _same(a, b):
    import torch
    assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a.nan_to_num(nan=0.0), b.nan_to_num(nan=0.0))


def _finite(x):
    import torch
    return torch.where(torch.isfinite(x), x, torch.ones_like(x))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [1, 5, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("K,gap", [(300, 0), (333, 0), (333, 3), (512, 0), (2037, 1)])
@pytest.mark.parametrize("power", [-60, 0, 60])
def test_every_value_through_a_unit_matrix(dtype, M, K, gap, power):
    """Each result is one value of x in 4 bits times a power of two: large ones are seen with small powers, small ones with large."""
    import torch
    rng = np.random.default_rng(M + K)
    x = _finite(hard_values(rng, M, K + gap, dtype)).cuda()[:, :K]
    w = _identity(K, power)
    got = B.linear_mx4(x, w)
    packed = B.linear_mx4(B.mx4_pack(x), w, dtype=x.dtype)
    _same(got, packed)
    # and against the definition, where the results are normal values of the type
    want = values64(*pack64(to64(x)), K) * 2.0 ** power
    info = torch.finfo(x.dtype)
    normal = (np.abs(want) >= float(info.smallest_normal)) & (np.abs(want) <= float(info.max))
    assert np.array_equal(to64(got)[normal], want[normal])


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("M", [1, 5, 16, 17, 32, 33, 64])
@pytest.mark.parametrize("N,K", [(96, 333), (40, 2037), (130, 64)])
def test_rows_that_are_not_finite_too(dtype, M, N, K):
    rng = np.random.default_rng(M * K)
    x = hard_values(rng, M, K, dtype).cuda()
    w = B.mx4_pack(hard_values(rng, N, K, "float32").clamp(-8.0, 8.0).nan_to_num(nan=1.0).cuda())
    _same(B.linear_mx4(x, w), B.linear_mx4(B.mx4_pack(x), w, dtype=x.dtype))
