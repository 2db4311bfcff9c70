"""Large fp32 dense layers whose operands go to the matrix cores in two fp16 parts: values that two parts do not hold, where they make up a sum.

Bound of every output, from the formats and before anything was run: an operand value is held to 2^-22 of itself and the product of two low
parts is left out, 2^-22 of the product at most, so a sum of K products is within (K + 16) 2^-24 of its sum of magnitudes as long as
K + 16 is well above 12 (here K is 1000 and more): the same bound as for any fp32 layer.  Nothing is allowed for the size of a row's largest value.
"""
import numpy as np
import pytest

from paper_2012_15667_amd import binding as B
from tests.test_dense import act64, assert_within, to64, values64

U = 2.0 ** -24
# M N K, the first with one workgroup to a block of sums, the second with shared K, the third ragged throughout
SHAPES = [(2304, 1100, 1536), (600, 640, 9216), (1111, 1301, 2501)]


def _data(M, N, K, seed):
    rng = np.random.default_rng(seed)
    return rng.standard_normal((M, K)).astype(np.float32), (rng.standard_normal((N, K)) / 32).astype(np.float32)


def _check(x, w, **kw):
    import torch
    xt, wt = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    x64, w64 = x.astype(np.float64), w.astype(np.float64)
    want, total = x64 @ w64.T, np.abs(x64) @ np.abs(w64).T
    assert_within(B.linear(xt, wt, **kw), want, (x.shape[1] + 16) * U * total + 2.0 ** -149)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("power", [-18, -25, -45, -90])
def test_weights_that_read_a_column_of_small_values(M, N, K, power):
    """One column of x lies far below its rows' largest values; a few rows of w read nothing else, so their sums are what was cut."""
    x, w = _data(M, N, K, 1)
    x[:, 7] *= 2.0 ** power
    for n in (0, 5, N // 2, N - 1):
        w[n] = 0
        w[n, 7] = 1 + n
    _check(x, w)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_rows_that_are_weighted_where_they_are_small(M, N, K):
    """The same with the operands' parts exchanged: rows of x that meet small values of w alone."""
    x, w = _data(M, N, K, 2)
    w[:, K - 1] *= 2.0 ** -33
    for m in (0, 1, 300, M - 1):
        x[m] = 0
        x[m, K - 1] = -3.0
    _check(x, w)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_many_such_weights(M, N, K):
    """A third of w reads small columns only: whole blocks of sums are taken in three parts, the others stay."""
    x, w = _data(M, N, K, 3)
    x[:, :8] *= 2.0 ** -30
    w[:N // 3, 8:] = 0
    _check(x, w)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", SHAPES)
@pytest.mark.parametrize("many", [False, True])
def test_such_weights_through_the_epilogue(M, N, K, many):
    """Bias, residual before and after the activation, y as the residual, checkpoint: for sums that are taken again and for those that are not."""
    import torch
    x, w = _data(M, N, K, 4)
    x[:, 3] *= 2.0 ** -26
    few = slice(0, N // 3) if many else slice(N - 2, N)
    w[few] = 0
    w[few, 3] = 2.0 ** 24
    rng = np.random.default_rng(5)
    b, r = rng.standard_normal(N).astype(np.float32), rng.standard_normal((M, N)).astype(np.float32)
    x64, w64, b64, r64 = (t.astype(np.float64) for t in (x, w, b, r))
    xt, wt, bt, rt = (torch.from_numpy(t).cuda() for t in (x, w, b, r))
    z, total = x64 @ w64.T + b64, np.abs(x64) @ np.abs(w64).T + np.abs(b64)
    off = (K + 16) * U * total
    want = act64(z, "relu") + r64
    inplace = rt.clone()
    assert B.linear(xt, wt, bt, act="relu", residual=inplace, y=inplace) is inplace
    assert_within(inplace, want, off + 2 * U * (np.abs(want) + np.abs(r64) + off))
    y, c = B.linear(xt, wt, bt, act="gelu", residual=rt, residual_first=True, checkpoint=True)
    z, off = z + r64, off + 2 * U * np.abs(r64)
    want = act64(z, "gelu")
    assert_within(y, want, 1.13 * off + 1e-6 * np.abs(z) + 1e-7 + U * np.abs(want))
    q, e = c.q.cpu().numpy(), c.e.cpu().numpy()
    unit = 2.0 ** (np.repeat(e.astype(int), 32, axis=1)[:, :N] - 127.0)
    assert np.all(np.abs(values64(q, e) - z) <= unit / 2 + off)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_one_hot_weights_and_rows_of_zeros(M, N, K):
    """w picks single values of rows that span fp32's whole range, and zeros of either operand are zeros of the result."""
    rng = np.random.default_rng(6)
    x, w = _data(M, N, K, 6)
    x[::3] *= (2.0 ** rng.integers(-60, 60, (len(x[::3]), 1))).astype(np.float32)
    x[:, 11] = (x[:, 11] * 2.0 ** rng.integers(-40, 0, M)).astype(np.float32)
    x[4] = 0
    w[9] = 0
    w[12] = 0
    w[12, 11] = 2.0 ** 20
    w[13] = 0
    w[13, 10] = 1
    _check(x, w)


@pytest.mark.gpu
def test_sums_taken_again_are_the_same_every_time():
    import torch
    M, N, K = SHAPES[0]
    x, w = _data(M, N, K, 7)
    x[:, 7] *= 2.0 ** -25
    w[:3] = 0
    w[:3, 7] = 1.0
    xt, wt = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    first = B.linear(xt, wt)
    for _ in range(4):
        assert torch.equal(B.linear(xt, wt), first)
    # not a bit of the other rows depends on them
    w[:3] = 0
    assert torch.equal(B.linear(xt, torch.from_numpy(w).cuda())[:, 3:], first[:, 3:])
