"""The workspace of large fp32 layers: three planes of each operand, which the two-part route before them uses as well."""
import ctypes

import numpy as np
import pytest

from paper_2012_15667_amd import binding as B


def _args(M, N, K, x, w, y):
    return B.LinearArgs(M, N, K, 0, 0, 0, x, w, None, None, y, K, K, 0, N, None, None)


def _need(args):
    need = ctypes.c_size_t(0)
    assert B.lib().iolb_linear_workspace_bytes(ctypes.byref(args), ctypes.byref(need)) == 0
    return need.value


@pytest.mark.parametrize("M,N,K", [(4096, 4096, 9216), (2048, 2048, 2048), (1111, 1301, 2501)])
def test_routes_share_the_room_of_their_operands(M, N, K):
    """Six bytes a value of both operands, sums of shares of K (at most eight of them at these sizes), and little more: scales and marks."""
    operands, sums = 6 * (M + N) * (K + 7), 8 * M * (N + 3) * 4
    need = _need(_args(M, N, K, 4096, 4096, 4096))
    assert operands * 0.99 <= need <= operands + (sums if K * M * N < 1e10 else 0) + (1 << 20)


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(2304, 1100, 1536), (600, 640, 9216), (1111, 1301, 2501)])
@pytest.mark.parametrize("data", ["even", "uneven", "some left"])
def test_exactly_as_many_bytes_as_told(M, N, K, data):
    import torch
    rng = np.random.default_rng(8)
    x, w = rng.standard_normal((M, K)).astype(np.float32), rng.standard_normal((N, K)).astype(np.float32)
    if data == "uneven":
        x[1, ::3] *= 2.0 ** -40
    if data == "some left":
        x[:, 5] *= 2.0 ** -40
        w[:N // 4] = 0
        w[:N // 4, 5] = 1
    xt, wt = torch.from_numpy(x).cuda(), torch.from_numpy(w).cuda()
    y = torch.full((M, N), 7.0, device="cuda")
    args = _args(M, N, K, xt.data_ptr(), wt.data_ptr(), y.data_ptr())
    need = _need(args)
    ws = torch.full((need + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
    B.lib().iolb_set_stream(torch.cuda.current_stream().cuda_stream)
    for _ in range(2):                                   # (the second with what the first left there)
        assert B.lib().iolb_linear(ctypes.byref(args), ws.data_ptr(), need) == 0
        torch.cuda.synchronize()
        assert bool((ws[need:] == 0xA5).all())
        x64, w64 = x.astype(np.float64), w.astype(np.float64)
        off = np.abs(y.double().cpu().numpy() - x64 @ w64.T) - (K + 16) * 2.0 ** -24 * (np.abs(x64) @ np.abs(w64).T)
        assert off.max() <= 2.0 ** -149
    assert B.lib().iolb_linear(ctypes.byref(args), ws.data_ptr(), need - 1) == -4


@pytest.mark.gpu
@pytest.mark.parametrize("M,N,K", [(2304, 1100, 1536), (600, 640, 9216)])
def test_replays_of_a_graph_with_data_of_another_kind(M, N, K):
    """What one replay finds of its operands (even, uneven, some sums or many to be taken again) is not the next one's."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(5)
    plain = [torch.randn(s, generator=g, device="cuda") for s in ((M, K), (N, K))]

    def data(kind):
        x, w = (t.clone() for t in plain)
        if kind == "uneven":
            x[1, ::3] *= 2.0 ** -40
        if kind in ("few", "many"):
            x[:, 5] *= 2.0 ** -40
            rows = slice(0, N // 4) if kind == "many" else slice(0, 1)
            w[rows] = 0
            w[rows, 5] = 1
        return x, w

    x, w = data("even")
    r = torch.randn((M, N), generator=g, device="cuda")
    B.linear(x, w)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        y, z = B.linear(x, w, act="silu", residual=r, residual_first=True, checkpoint=True)
    for kind in ("many", "even", "uneven", "few", "many", "few", "even"):
        for to, t in zip((x, w), data(kind)):
            to.copy_(t)
        want, z_want = B.linear(x, w, act="silu", residual=r, residual_first=True, checkpoint=True)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want) and torch.equal(z.q, z_want.q) and torch.equal(z.e, z_want.e), kind
