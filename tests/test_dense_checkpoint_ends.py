"""What a checkpoint holds at the two ends of its exponents, of sums beyond the type, and read as another type.  All values here are exact."""
import pytest

from paper_2012_15667_amd import binding as B


def _packed(values, dtype):
    import torch
    T = getattr(torch, dtype)
    c = B.checkpoint_pack(torch.tensor([values], dtype=T).cuda())
    return c, B.checkpoint_unpack(c, T).double().cpu()[0].tolist()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,top,last,least", [("float16", 65504.0, 63 * 2.0 ** 10, 2.0 ** -24), ("float32", 2.0 ** 128 - 2.0 ** 104, 63 * 2.0 ** 122, 2.0 ** -126),
                                                  ("bfloat16", 2.0 ** 128 - 2.0 ** 120, 63 * 2.0 ** 122, 2.0 ** -126)])
def test_ends(dtype, top, last, least):
    assert _packed([top, -top, 1.0], dtype)[1] == [last, -last, 0.0]
    assert _packed([least, 3 * least, 0.0], dtype)[1] == [least, 3 * least, 0.0]
    if dtype != "float16":
        assert _packed([least / 2, least / 4, -least / 2 - least / 64], dtype)[1] == [0.0, 0.0, -least]     # a tie to even, and past it


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 40, 600])
def test_sums_beyond_fp16(M):
    import torch
    x = torch.full((M, 64), 100.0, dtype=torch.float16, device="cuda")
    w = torch.full((40, 64), 16.0, dtype=torch.float16, device="cuda")
    w[1::2] = -16
    y, z = B.linear(x, w, checkpoint=True)
    v = B.checkpoint_unpack(z)
    assert bool((y[:, ::2] == float("inf")).all()) and bool((y[:, 1::2] == float("-inf")).all())
    assert bool((v[:, ::2] == 64512).all()) and bool((v[:, 1::2] == -64512).all())


@pytest.mark.gpu
def test_read_as_another_type():
    import torch
    c, _ = _packed([2.0 ** 100, 2.0 ** 95, -2.0 ** 100], "float32")
    assert B.checkpoint_unpack(c, torch.float16).tolist() == [[float("inf"), float("inf"), float("-inf")]]
    assert B.checkpoint_unpack(c, torch.bfloat16).tolist() == [[2.0 ** 100, 2.0 ** 95, -2.0 ** 100]]
