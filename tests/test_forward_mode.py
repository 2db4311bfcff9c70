"""Tensors with tangents (forward-mode derivatives): the calls have none to give, and say so instead of dropping them."""
import pytest

from paper_2012_15667_amd import binding as B


def _tensors():
    import torch
    g = torch.Generator().manual_seed(3)
    return [torch.randn(s, generator=g).cuda() for s in ((8, 64), (64, 64), (64,), (8, 64))]


def _calls():
    """name: (inputs of [8][64], [64][64], [64], [8][64] that it takes, the call)"""
    four = B.mx4_pack(_tensors()[1])
    eight = B.checkpoint_pack(_tensors()[0])
    return dict(
        linear=((0, 1, 2, 3), lambda x, w, b, r: B.linear(x, w, b, residual=r)),
        linear_into=((3,), lambda x, w, b, r: B.linear(x, w, b, y=r)),
        block_norm=((0, 2, 3), lambda x, w, b, r: B.block_norm(x, r, post="rms", post_weight=b, gate=b, pre_weight=b)),
        block_norm_alone=((0, 2), lambda x, w, b, r: B.block_norm(x, pre_weight=b)),
        block_norm_into=((3,), lambda x, w, b, r: B.block_norm(x, y=r)),
        dropout=((0, 3), lambda x, w, b, r: B.dropout(x, 0.5, 1, residual=r)),
        dropout_into=((3,), lambda x, w, b, r: B.dropout(x, 0.5, 1, y=r)),
        linear_mx4=((0, 2, 3), lambda x, w, b, r: B.linear_mx4(x, four, b, residual=r)),
        linear_backward=((1, 3), lambda x, w, b, r: B.linear_backward(r, w, eight)),
        block_norm_backward=((0, 1, 2, 3), lambda x, w, b, r: B.block_norm_backward(r, x, w[:8], x, gate=b, pre_weight=b)))


NAMES = ["linear", "linear_into", "block_norm", "block_norm_alone", "block_norm_into", "dropout", "dropout_into", "linear_mx4", "linear_backward", "block_norm_backward"]


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
@pytest.mark.parametrize("recording", [True, False])
def test_tangents_are_refused_and_nothing_is_written(name, recording):
    import torch
    from torch.autograd import forward_ad
    inputs, call = _calls()[name]
    for which in inputs:
        t = _tensors()
        with forward_ad.dual_level(), torch.set_grad_enabled(recording):
            held = t[which].clone()
            t[which] = forward_ad.make_dual(t[which], torch.ones_like(t[which]))
            with pytest.raises(RuntimeError, match="forward-mode"):
                call(*t)
            assert torch.equal(forward_ad.unpack_dual(t[which]).primal, held)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_tensors_without_tangents_are_taken_where_others_have_them(name):
    import torch
    from torch.autograd import forward_ad
    call = _calls()[name][1]
    want = call(*_tensors())
    with forward_ad.dual_level():
        got = call(*_tensors())
    for a, b in zip([want] if isinstance(want, torch.Tensor) else want, [got] if isinstance(got, torch.Tensor) else got):
        assert (a is None and b is None) or torch.equal(a, b)


@pytest.mark.gpu
@pytest.mark.parametrize("name", NAMES)
def test_transforms_of_functions_are_refused(name):
    import torch
    inputs, call = _calls()[name]

    def first(t):
        all_of_them = _tensors()
        all_of_them[inputs[0]] = t
        got = call(*all_of_them)
        return got if isinstance(got, torch.Tensor) else next(v for v in got if v is not None)
    x = _tensors()[inputs[0]]
    with pytest.raises(RuntimeError):
        torch.func.jvp(first, (x,), (torch.ones_like(x),))
