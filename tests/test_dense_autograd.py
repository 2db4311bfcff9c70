"""Tensors that require gradients: linear() has no graph behind it, and says so when one is asked for instead of ending it silently."""
import pytest

from paper_2012_15667_amd import binding as B


def _tensors():
    import torch
    g = torch.Generator().manual_seed(3)
    return [torch.randn(s, generator=g).cuda() for s in ((5, 40), (24, 40), (24,), (5, 24))]


@pytest.mark.gpu
@pytest.mark.parametrize("which", range(4))
@pytest.mark.parametrize("checkpoint", [False, True])
@pytest.mark.parametrize("given", [False, True])
def test_gradients_through_linear_are_refused_where_they_are_asked_for(which, checkpoint, given):
    import torch
    x, w, b, r = t = _tensors()
    want = B.linear(x, w, b, residual=r)
    t[which].requires_grad_()
    out = torch.empty_like(want) if given else None
    y = B.linear(x, w, b, residual=r, checkpoint=checkpoint, y=out)
    y = y[0] if checkpoint else y
    assert torch.equal(y.detach(), want) and y.requires_grad and (out is None or y is out)
    with pytest.raises(RuntimeError, match="linear_backward"):
        (2 * y).sum().backward()
    with torch.no_grad():
        y = B.linear(x, w, b, residual=r, checkpoint=checkpoint)
        y = y[0] if checkpoint else y
        assert torch.equal(y, want) and not y.requires_grad


@pytest.mark.gpu
def test_y_that_requires_gradients_is_refused():
    import torch
    x, w, b, r = _tensors()
    with pytest.raises(RuntimeError):
        B.linear(x, w, b, y=r.requires_grad_())
    with torch.no_grad():
        assert B.linear(x, w, b, y=r) is r


@pytest.mark.gpu
def test_a_function_around_the_pair():
    """The intended way: a forward that keeps checkpoints, a backward that reads them.  Inside, nothing is refused."""
    import torch

    class Layer(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, w, b):
            y, z = B.linear(x, w, b, act="gelu", checkpoint=True)
            ctx.kept = B.checkpoint_pack(x), z, w
            return y

        @staticmethod
        def backward(ctx, dy):
            x8, z8, w = ctx.kept
            g = B.linear_backward(dy.contiguous(), w, x8, z8, act="gelu")
            return g.dx, g.dw, g.db

    x, w, b, dy = _tensors()
    for t in (x, w, b):
        t.requires_grad_()
    Layer.apply(x, w, b).backward(dy)
    with torch.no_grad():
        _, z8 = B.linear(x, w, b, act="gelu", checkpoint=True)
        g = B.linear_backward(dy, w, B.checkpoint_pack(x), z8, act="gelu")
    assert torch.equal(x.grad, g.dx) and torch.equal(w.grad, g.dw) and torch.equal(b.grad, g.db)
