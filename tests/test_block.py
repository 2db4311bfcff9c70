"""Residual dense blocks (block.py) and the head with dropout (head.py): norms, layers, dropout and 4 bits together, as they are used."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _mask(shape, p, seed, offset):
    """What dropout multiplies by, in 64 bits."""
    import torch
    from paper_2012_15667_amd import binding as B
    one = torch.ones(shape, device="cuda")
    return B.dropout(one, p, seed, offset).double()


def _hat(v, kind, eps=1e-6):
    if kind == "layer":
        v = v - v.mean(1, keepdim=True)
    return v / (v.square().mean(1, keepdim=True) + eps).sqrt()


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("rows,width,hidden", [(40, 64, 160), (70, 96, 520)])
def test_gradients_of_blocks_from_what_they_keep(norm, rows, width, hidden):
    """fp32.  The reference differentiates the blocks in 64 bits with the layers' inputs and pre-activations replaced by what the checkpoints hold.  Sums of at most
    600 products are within 700 2^-24 = 4.2e-5 of their magnitudes; two blocks, each two products and four norms deep, whose factors are of order 1,
    stay below 24 times that, 1e-3, of a gradient's largest value."""
    import torch
    from paper_2012_15667_amd import binding as B
    from paper_2012_15667_amd.block import Blocks
    model = Blocks(width, hidden, 2, torch.float32, norm, 0.25, 0.9, seed=5)
    g = torch.Generator(device="cuda")
    g.manual_seed(2)
    for w in model.blocks:
        for t in w[4:]:
            t.add_(0.2 * torch.randn(t.shape, generator=g, device="cuda"))
    x = torch.randn((rows, width), generator=g, device="cuda")
    dn = torch.randn((rows, width), generator=g, device="cuda")
    n, kept = model.forward(x, step=3)
    dx, dfirst, grads = model.backward(dn, x, kept, step=3)

    class Gelu(torch.autograd.Function):
        """gelu of the value itself, its slope at what the checkpoint holds."""
        @staticmethod
        def forward(ctx, z, held):
            ctx.save_for_backward(held)
            return z * torch.special.ndtr(z)

        @staticmethod
        def backward(ctx, d):
            z, = ctx.saved_tensors
            return d * (torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / (2 * np.pi) ** 0.5), None

    class Linear(torch.autograd.Function):
        """x w^T + b; the weights' gradient from what the input's checkpoint holds."""
        @staticmethod
        def forward(ctx, x, w, b, held):
            ctx.save_for_backward(w, held)
            return x @ w.T + b

        @staticmethod
        def backward(ctx, d):
            w, held = ctx.saved_tensors
            return d @ w, d.T @ held, d.sum(0), None

    leaves = [x.double().requires_grad_(), model.first.double().requires_grad_()] + [t.double().requires_grad_() for w in model.blocks for t in w]
    s, m = leaves[0], _hat(leaves[0], norm) * leaves[1]
    for i in range(2):
        up, up_bias, down, down_bias, wp, gate, w = leaves[2 + 7 * i:9 + 7 * i]
        n8, z8, d8 = (B.checkpoint_unpack(c).double() for c in kept[i][:3])
        a = Gelu.apply(Linear.apply(m, up, up_bias, n8), z8) * _mask((rows, hidden), 0.25, 5, 3 * 2 + i)
        h = Linear.apply(a, down, down_bias, d8)
        # the norms' statistics are of h and x' as stored, which in 32 bits are these values to 2^-24
        s = 0.9 * s + gate * (_hat(h, norm) * wp)
        m = _hat(s, norm) * w
    assert float((n.double() - m.detach()).abs().max()) <= 1e-3 * float(m.detach().abs().max())
    want = torch.autograd.grad(m, leaves, dn.double())
    for got, ref in zip([dx, dfirst, *[t for w in grads for t in w]], want):
        assert got.shape == ref.shape
        assert float((got.double() - ref).abs().max()) <= 1e-3 * float(ref.abs().max())


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_training_steps_captured_in_a_graph(dtype):
    """Forward and backward pass recorded once and replayed with other data: what eager calls give, to the last bit."""
    import torch
    from paper_2012_15667_amd.block import Blocks
    T = getattr(torch, dtype)
    model = Blocks(64, 192, 2, T, "rms", 0.2)
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x, dn = (torch.randn((50, 64), generator=g, device="cuda").to(T) for _ in range(2))

    def step():
        n, kept = model.forward(x, 7)
        dx, dfirst, grads = model.backward(dn, x, kept, 7)
        return [n, dx, dfirst, *[t for w in grads for t in w]]
    step()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for turn in range(3):
        x.copy_(torch.randn((50, 64), generator=g, device="cuda").to(T))
        dn.copy_(torch.randn((50, 64), generator=g, device="cuda").to(T))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(step(), held)), turn


@pytest.mark.parametrize("rows", [1, 16, 40])
def test_answers_in_4_bits_are_those_of_the_values_that_4_bits_hold(rows):
    """fp32: each layer's product of the values that its operands' 4 bits stand for, 3e-5 of its magnitudes; the same steps in 64 bits would differ where a
    value lies beside the middle of two codes, so each layer is compared from the input that it had."""
    import torch
    from paper_2012_15667_amd import binding as B
    from paper_2012_15667_amd.block import Blocks
    model = Blocks(128, 320, 2, torch.float32, "rms")
    g = torch.Generator(device="cuda")
    g.manual_seed(4)
    x = torch.randn((rows, 128), generator=g, device="cuda")
    got = model.answer(x, in_4_bits=True)
    n = B.block_norm(x, pre="rms", pre_weight=model.first).y
    s = x
    for i, w in enumerate(model.blocks):
        up, down = model.in_4_bits[i]
        a = B.linear_mx4(n, up, w.up_bias, act="gelu")
        h = B.linear_mx4(a, down, w.down_bias)
        for y, inp, four, act in ((a, n, up, True), (h, a, down, False)):
            xv, wv = B.mx4_unpack(B.mx4_pack(inp)).double(), B.mx4_unpack(four).double()
            z = xv @ wv.T
            want = z * torch.special.ndtr(z) if act else z
            assert bool(((y.double() - want).abs() <= 1.13 * 340 * 2.0 ** -24 * (xv.abs() @ wv.abs().T) + 2e-6 * want.abs() + 2e-7).all())
        s, n = B.block_norm(s, h, **model._end(w))
    assert torch.equal(got, n)


def test_gradients_of_the_head_with_dropout():
    """As without dropout (test_dense_head.py), the hidden layers' outputs from the checkpoints of what dropout left: 2e-4 of a gradient's largest value."""
    import torch
    from paper_2012_15667_amd import binding as B
    from paper_2012_15667_amd import head as H
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    x = torch.rand((20, 600), generator=g, device="cuda")
    labels = torch.randint(0, 17, (20,), generator=g, device="cuda")
    head = H.Head(600, 96, 17)
    logits, kept = head.forward(x, 0.5, 9, 4)
    _, slope = H.loss_and_slope(logits, labels)
    grads, dx = head.backward(slope, kept)
    x8, z1, z2, d1, d2 = (B.checkpoint_unpack(c).double() for c in kept[:5])
    m1, m2 = _mask((20, 96), 0.5, 9, 8), _mask((20, 96), 0.5, 9, 9)
    (w1, _), (w2, _), (w3, _) = [(w.double(), b.double()) for w, b in head.layers]
    e3 = slope.double()
    e2 = (e3 @ w3) * m2 * (z2 > 0)
    e1 = (e2 @ w2) * m1 * (z1 > 0)
    for (dw, db), e, inp in zip(grads, (e1, e2, e3), (x8, d1, d2)):
        for got, ref in ((dw, e.T @ inp), (db, e.sum(0))):
            assert float((got.double() - ref).abs().max()) <= 2e-4 * float(ref.abs().max())
    assert float((dx.double() - e1 @ w1).abs().max()) <= 2e-4 * float((e1 @ w1).abs().max())
    # what is kept is what dropout left of the layers' outputs, to half a unit of the checkpoint
    y1 = B.linear(x, *head.layers[0], act="relu").double() * m1
    assert float((y1 - d1).abs().max()) <= float(y1.abs().max()) / 127 + 1e-6
    assert not bool((d1 != 0)[m1 == 0].any())


def test_the_commands_run(capsys):
    from paper_2012_15667_amd import block, head
    block.main(["--rows", "33", "--width", "64", "--steps", "2", "--dtype", "float16"])
    block.main(["--rows", "20", "--width", "72", "--hidden", "100", "--blocks", "1", "--norm", "layer", "--steps", "1", "--dtype", "float32"])
    block.main(["--one-token", "--width", "64"])
    small = ["--channels", "32", "--size", "8", "--hidden", "64", "--classes", "10"]
    head.main(["--batch", "6", "--steps", "2", "--dtype", "bfloat16", "--dropout", "0.5", *small])
    head.main(["--one-image", "--mx4", *small])
    assert capsys.readouterr().out.count("{") == 8
