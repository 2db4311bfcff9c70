"""The dense head of head.py: three layers with their activations in 8 bits, against the same layers in 64 bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _setup(dtype):
    import torch
    from paper_2012_15667_amd import head as H
    g = torch.Generator(device="cuda")
    g.manual_seed(3)
    images = torch.rand((20, 24, 10, 10), generator=g, device="cuda")
    kernels = torch.randn((24, 24, 3, 3), generator=g, device="cuda") * 0.1
    labels = torch.randint(0, 17, (20,), generator=g, device="cuda")
    x = H.features_of(images, kernels, getattr(torch, dtype))
    return H, x, labels, H.Head(x.shape[1], 96, 17, getattr(torch, dtype))


def test_gradients_of_the_head_from_what_it_keeps():
    """fp32.  From the head's own checkpoints the gradients are the formula's: sums of at most 600 products, within 700 2^-24 = 4.2e-5 of
    each layer's magnitudes; three layers of them stay below 2e-4 of a gradient's largest value (norms here are well conditioned)."""
    import torch
    from paper_2012_15667_amd import binding as B
    H, x, labels, head = _setup("float32")
    logits, kept = head.forward(x)
    _, slope = H.loss_and_slope(logits, labels)
    grads, dx = head.backward(slope, kept)
    x8, z1, z2 = (B.checkpoint_unpack(c).double() for c in kept)
    (w1, _), (w2, _), (w3, _) = [(w.double(), b.double()) for w, b in head.layers]
    d3 = slope.double()
    d2 = (d3 @ w3) * (z2 > 0)
    d1 = (d2 @ w2) * (z1 > 0)
    want = [(d1.T @ x8, d1.sum(0)), (d2.T @ z1.clamp(min=0), d2.sum(0)), (d3.T @ z2.clamp(min=0), d3.sum(0))]
    for (dw, db), (ew, eb) in zip(grads, want):
        assert float((dw.double() - ew).abs().max()) <= 2e-4 * float(ew.abs().max())
        assert float((db.double() - eb).abs().max()) <= 2e-4 * float(eb.abs().max())
    assert float((dx.double() - d1 @ w1).abs().max()) <= 2e-4 * float((d1 @ w1).abs().max())
    # a byte and a 32nd for each value kept, and nothing else
    assert H.bytes_of(kept) == sum(r * (c + -(-c // 32)) for r, c in ((20, x.shape[1]), (20, 96), (20, 96)))
    del torch


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_the_head_learns(dtype):
    H, x, labels, head = _setup(dtype)
    losses = []
    for _ in range(30):
        logits, kept = head.forward(x)
        loss, slope = H.loss_and_slope(logits, labels)
        head.descend(head.backward(slope, kept)[0], 0.05)
        losses.append(float(loss))
    assert np.isfinite(losses).all() and losses[-1] < 0.5 * losses[0], losses


def test_the_command_runs(capsys):
    from paper_2012_15667_amd import head
    head.main(["--batch", "6", "--channels", "32", "--size", "8", "--hidden", "64", "--classes", "10", "--steps", "2", "--dtype", "bfloat16"])
    head.main(["--one-image", "--channels", "32", "--size", "8", "--hidden", "64", "--classes", "10"])
    assert capsys.readouterr().out.count("{") == 3
