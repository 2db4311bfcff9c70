"""The dense head of a convolutional network, trained with its activations held in 8 bits.

The last convolution layer of a VGG-shaped network (Winograd, as the library runs it), 2 x 2 pooling, and three dense layers on
the dense-layer operators: features -> hidden -> hidden -> classes with ReLU between them.  What the forward pass keeps for the
backward pass is the 8-bit checkpoint of the features and of the two hidden layers' pre-activations, a byte and a 32nd for each value;
the hidden layers' outputs are recomputed from the checkpoints (x_act="relu") and not kept.

    python -m paper_2012_15667_amd.head                                # one batch, a few steps of gradient descent
    python -m paper_2012_15667_amd.head --batch 64 --hidden 4096 --dtype bfloat16
    python -m paper_2012_15667_amd.head --one-image                    # latency of the head on a single image

Synthetic images and labels; one JSON line a step.
"""
import argparse
import json
import math
import time

import torch

from . import binding as B


class Head:
    """Weights of the three layers, as linear() takes them: [outputs][inputs]."""

    def __init__(self, features, hidden, classes, dtype=torch.float32, seed=0):
        g = torch.Generator(device="cuda")
        g.manual_seed(seed)

        def layer(n, k):
            w = torch.randn((n, k), generator=g, device="cuda") * math.sqrt(2.0 / k)
            return w.to(dtype), torch.zeros((n,), device="cuda", dtype=dtype)

        self.layers = [layer(hidden, features), layer(hidden, hidden), layer(classes, hidden)]

    def infer(self, x):
        (w1, b1), (w2, b2), (w3, b3) = self.layers
        return B.linear(B.linear(B.linear(x, w1, b1, act="relu"), w2, b2, act="relu"), w3, b3)

    def forward(self, x):
        """(logits, what the backward pass needs: three checkpoints)."""
        (w1, b1), (w2, b2), (w3, b3) = self.layers
        x8 = B.checkpoint_pack(x)
        y1, z1 = B.linear(x, w1, b1, act="relu", checkpoint=True)
        y2, z2 = B.linear(y1, w2, b2, act="relu", checkpoint=True)
        return B.linear(y2, w3, b3), (x8, z1, z2)

    def backward(self, dlogits, kept):
        """[(dw, db)] of the three layers, and dx."""
        x8, z1, z2 = kept
        (w1, _), (w2, _), (w3, _) = self.layers
        g3 = B.linear_backward(dlogits, w3, z2, x_act="relu")
        g2 = B.linear_backward(g3.dx, w2, z1, z2, act="relu", x_act="relu")
        g1 = B.linear_backward(g2.dx, w1, x8, z1, act="relu")
        return [(g.dw, g.db) for g in (g1, g2, g3)], g1.dx

    def descend(self, grads, rate):
        for (w, b), (dw, db) in zip(self.layers, grads):
            w.add_(dw, alpha=-rate)
            b.add_(db, alpha=-rate)


def features_of(images, kernels, dtype):
    """The network's last convolution layer, ReLU and 2 x 2 pooling, one row of features an image."""
    y = B.conv_winograd(images, kernels, 2).clamp_(min=0)
    n, k, h, w = y.shape
    return y.view(n, k, h // 2, 2, w // 2, 2).amax((3, 5)).reshape(n, -1).to(dtype)


def loss_and_slope(logits, labels):
    """Cross entropy of the batch's mean, and its gradient with respect to the logits."""
    p = logits.float()
    p = p - p.amax(1, keepdim=True)
    log_sum = p.exp().sum(1, keepdim=True).log()
    rows = torch.arange(labels.numel(), device=labels.device)
    loss = (log_sum[:, 0] - p[rows, labels]).mean()
    slope = (p - log_sum).exp()
    slope[rows, labels] -= 1
    return loss, (slope / labels.numel()).to(logits.dtype)


def bytes_of(kept):
    return sum(t.numel() * t.element_size() for c in kept for t in c)


def main(argv=None):
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--batch", type=int, default=64)
    ap.add_argument("--channels", type=int, default=512)
    ap.add_argument("--size", type=int, default=14, help="edge of the last convolution layer's images")
    ap.add_argument("--hidden", type=int, default=4096)
    ap.add_argument("--classes", type=int, default=1000)
    ap.add_argument("--steps", type=int, default=8)
    ap.add_argument("--rate", type=float, default=0.002)
    ap.add_argument("--dtype", default="float32", choices=["float32", "float16", "bfloat16"])
    ap.add_argument("--one-image", action="store_true")
    a = ap.parse_args(argv)
    dtype = getattr(torch, a.dtype)
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    n = 1 if a.one_image else a.batch
    images = torch.rand((n, a.channels, a.size, a.size), generator=g, device="cuda")
    kernels = torch.randn((a.channels, a.channels, 3, 3), generator=g, device="cuda") * math.sqrt(2.0 / (9 * a.channels))
    labels = torch.randint(0, a.classes, (n,), generator=g, device="cuda")
    x = features_of(images, kernels, dtype)
    head = Head(x.shape[1], a.hidden, a.classes, dtype)
    if a.one_image:
        for _ in range(3):
            head.infer(x)
        torch.cuda.synchronize()
        began = time.perf_counter()
        for _ in range(100):
            head.infer(x)
        torch.cuda.synchronize()
        print(json.dumps({"one_image_us": round((time.perf_counter() - began) * 1e4, 1), "dtype": a.dtype}))
        return
    for step in range(a.steps):
        torch.cuda.synchronize()
        began = time.perf_counter()
        logits, kept = head.forward(x)
        loss, slope = loss_and_slope(logits, labels)
        grads, _ = head.backward(slope, kept)
        head.descend(grads, a.rate)
        torch.cuda.synchronize()
        print(json.dumps({"step": step, "loss": round(float(loss), 4), "ms": round((time.perf_counter() - began) * 1e3, 3),
                          "kept_bytes": bytes_of(kept), "dtype": a.dtype}), flush=True)


if __name__ == "__main__":
    main()
