"""Fits the weight-quantised feed-forward half of a transformer block to its full-precision outputs, then corrects what is left
cluster by cluster.

    python examples/fit_block.py [--rows 8192] [--dim 256] [--steps 40] [--bits 4]

The half block (norm, two products, residual; ``paper_2509_26277_amd/block.py``) runs in bfloat16 with weights of a few bits a
row; its gradients come from checkpoints in 8 bits and go straight through the quantiser to the float weights.  The
outputs of the fitted block are the low-bit rows of ``cat_fit``, those of the full-precision block its targets.  Weights and
calibration rows are drawn at random.  Prints the mean squared error to the full-precision outputs after each stage.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2509_26277_amd import cat_apply, cat_fit  # noqa: E402
from paper_2509_26277_amd.block import block_backward, block_forward  # noqa: E402

MATRICES = ("w1", "w2")


def random_block(D, F, g):
    def normal(*shape, scale):
        return torch.randn(*shape, generator=g, device="cuda") * scale

    return dict(norm_weight=1.0 + normal(D, scale=0.1), norm_bias=normal(D, scale=0.1), w1=normal(F, D, scale=D ** -0.5),
                b1=normal(F, scale=0.1), w2=normal(D, F, scale=F ** -0.5), b2=normal(D, scale=0.1))


def quantised(w, bits):
    """Symmetric, one scale a row."""
    top = 2 ** (bits - 1) - 1
    step = w.abs().amax(1, keepdim=True).clamp(min=1e-12) / top
    return (torch.round(w / step).clamp(-top, top) * step).bfloat16()


def deployed(p, bits):
    """What the kernels take: matrices in bfloat16 (of a few bits, or of all), the rest as it is."""
    return {k: (quantised(v, bits) if bits else v.bfloat16()) if k in MATRICES else v for k, v in p.items()}


def fit_block(rows=8192, dim=256, steps=40, bits=4, lr=5e-4, clusters=8, seed=0, say=print):
    g = torch.Generator(device="cuda").manual_seed(seed)
    full = random_block(dim, 4 * dim, g)
    x = torch.randn(rows, dim, generator=g, device="cuda").bfloat16()
    target = block_forward(x, deployed(full, None), keep=False)[0]
    p = {k: v.clone() for k, v in full.items()}
    mean = {k: torch.zeros_like(v) for k, v in p.items()}
    square = {k: torch.zeros_like(v) for k, v in p.items()}
    errors = []
    for step in range(1, steps + 1):
        q = deployed(p, bits)
        y, saved = block_forward(x, q)
        off = y.float() - target.float()
        errors.append((off * off).mean())
        _, grads = block_backward((off * (2.0 / dim)).bfloat16(), q, saved)
        rate = lr * (1 - (step - 1) / steps)  # to zero: at a constant rate the rounded weights go on changing back and forth
        for k, v in p.items():  # Adam
            d = grads[k].float()
            mean[k].lerp_(d, 0.1)
            square[k].lerp_(d * d, 0.01)
            v -= rate * (mean[k] / (1 - 0.9 ** step)) / ((square[k] / (1 - 0.99 ** step)).sqrt() + 1e-8)
    y = block_forward(x, deployed(p, bits), keep=False)[0]
    m = cat_fit(y, target, clusters, 20, seed=seed)
    corrected, _ = cat_apply(y, m["centroids"], m["gamma"], m["beta"], alpha=1.0)
    mse = [float(errors[0]), float((y.float() - target.float()).square().mean()),
           float((corrected.float() - target.float()).square().mean())]
    say("mean squared error: quantised %.5f, fitted %.5f, corrected %.5f" % tuple(mse))
    return mse


if __name__ == "__main__":
    a = argparse.ArgumentParser()
    for name, value in (("rows", 8192), ("dim", 256), ("steps", 40), ("bits", 4)):
        a.add_argument("--" + name, type=int, default=value)
    fit_block(**vars(a.parse_args()))
