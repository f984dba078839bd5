"""A block's step through the library against its definition in 64 bits, and the example that trains with it."""
import math
import os
import sys

import pytest
import torch

from paper_2509_26277_amd.block import block_backward, block_forward

from block_util import ACTS, TYPES, act_ref, norm_backward_ref, norm_ref, unpack_ref

pytestmark = pytest.mark.gpu


def _params(D, F, dtype, seed):
    g = torch.Generator().manual_seed(seed)

    def n(*shape, scale):
        return torch.randn(*shape, generator=g) * scale

    p = dict(norm_weight=1.0 + n(D, scale=0.2), norm_bias=n(D, scale=0.1), w1=n(F, D, scale=D ** -0.5).to(dtype), b1=n(F, scale=0.1),
             w2=n(D, F, scale=F ** -0.5).to(dtype), b2=n(D, scale=0.1))
    return {k: v.cuda() for k, v in p.items()}, g


def _reference(x, dy, p, act, x8, z8):
    """In 64 bits, the checkpoints' values in the places where the step reads them."""
    p = {k: v.double().cpu() for k, v in p.items()}
    x, dy = x.double().cpu(), dy.double().cpu()
    h, mean, rstd = norm_ref(x, p["norm_weight"], p["norm_bias"], 1e-5)
    z = h @ p["w1"].t() + p["b1"]
    y = x + act_ref(z, act)[0] @ p["w2"].t() + p["b2"]
    u, du = act_ref(unpack_ref(*z8), act)
    xh = (unpack_ref(*x8) - mean[:, None]) * rstd[:, None]
    dz = (dy @ p["w2"]) * du
    dx, dg, db = norm_backward_ref(dz @ p["w1"], xh, rstd, p["norm_weight"])
    h8 = xh * p["norm_weight"] + p["norm_bias"]
    return y, dx + dy, dict(norm_weight=dg, norm_bias=db, w1=dz.t() @ h8, b1=dz.sum(0), w2=dy.t() @ u, b2=dy.sum(0))


def _off(got, want):
    """Root mean square of the difference, in units of the values'."""
    got = got.double().cpu()
    return float((got - want).norm() / want.norm().clamp(min=1e-300))


# The step's roundings in a row (norm's output, the first product's, the second's, and as many backwards) are independent of one
# another: no more than six of them, each half a step at most, add up in root mean square to 6 half steps at the very most.
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,act", [(1, 8, "gelu"), (3, 33, "silu"), (70, 128, "relu"), (300, 100, "gelu_tanh"), (1030, 256, "none")])
def test_step(M, D, act, dtype):
    assert act in ACTS
    t = TYPES[dtype]
    p, g = _params(D, 4 * D, t, M)
    x, dy = torch.randn(M, D, generator=g).to(t).cuda(), (0.1 * torch.randn(M, D, generator=g)).to(t).cuda()
    y, saved = block_forward(x, p, act=act)
    dx, grads = block_backward(dy, p, saved)
    assert torch.equal(block_forward(x, p, act=act, keep=False)[0], y)
    want_y, want_dx, want = _reference(x, dy, p, act, saved["x8"], saved["z8"])
    # fp32: sums of up to 4 D products, of both passes
    tol = 6 * torch.finfo(t).eps / 2 + 2 * math.sqrt(max(4 * D, M)) * 2.0 ** -24 + 64 * 2.0 ** -24
    assert _off(y, want_y) < tol
    assert _off(dx, want_dx) < tol
    assert grads.keys() == p.keys()
    for k in p:
        assert grads[k].shape == p[k].shape and grads[k].dtype == p[k].dtype
        assert _off(grads[k], want[k]) < tol, k


def test_gradients_against_differences():
    """The whole step's, within what 8 bits of the checkpoints leave (their steps are 1 / 127 of a group's largest value: the
    gradient moves by some 1 %; a wrong term moves it by its own size)."""
    D, M = 32, 64
    p, g = _params(D, 4 * D, torch.float32, 5)
    x, dy = torch.randn(M, D, generator=g).cuda(), torch.randn(M, D, generator=g).cuda()
    dx, grads = block_backward(dy, p, block_forward(x, p)[1])
    q = {k: v.double().cpu() for k, v in p.items()}

    def f(x, q):
        h = norm_ref(x, q["norm_weight"], q["norm_bias"], 1e-5)[0]
        return float((dy.double().cpu() * (x + act_ref(h @ q["w1"].t() + q["b1"], "gelu")[0] @ q["w2"].t() + q["b2"])).sum())

    e = 1e-5
    for k in [None, *p]:
        at, got = (x.double().cpu(), dx) if k is None else (q[k], grads[k])
        for _ in range(3):
            d = torch.randn(at.shape, generator=g).double()
            hi, lo = at + e * d, at - e * d
            slope = (f(hi, q) - f(lo, q)) if k is None else (f(x.double().cpu(), {**q, k: hi}) - f(x.double().cpu(), {**q, k: lo}))
            # a random direction sees the whole gradient: its error there is the gradient's, in units of its norm
            assert abs(slope / (2 * e) - float((got.double().cpu() * d).sum())) < 0.05 * float(got.double().norm()), k


def test_example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    try:
        from fit_block import fit_block
    finally:
        sys.path.pop(0)
    quantised, fitted, corrected = fit_block(rows=2048, dim=64, steps=20)
    assert fitted < quantised and corrected < fitted * (1 + 2.0 ** -8)
