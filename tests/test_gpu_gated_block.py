"""The gated block's step and the blocks on 8-bit integers as they are used: against their definitions in 64 bits, on a stream, in graphs,
and from training to 8 bits."""
import math
import os
import sys

import pytest
import torch

from paper_2509_26277_amd import (cat_gated_backward_input, cat_gated_linear, cat_gated_linear8, cat_layer_norm_quantize, cat_linear8,
                                  cat_quantize_rows, cat_unpack8)
from paper_2509_26277_amd.block import block_backward, block_forward, block_forward8, quantize_block

from block_util import ACTS, TYPES, act_ref, norm_backward_ref, norm_ref, unpack_ref

pytestmark = pytest.mark.gpu


def _params(D, F, dtype, seed, gated):
    g = torch.Generator().manual_seed(seed)
    wide = 2 * F if gated else F

    def n(*shape, scale):
        return torch.randn(*shape, generator=g) * scale

    p = dict(norm_weight=1.0 + n(D, scale=0.2), norm_bias=n(D, scale=0.1), w1=n(wide, D, scale=D ** -0.5).to(dtype), b1=n(wide, scale=0.1),
             w2=n(D, F, scale=F ** -0.5).to(dtype), b2=n(D, scale=0.1))
    return {k: v.cuda() for k, v in p.items()}, g


def _reference(x, dy, p, act, x8, z8):
    """In 64 bits, the checkpoints' values in the places where the step reads them."""
    p = {k: v.double().cpu() for k, v in p.items()}
    x, dy = x.double().cpu(), dy.double().cpu()
    F = p["w2"].shape[1]
    h, mean, rstd = norm_ref(x, p["norm_weight"], p["norm_bias"], 1e-5)
    z = h @ p["w1"].t() + p["b1"]
    y = x + (act_ref(z[:, :F], act)[0] * z[:, F:]) @ p["w2"].t() + p["b2"]
    gate, value = (unpack_ref(c, s) for c, s in zip(*z8))
    u, du = act_ref(gate, act)
    xh = (unpack_ref(*x8) - mean[:, None]) * rstd[:, None]
    dh = dy @ p["w2"]
    dz = torch.cat((dh * value * du, dh * u), 1)
    dx, dg, db = norm_backward_ref(dz @ p["w1"], xh, rstd, p["norm_weight"])
    h8 = xh * p["norm_weight"] + p["norm_bias"]
    return y, dx + dy, dict(norm_weight=dg, norm_bias=db, w1=dz.t() @ h8, b1=dz.sum(0), w2=dy.t() @ (u * value), b2=dy.sum(0))


def _off(got, want):
    """Root mean square of the difference, in units of the values'."""
    return float((got.double().cpu() - want).norm() / want.norm().clamp(min=1e-300))


# (as for the step without a gate: no more than six independent roundings in a row, half a step at most each)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,F,act", [(1, 8, 16, "silu"), (3, 33, 65, "gelu"), (70, 128, 256, "relu"), (300, 100, 250, "gelu_tanh"), (1030, 256, 700, "none"),
                                       (2100, 256, 1032, "silu")])
def test_gated_step(M, D, F, act, dtype):
    assert act in ACTS
    t = TYPES[dtype]
    p, g = _params(D, F, t, M, True)
    x, dy = torch.randn(M, D, generator=g).to(t).cuda(), (0.1 * torch.randn(M, D, generator=g)).to(t).cuda()
    y, saved = block_forward(x, p, act=act)
    dx, grads = block_backward(dy, p, saved)
    want_y, want_dx, want = _reference(x, dy, p, act, saved["x8"], saved["z8"])
    tol = 6 * torch.finfo(t).eps / 2 + 2 * math.sqrt(max(4 * D, M)) * 2.0 ** -24 + 64 * 2.0 ** -24
    assert _off(block_forward(x, p, act=act, keep=False)[0], want_y) < tol
    assert _off(y, want_y) < tol
    assert _off(dx, want_dx) < tol
    assert grads.keys() == p.keys()
    for k in p:
        assert grads[k].shape == p[k].shape and grads[k].dtype == p[k].dtype
        assert _off(grads[k], want[k]) < tol, k


def test_gated_gradients_against_differences():
    """The whole step's, within what 8 bits of the checkpoints leave (their steps are 1 / 127 of a group's largest value: the
    gradient moves by some 1 %, of two of them; a wrong term moves it by its own size)."""
    D, F, M = 32, 96, 64
    p, g = _params(D, F, torch.float32, 5, True)
    x, dy = torch.randn(M, D, generator=g).cuda(), torch.randn(M, D, generator=g).cuda()
    dx, grads = block_backward(dy, p, block_forward(x, p, act="silu")[1])
    q = {k: v.double().cpu() for k, v in p.items()}

    def f(x, q):
        z = norm_ref(x, q["norm_weight"], q["norm_bias"], 1e-5)[0] @ q["w1"].t() + q["b1"]
        return float((dy.double().cpu() * (x + (act_ref(z[:, :F], "silu")[0] * z[:, F:]) @ q["w2"].t() + q["b2"])).sum())

    e, x = 1e-5, x.double().cpu()
    for k in [None, *p]:
        at, got = (x, dx) if k is None else (q[k], grads[k])
        for _ in range(3):
            d = torch.randn(at.shape, generator=g).double()
            hi, lo = at + e * d, at - e * d
            slope = (f(hi, q) - f(lo, q)) if k is None else (f(x, {**q, k: hi}) - f(x, {**q, k: lo}))
            assert abs(slope / (2 * e) - float((got.double().cpu() * d).sum())) < 0.05 * float(got.double().norm()), k


@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,D,act", [(1, 64, "gelu"), (37, 100, "silu"), (300, 256, "gelu_tanh")])
def test_block_on_8_bit_integers(M, D, act, dtype, gated):
    """Against the block in full precision.  A row in 8 bits is off by a step's root mean square, a / 127 / sqrt(12); the largest entry a
    of a row is below 6 of its root mean squares for norm's rows and weights (5.5 is one in 3e7), below 14 for products of two: 1.4 % of
    h, of both weights (the gate's path and the value's: twice) and 3.2 % of u, together at most 4.4 % of what the block adds to x."""
    t = TYPES[dtype]
    p, g = _params(D, 4 * D, t, M, gated)
    x = torch.randn(M, D, generator=g).to(t).cuda()
    q = quantize_block(p)
    y = block_forward8(x, q, act=act)
    assert y.dtype == t and q["w1"].dtype == torch.int8 and q["w2_scales"].shape == (D,)
    full = block_forward(x.float(), {k: v.float() for k, v in p.items()}, act=act, keep=False)[0].double().cpu()
    added = full - x.double().cpu()
    assert float((y.double().cpu() - full).norm() / added.norm()) < 0.044 + 4 * torch.finfo(t).eps * float(full.norm() / added.norm())
    # and it is what its calls give
    h = cat_layer_norm_quantize(x, q["norm_weight"], q["norm_bias"])
    u = (cat_gated_linear8 if gated else cat_linear8)(*h, q["w1"], q["w1_scales"], q["b1"], act=act, dtype=t)
    assert torch.equal(cat_linear8(*cat_quantize_rows(u), q["w2"], q["w2_scales"], q["b2"], residual=x, dtype=t), y)


def _step(x, dy, p, q):
    y, saved = block_forward(x, p, act="silu")
    dx, grads = block_backward(dy, p, saved)
    return [y, dx, *grads.values(), block_forward8(x, q, act="silu")]


@pytest.mark.parametrize("M,D,F", [(40, 96, 200), (300, 96, 200), (1, 33, 7), (131, 131, 1027), (2100, 131, 1027)])
def test_on_a_stream_and_in_graphs(M, D, F):
    """On a stream of its own, and in two graphs captured one after the other, replayed in turn with eager work between: every replay,
    on new inputs, gives the eager calls' bits."""
    p, g = _params(D, F, torch.bfloat16, 3, True)
    q = quantize_block(p)
    inputs = [[torch.randn(M, D, generator=g).bfloat16().cuda() for _ in range(2)] for _ in range(2)]
    eager = _step(*inputs[0], p, q)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = _step(*inputs[0], p, q)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    graphs = []
    for x, dy in inputs:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            out = _step(x, dy, p, q)
        graphs.append((graph, out))
    for k in range(4):
        for (x, dy), (graph, out) in zip(inputs, graphs):
            x.copy_(torch.randn(M, D, generator=g).bfloat16())
            dy.copy_(torch.randn(M, D, generator=g).bfloat16())
            want = _step(x, dy, p, q)
            graph.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(want, out)), f"replay {k}"


def test_two_streams_at_once():
    """The same calls on two streams, with workspaces of their own: neither sees the other's."""
    p, g = _params(256, 512, torch.bfloat16, 9, True)
    q = quantize_block(p)
    x = [torch.randn(700, 256, generator=g).bfloat16().cuda() for _ in range(2)]
    want = [_step(a, a, p, q) for a in x]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in x]
    got = [None, None]
    for _ in range(3):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i] = _step(x[i], x[i], p, q)
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(u, v) for u, v in zip(a, b))


def test_refusals_of_what_is_not_a_plain_matrix():
    x, w = torch.randn(64, 96, device="cuda"), torch.randn(40, 96, device="cuda")
    for bad in (x.t(), x[:, ::2], x[:, :40]):
        for call in (cat_quantize_rows, cat_layer_norm_quantize, lambda t: cat_gated_linear(t, w)):
            with pytest.raises(ValueError):
                call(bad)
    q, s = cat_quantize_rows(x)
    v, t = cat_quantize_rows(w)
    with pytest.raises(ValueError):
        cat_linear8(q, s[:10].contiguous(), v, t)
    with pytest.raises(ValueError):
        cat_linear8(q, s, v[:, :90].contiguous(), t)
    with pytest.raises(TypeError):
        cat_linear8(q.to(torch.uint8), s, v, t)
    with pytest.raises(ValueError):
        cat_linear8(q, s, v, t, out=torch.empty(64, 41, device="cuda", dtype=torch.bfloat16))
    with pytest.raises(ValueError):
        cat_linear8(q, s, v, t.cpu())
    with pytest.raises(ValueError, match="activation"):
        cat_gated_linear(x, w, act="tanh")
    _, packed = cat_gated_linear(x, w, pack=True)
    with pytest.raises(ValueError):
        cat_gated_backward_input(x, torch.randn(96, 21, device="cuda"), packed)
    with pytest.raises(TypeError):
        cat_gated_backward_input(x, torch.randn(96, 20, device="cuda").bfloat16(), packed)


def test_halves_of_a_checkpoint_decode_wherever_they_start():
    """The value's checkpoint begins where the gate's ends: on any byte."""
    x, w = torch.randn(5, 24, device="cuda"), torch.randn(2 * 13, 24, device="cuda")
    _, (codes, scales) = cat_gated_linear(x, w, act="none", pack=True)
    assert codes[1].data_ptr() % 16
    for c, k in zip(codes, scales):
        for t in TYPES.values():
            assert torch.equal(cat_unpack8(c, k, dtype=t).cpu(), unpack_ref(c, k).float().to(t))


def test_example():
    sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))
    try:
        from fit_block import fit_block
    finally:
        sys.path.pop(0)
    said = []
    values = fit_block(rows=512, dim=64, steps=2, gated=True, integers=True, say=said.append)
    assert len(values) == 3 and all(math.isfinite(v) and v > 0 for v in values) and len(said) == 1
