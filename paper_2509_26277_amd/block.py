"""The feed-forward half of a transformer block as a training step: y = x + act(norm(x) w1^T + b1) w2^T + b2.

What the backward pass reads again is kept in 8 bits: the rows x and the pre-activation z = norm(x) w1^T + b1, with the rows'
statistics; a quarter of the bytes of x, norm(x), z and act(z) in bfloat16.  norm(x) is made again from the checkpoint of x,
act(z) from the one of z.

Parameters are a dict: ``norm_weight``, ``norm_bias`` (float32, D), ``w1`` (F x D), ``b1`` (float32, F), ``w2`` (D x F),
``b2`` (float32, D); the matrices are of the rows' type.  Gradients come as a dict of the same names.
"""
from .binding import (cat_layer_norm, cat_layer_norm_backward, cat_layer_norm_packed, cat_linear, cat_linear_backward_input,
                      cat_linear_backward_weight)


def block_forward(x, p, act="gelu", eps=1e-5, keep=True):
    """(y, saved) for rows x (M x D); ``saved`` is what block_backward takes, None without ``keep``."""
    if not keep:
        h = cat_layer_norm(x, p["norm_weight"], p["norm_bias"], eps=eps)
        return cat_linear(cat_linear(h, p["w1"], p["b1"], act=act), p["w2"], p["b2"], residual=x), None
    h, mean, rstd, x8 = cat_layer_norm(x, p["norm_weight"], p["norm_bias"], eps=eps, pack=True)
    u, z8 = cat_linear(h, p["w1"], p["b1"], act=act, pack=True)
    return cat_linear(u, p["w2"], p["b2"], residual=x), dict(x8=x8, z8=z8, mean=mean, rstd=rstd, act=act)


def block_backward(dy, p, saved):
    """(dx, gradients) for the gradient dy of block_forward's rows."""
    act, x8, z8, mean, rstd = (saved[k] for k in ("act", "x8", "z8", "mean", "rstd"))
    g = {}
    g["w2"], g["b2"] = cat_linear_backward_weight(dy, packed=z8, act=act)
    dz = cat_linear_backward_input(dy, p["w2"], act=act, packed=z8)
    h = cat_layer_norm_packed(x8, mean, rstd, p["norm_weight"], p["norm_bias"], dtype=dy.dtype)
    g["w1"], g["b1"] = cat_linear_backward_weight(dz, x=h)
    dh = cat_linear_backward_input(dz, p["w1"])
    dx, g["norm_weight"], g["norm_bias"] = cat_layer_norm_backward(dh, mean, rstd, p["norm_weight"], packed=x8, residual_grad=dy)
    return dx, g
