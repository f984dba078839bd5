"""The feed-forward half of a transformer block as a training step: y = x + act(norm(x) w1^T + b1) w2^T + b2, or gated,
y = x + (act(norm(x) wg^T + bg) * (norm(x) wv^T + bv)) w2^T + b2, where w1 holds the rows of wg and then those of wv (b1 likewise);
and the same on 8-bit integers, as it runs quantised.

What the backward pass reads again is kept in 8 bits: the rows x and the pre-activation z = norm(x) w1^T + b1, with the rows'
statistics; a quarter of the bytes of x, norm(x), z and act(z) in bfloat16.  norm(x) is made again from the checkpoint of x,
act(z) from the one of z.

Parameters are a dict: ``norm_weight``, ``norm_bias`` (float32, D), ``w1`` (F x D), ``b1`` (float32, F), ``w2`` (D x F),
``b2`` (float32, D); the matrices are of the rows' type.  Gradients come as a dict of the same names.  A block is gated if w1 and b1
have 2 F rows to the F columns of w2.
"""
from .binding import (cat_gated_backward_input, cat_gated_backward_weight, cat_gated_linear, cat_gated_linear8, cat_layer_norm,
                      cat_layer_norm_backward, cat_layer_norm_packed, cat_layer_norm_quantize, cat_linear, cat_linear8,
                      cat_linear_backward_input, cat_linear_backward_weight, cat_quantize_rows)


def _gated(p):
    return p["w1"].shape[0] == 2 * p["w2"].shape[1]


def block_forward(x, p, act="gelu", eps=1e-5, keep=True):
    """(y, saved) for rows x (M x D); ``saved`` is what block_backward takes, None without ``keep``."""
    if not keep:
        h = cat_layer_norm(x, p["norm_weight"], p["norm_bias"], eps=eps)
        u = cat_gated_linear(h, p["w1"], p["b1"], act=act) if _gated(p) else cat_linear(h, p["w1"], p["b1"], act=act)
        return cat_linear(u, p["w2"], p["b2"], residual=x), None
    h, mean, rstd, x8 = cat_layer_norm(x, p["norm_weight"], p["norm_bias"], eps=eps, pack=True)
    u, z8 = (cat_gated_linear if _gated(p) else cat_linear)(h, p["w1"], p["b1"], act=act, pack=True)
    return cat_linear(u, p["w2"], p["b2"], residual=x), dict(x8=x8, z8=z8, mean=mean, rstd=rstd, act=act)


def block_backward(dy, p, saved):
    """(dx, gradients) for the gradient dy of block_forward's rows."""
    act, x8, z8, mean, rstd = (saved[k] for k in ("act", "x8", "z8", "mean", "rstd"))
    g = {}
    gated = _gated(p)
    if gated:
        g["w2"], g["b2"] = cat_gated_backward_weight(dy, z8, act=act)
        dz, g["b1"] = cat_gated_backward_input(dy, p["w2"], z8, act=act)
    else:
        g["w2"], g["b2"] = cat_linear_backward_weight(dy, packed=z8, act=act)
        dz = cat_linear_backward_input(dy, p["w2"], act=act, packed=z8)
    h = cat_layer_norm_packed(x8, mean, rstd, p["norm_weight"], p["norm_bias"], dtype=dy.dtype)
    if gated:  # (its bias' gradient came with dz)
        g["w1"] = cat_linear_backward_weight(dz, x=h, want_bias=False)[0]
    else:
        g["w1"], g["b1"] = cat_linear_backward_weight(dz, x=h)
    dh = cat_linear_backward_input(dz, p["w1"])
    dx, g["norm_weight"], g["norm_bias"] = cat_layer_norm_backward(dh, mean, rstd, p["norm_weight"], packed=x8, residual_grad=dy)
    return dx, g


def quantize_block(p):
    """The block on 8-bit integers, for block_forward8: both matrices as codes and a scale for every output channel."""
    q = {k: v for k, v in p.items() if k not in ("w1", "w2")}
    for k in ("w1", "w2"):
        q[k], q[k + "_scales"] = cat_quantize_rows(p[k])
    return q


def block_forward8(x, q, act="gelu", eps=1e-5):
    """block_forward's rows of a block that quantize_block gave: both products on 8-bit integers, the rows that enter them with a
    scale each; norm, activation, gate and residual as they are."""
    h, h_scales = cat_layer_norm_quantize(x, q["norm_weight"], q["norm_bias"], eps=eps)
    u = (cat_gated_linear8 if _gated(q) else cat_linear8)(h, h_scales, q["w1"], q["w1_scales"], q["b1"], act=act, dtype=x.dtype)
    u, u_scales = cat_quantize_rows(u)
    return cat_linear8(u, u_scales, q["w2"], q["w2_scales"], q["b2"], residual=x, dtype=x.dtype)
