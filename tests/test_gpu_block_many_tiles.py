"""Products with more tiles than workgroups, of several steps of k each, through the whole epilogue: what a workgroup carries from
one tile to the next (the bias, the residual and the derivative's argument requested ahead, the first loads of the next tile)."""
import pytest
import torch

from paper_2509_26277_amd import cat_linear, cat_linear_backward_input, cat_linear_backward_weight, cat_pack8, cat_unpack8

from block_util import ACT_ERR, ACTS, SLOPE, TYPES, U32, act_ref, half_step

pytestmark = pytest.mark.gpu

# (M, N, K): bfloat16 tiles of 256 x 256, 480 of them on 256 workgroups, rows that are whole 16-byte groups and rows that are not; the
# same out of tiles of 128 x 128 with k of 128 (two steps), 1216 and 1287 of them on 512
LARGE = [(6144, 5120, 512), (6001, 5003, 300)]
SMALL = [(4864, 4096, 128), (4867, 4099, 131)]


def _normal(M, N, dtype, seed, scale=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(M, N, generator=g, device="cuda") * scale).to(TYPES[dtype])


def _close(got, want, bound, what):
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist())


def _groups(t, reduce):
    G = -(-t.shape[1] // 128)
    return reduce(torch.nn.functional.pad(t, (0, G * 128 - t.shape[1])).view(t.shape[0], G, 128))


@pytest.mark.parametrize("dtype,act", [("bf16", a) for a in ACTS] + [("f32", "gelu"), ("f32", "silu")])
@pytest.mark.parametrize("M,N,K", LARGE + SMALL)
def test_forward(M, N, K, dtype, act):
    x, w, res = _normal(M, K, dtype, 1), _normal(N, K, dtype, 2, K ** -0.5), _normal(M, N, dtype, 3)
    b = _normal(1, N, "f32", 4)[0]
    product, size = x.double() @ w.double().t(), x.double().abs() @ w.double().abs().t() + b.double().abs()
    z = product + b.double()
    z_err = U32 * (K + 8) * size
    half = half_step(x.dtype)
    err = SLOPE * z_err + ACT_ERR * (1.0 + z.abs())
    y, packed = cat_linear(x, w, b, act=act, residual=res, pack=True)
    u = act_ref(z, act)[0]
    want = u + res.double()
    _close(y, want, half * want.abs() + err + U32 * want.abs(), "y")
    del want
    # the checkpoint: half a step of 1 / 127 of the group's largest magnitude, on top of the product's error
    top, perr = _groups(z.abs(), lambda t: t.amax(2)), _groups(z_err, lambda t: t.amax(2))
    _close(packed[1], top / 127, (perr + 4 * U32 * top) / 127, "scales")
    step, off = ((t.repeat_interleave(128, 1)[:, :N]) for t in (top / 127, perr))
    _close(cat_unpack8(*packed), z, 0.5 * step + 2 * z_err + 2 * off + 256 * U32 * step, "checkpoint")
    del step, off
    assert torch.equal(cat_linear(x, w, b, act=act, residual=res), y)
    _close(cat_linear(x, w, b, act=act), u, half * u.abs() + err, "without the residual")
    _close(cat_linear(x, w), product, half * product.abs() + z_err, "the product alone")


@pytest.mark.parametrize("dtype,act", [("bf16", a) for a in ACTS] + [("f32", "gelu"), ("f32", "gelu_tanh")])
@pytest.mark.parametrize("M,K,N", LARGE + SMALL)
def test_input_gradient(M, K, N, dtype, act):
    """M x K from a contraction over N, times the derivative at a checkpoint's values."""
    dy, w = _normal(M, N, dtype, 5), _normal(N, K, dtype, 6, N ** -0.5)
    packed = cat_pack8(_normal(M, K, dtype, 7, 2.0))
    held = cat_unpack8(*packed).double()
    product, size = dy.double() @ w.double(), dy.double().abs() @ w.double().abs()
    want = product * act_ref(held, act)[1]
    err = U32 * (N + 8) * size * SLOPE + ACT_ERR * (1.0 + held.abs()) * size
    got = cat_linear_backward_input(dy, w, act=act, packed=packed)
    _close(got, want, half_step(dy.dtype) * want.abs() + err, "dx")
    assert torch.equal(cat_linear_backward_input(dy, w, act=act, packed=packed), got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("N,K,M", LARGE + SMALL)
def test_weight_gradient(N, K, M, dtype):
    """N x K from a contraction over M rows, of rows and of a checkpoint's activation."""
    dy, x = _normal(M, N, dtype, 8), _normal(M, K, dtype, 9)
    half = half_step(dy.dtype)
    want, size = dy.double().t() @ x.double(), dy.double().abs().t() @ x.double().abs()
    dw, db = cat_linear_backward_weight(dy, x=x)
    _close(dw, want, half * want.abs() + U32 * (M + 8) * size, "dw")
    _close(db, dy.double().sum(0), U32 * (M + 8) * dy.double().abs().sum(0), "db")
    packed = cat_pack8(x)
    held = cat_unpack8(*packed).double()
    u = act_ref(held, "gelu")[0]
    want, size = dy.double().t() @ u, dy.double().abs().t() @ u.abs()
    # (with bfloat16 rows u is rounded: half a step of each term)
    u_err = half * size + dy.double().abs().t() @ (ACT_ERR * (1.0 + held.abs()))
    dw = cat_linear_backward_weight(dy, packed=packed, act="gelu", want_bias=False)[0]
    _close(dw, want, half * want.abs() + U32 * (M + 8) * size + u_err, "dw of a checkpoint")
