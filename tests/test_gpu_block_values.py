"""The block's operators at values where formulas end: infinities, the largest floats, groups that hold a NaN, and activations
of either type at their precision."""
import math

import pytest
import torch

from paper_2509_26277_amd import cat_activation_backward, cat_layer_norm, cat_linear, cat_linear_backward_weight, cat_pack8, cat_unpack8

from block_util import ACT_ERR, ACTS, TYPES, U32, act_ref, assert_close, half_step, unpack_ref

pytestmark = pytest.mark.gpu

INF, NAN = float("inf"), float("nan")
FAR = [INF, -INF, NAN, 3e38, -3e38, 1e20, -1e20, 1000.0, -1000.0, 200.0, -200.0, 90.0, -90.0, 50.0, -50.0]


def test_a_checkpoint_s_activation_in_either_type():
    """With bfloat16 rows the weight's gradient takes act(c) rounded to bfloat16, as the product that took it forward did; with
    float rows it takes all of it, from the same checkpoint."""
    g = torch.Generator().manual_seed(1)
    M, N, K = 4000, 72, 200
    packed = cat_pack8(torch.randn(M, K, generator=g).cuda())
    dy = (0.01 * torch.randn(M, N, generator=g)).bfloat16().cuda()
    u = act_ref(unpack_ref(*packed), "gelu")[0]
    want = dy.double().cpu().t() @ u
    size = dy.double().cpu().abs().t() @ u.abs()
    dw = cat_linear_backward_weight(dy.float(), packed=packed, act="gelu", want_bias=False)[0]
    off = ACT_ERR * (1.0 + unpack_ref(*packed).abs())
    err = U32 * (M + 8) * size + dy.double().cpu().abs().t() @ off
    assert dw.dtype == torch.float32
    assert_close(dw, want, err, "float rows")
    rounded = dy.double().cpu().t() @ u.bfloat16().double()
    # (where act's own error reaches over a rounding's border, u may be the value on its other side)
    border = dy.double().cpu().abs().t() @ ((u + off).bfloat16().double() - (u - off).bfloat16().double())
    got = cat_linear_backward_weight(dy, packed=packed, act="gelu", want_bias=False)[0]
    assert_close(got, rounded, half_step(torch.bfloat16) * rounded.abs() + err + border, "bfloat16 rows")


@pytest.mark.parametrize("N", [128, 131])
@pytest.mark.parametrize("M", [15, 150])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_values_far_out(dtype, act, M, N):
    """One activation, whatever the type and the kernel: of -infinity GELU and SiLU are -inf * 0, a NaN."""
    z = torch.tensor(FAR).repeat(M // len(FAR))[:, None].to(TYPES[dtype]).cuda()
    y = cat_linear(z, torch.ones(N, 1, dtype=z.dtype, device="cuda"), act=act).double().cpu()
    z = z.double().cpu()[:, 0]
    for i in range(M):
        v, got = float(z[i]), y[i]
        if v != v or (v == -INF and act not in ("none", "relu")):
            assert bool(torch.isnan(got).all()), (act, v, got[0])
        elif act == "none" or v > 0:
            # (50 and more: the logistic function and the normal distribution are one but for less than a half step)
            assert bool((got == v).all()) if math.isinf(v) or act in ("none", "relu") else bool(
                ((got - v).abs() <= (4 * U32 + half_step(TYPES[dtype])) * v).all()), (act, v, got[0])
        else:
            assert bool((got.abs() < 1e-18).all()), (act, v, got[0])  # (50 e^-50 is 1e-20)


@pytest.mark.parametrize("M", [25, 150])
def test_silu_of_float_rows_is_a_float_silu(M):
    """z / (1 + exp(-z)): two half steps of the exponential and one each of the sum, the quotient and the product, at any |z|."""
    z = torch.linspace(-80.0, 80.0, M).reshape(M, 1).cuda()
    want = act_ref(z.double().cpu(), "silu")[0].expand(M, 130)
    got = cat_linear(z, torch.ones(130, 1, device="cuda"), act="silu")
    assert_close(got, want, 8 * U32 * want.abs(), "silu")


def test_derivative_of_silu_of_float_rows():
    """p (1 + z (1 - p)), p = 1 / (1 + exp(-z)) as above: the inner sum is off by a few half steps of 1 + |z|."""
    z = torch.linspace(-80.0, 80.0, 161).reshape(161, 1).cuda()  # (a row each: its checkpoint's scale is its own)
    packed = cat_pack8(z)
    held = unpack_ref(*packed).float().double()  # (the value that the kernel reads: code times scale, a float)
    p = torch.sigmoid(held)
    got = cat_activation_backward(torch.ones_like(z), packed, "silu")
    assert_close(got, act_ref(held, "silu")[1], 8 * U32 * p * (1.0 + held.abs()), "silu'")
    for act in ("gelu", "gelu_tanh"):
        got = cat_activation_backward(torch.ones_like(z), packed, act)
        assert_close(got, act_ref(held, act)[1], ACT_ERR * (1.0 + held.abs()), act)


LARGEST = torch.finfo(torch.float32).max


def test_the_largest_float_comes_back_finite():
    """As a mask's lowest value has it: 127 steps of a group's scale stay a float, from whichever kernel the group is."""
    x = torch.ones(4, 300)
    x[0, 5], x[1, 130], x[2, 299], x[2, 0] = LARGEST, -LARGEST, LARGEST, -LARGEST
    x = x.cuda()
    codes, scales = cat_pack8(x)
    for t in TYPES.values():
        y = cat_unpack8(codes, scales, dtype=t)
        # (as bfloat16 the values round to the next power of two, which is infinity)
        assert bool(torch.isfinite(cat_unpack8(codes, scales)).all())
        assert torch.equal(y, cat_unpack8(codes, scales).to(t))
    got = cat_unpack8(codes, scales).double().cpu()
    want = x.double().cpu()
    big = want.abs() > 1.0
    assert bool(((got - want).abs()[big] <= 2.0 ** -22 * LARGEST).all())
    assert bool((got[3] == 1.0).all())
    packed = cat_layer_norm(x, pack=True)[3]
    assert torch.equal(packed[0], codes) and torch.equal(packed[1], scales)
    for M in (4, 68):  # through a product with the unit matrix
        rows = x.repeat(M // 4, 1)
        packed = cat_linear(rows, torch.eye(300, device="cuda"), pack=True)[1]
        assert torch.equal(packed[0], codes.repeat(M // 4, 1)) and torch.equal(packed[1], scales.repeat(M // 4, 1))


@pytest.mark.parametrize("D", [300, 515, 3000, 9000])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_group_with_a_nan_or_an_infinity_from_the_norm(dtype, D):
    """The definition's: scales of NaN or infinity, every value of the group a NaN, the other groups as they would be."""
    x = torch.randn(5, D, generator=torch.Generator().manual_seed(D)).to(TYPES[dtype]).cuda()
    clean = cat_pack8(x)
    x[1, 130], x[2, D - 1], x[3, 0] = NAN, -INF, INF
    packed = cat_layer_norm(x, pack=True)[3]
    alone = cat_pack8(x)
    bad = torch.zeros(5, -(-D // 128), dtype=torch.bool, device="cuda")
    bad[1, 1] = bad[2, -1] = bad[3, 0] = True
    per = bad.repeat_interleave(128, 1)[:, :D]
    for codes, scales in (packed, alone):
        assert torch.equal(codes[~per], clean[0][~per]) and torch.equal(scales[~bad], clean[1][~bad])
        assert not bool(torch.isfinite(scales[bad]).any())
        assert torch.equal(torch.isnan(cat_unpack8(codes, scales)), per)


@pytest.mark.parametrize("M,N,K", [(5, 300, 40), (200, 300, 40), (200, 304, 2048), (600, 1024, 64)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_group_with_a_nan_or_an_infinity_from_a_product(dtype, M, N, K):
    g = torch.Generator().manual_seed(N)
    x, w = (torch.randn(r, K, generator=g).to(TYPES[dtype]).cuda() for r in (M, N))
    y0, clean = cat_linear(x, w, pack=True)
    x[3, 7], w[140, 0] = NAN, INF
    y, (codes, scales) = cat_linear(x, w, pack=True)
    bad = torch.zeros(M, -(-N // 128), dtype=torch.bool, device="cuda")
    bad[3] = bad[:, 1] = True
    per = bad.repeat_interleave(128, 1)[:, :N]
    assert torch.equal(codes[~per], clean[0][~per]) and torch.equal(scales[~bad], clean[1][~bad])
    assert not bool(torch.isfinite(scales[bad]).any())
    assert torch.equal(torch.isnan(cat_unpack8(codes, scales)), per)
    hit = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    hit[3] = hit[:, 140] = True
    assert torch.equal(y[~hit], y0[~hit]) and bool(torch.isnan(y[3]).all())
