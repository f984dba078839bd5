"""The block's operators at values where formulas end: infinities, the largest floats, groups that hold a NaN, and activations
of either type at their precision."""
import pytest
import torch

from paper_2509_26277_amd import cat_linear_backward_weight, cat_pack8

from block_util import ACT_ERR, U32, act_ref, assert_close, half_step, unpack_ref

pytestmark = pytest.mark.gpu


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
