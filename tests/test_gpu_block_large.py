"""The block's operators where shares of k meet large tiles, and on matrices of more than 2^31 entries."""
import pytest
import torch

from paper_2509_26277_amd import (cat_layer_norm, cat_layer_norm_backward, cat_linear, cat_linear_backward_input,
                                  cat_linear_backward_weight, cat_pack8, cat_unpack8)

from block_util import ACT_ERR, SLOPE, U32, act_ref, assert_close, half_step

pytestmark = pytest.mark.gpu


def _normal(M, N, seed, scale=1.0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(M, N, generator=g, device="cuda") * scale).to(dtype)


@pytest.mark.parametrize("ragged", [0, 3])
def test_shares_of_k_of_large_tiles(ragged):
    """Few large tiles and a long k, rows of whole 16-byte groups and not, in all three products."""
    n, k = 2000 + ragged, 12000
    x, w, b, res = _normal(2000, k, 1), _normal(n, k, 2, k ** -0.5), 0.3 * _normal(1, n, 3, dtype=torch.float32)[0], _normal(2000, n, 4)
    z, size = x.double() @ w.double().t() + b.double(), x.double().abs() @ w.double().abs().t() + b.double().abs()
    want = act_ref(z, "gelu")[0] + res.double()
    y = cat_linear(x, w, b, act="gelu", residual=res)
    half = half_step(torch.bfloat16)
    err = SLOPE * U32 * (k + 8) * size + ACT_ERR * (1 + z.abs()) + U32 * want.abs()
    assert_close(y, want, (half * want.abs() + err).cpu(), "y")
    assert torch.equal(cat_linear(x, w, b, act="gelu", residual=res), y)

    dy, w2 = _normal(2000, k, 5), _normal(k, n, 6, k ** -0.5)
    want, size = dy.double() @ w2.double(), dy.double().abs() @ w2.double().abs()
    assert_close(cat_linear_backward_input(dy, w2), want, (half * want.abs() + U32 * (k + 8) * size).cpu(), "dx")

    dy, x = _normal(k, 2000, 7), _normal(k, n, 8)
    want, size = dy.double().t() @ x.double(), dy.double().abs().t() @ x.double().abs()
    dw, db = cat_linear_backward_weight(dy, x=x)
    assert_close(dw, want, (half * want.abs() + U32 * (k + 8) * size).cpu(), "dw")
    assert_close(db, dy.double().sum(0), (U32 * (k + 8) * dy.double().abs().sum(0)).cpu(), "db")


@pytest.mark.parametrize("k", [8, 20, 64, 72])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_many_tiles_of_few_steps(k, dtype):
    """More tiles than workgroups, each of one step of k or two."""
    M, N = 5000, 4100
    x, w = _normal(M, k, 1, dtype=dtype), _normal(N, k, 2, k ** -0.5, dtype=dtype)
    half = half_step(dtype)

    def check(got, a, b, what):
        want, size = a.double() @ b.double(), a.double().abs() @ b.double().abs()
        assert_close(got, want, (half * want.abs() + U32 * (k + 8) * size).cpu(), what)

    check(cat_linear(x, w), x, w.t(), "y")
    check(cat_linear_backward_input(x, w.t().contiguous()), x, w.t(), "dx")
    check(cat_linear_backward_weight(x.t().contiguous(), x=w.t().contiguous())[0], x, w.t(), "dw")


def _same_rows(big, small, at):
    assert torch.equal(big[at:at + len(small)], small)


def test_more_than_2_31_entries():
    """Rows behind entry 2^31 come out as they do by themselves (norm, checkpoint), and as the definition has them (product)."""
    M, D = 262300, 8192  # 2.15e9 entries
    x = _normal(1, D, 1).expand(M, D).contiguous()
    tail = M - 70
    x[tail:] = _normal(70, D, 2)
    y, mean, rstd, packed = cat_layer_norm(x, pack=True)
    y2, mean2, rstd2, packed2 = cat_layer_norm(x[tail - 2:].clone(), pack=True)
    for a, b in ((y, y2), (mean, mean2), (rstd, rstd2), (packed[0], packed2[0]), (packed[1], packed2[1])):
        _same_rows(a, b, tail - 2)
    del y
    dx = cat_layer_norm_backward(x, mean, rstd, packed=packed, want_params=False)[0]
    _same_rows(dx, cat_layer_norm_backward(x[tail - 2:].clone(), mean2, rstd2, packed=packed2, want_params=False)[0], tail - 2)
    del dx
    _same_rows(cat_unpack8(*packed, dtype=torch.bfloat16), cat_unpack8(*packed2, dtype=torch.bfloat16), tail - 2)
    again = cat_pack8(x)
    _same_rows(again[0], packed2[0], tail - 2)
    _same_rows(again[1], packed2[1], tail - 2)
    del again, packed

    N = 72
    w = _normal(N, D, 3, D ** -0.5)  # the long operand is read behind 2^31
    want, size = x[tail:].double() @ w.double().t(), x[tail:].double().abs() @ w.double().abs().t()
    got = cat_linear(x, w)[tail:]
    assert_close(got, want, (half_step(x.dtype) * want.abs() + U32 * (D + 8) * size).cpu(), "product")
    u, w = x[:, :40].contiguous(), _normal(D, 40, 4, 0.2)  # the long one is written
    out, packed = cat_linear(u, w, pack=True)
    want, size = u[tail:].double() @ w.double().t(), u[tail:].double().abs() @ w.double().abs().t()
    err = U32 * 48 * size
    assert_close(out[tail:], want, (half_step(x.dtype) * want.abs() + err).cpu(), "long rows")
    _same_rows(packed[0], cat_linear(u[tail:].clone(), w, pack=True)[1][0], tail)
    want, size = x[tail:].double() @ w.double(), x[tail:].double().abs() @ w.double().abs()
    got = cat_linear_backward_input(x, w)[tail:]
    assert_close(got, want, (half_step(x.dtype) * want.abs() + U32 * (D + 8) * size).cpu(), "dx of long rows")
