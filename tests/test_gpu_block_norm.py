"""Checkpoints in 8 bits and layer norm (forward, from a checkpoint, backward) against their definitions in 64 bits."""
import pytest
import torch

from paper_2509_26277_amd import (cat_activation_backward, cat_layer_norm, cat_layer_norm_backward, cat_layer_norm_packed, cat_pack8,
                                  cat_unpack8)

from block_util import (ACT_ERR, ACTS, TYPES, U32, act_ref, assert_close, half_step, norm_backward_ref, norm_ref, pack_ref, unpack_ref)

pytestmark = pytest.mark.gpu

# row lengths around every boundary of the kernels: 16-byte groups, lanes and waves of a row, scale groups, the longest
# row held in registers (8192), odd lengths of either type
LENGTHS = [1, 2, 7, 8, 24, 33, 63, 64, 65, 120, 128, 129, 200, 256, 257, 500, 512, 515, 1000, 1001, 1024, 1030, 2048, 2050, 4096, 4104,
           8191, 8192, 8200, 20001]


def _rows(N, D, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, D, generator=g) * torch.exp(0.5 * torch.randn(D, generator=g)) + 0.5 * torch.randn(D, generator=g)
    return (x * scale).to(TYPES[dtype]).cuda()


def _params(D, seed):
    g = torch.Generator().manual_seed(seed + 1000)
    return (1.0 + 0.3 * torch.randn(D, generator=g)).cuda(), (0.2 * torch.randn(D, generator=g)).cuda()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", LENGTHS)
def test_checkpoint_is_the_definitions(D, dtype):
    """Codes and scales bit for bit, the values that come back rounded once."""
    N = 5 if D > 4096 else 67
    x = _rows(N, D, dtype, D)
    x[0] = 0  # a group without a largest magnitude
    x[1] *= 1e-35  # below 2^-100: held as zeros
    if N > 3 and D > 2:
        x[2, D // 2] = 1000.0  # one large entry: codes of the others near zero
        x[3] = x[3].abs().max()  # all at the end of the range
    codes, scales = cat_pack8(x)
    want_c, want_s = pack_ref(x)
    assert torch.equal(scales.cpu(), want_s)
    assert torch.equal(codes.cpu(), want_c)
    for t in TYPES.values():
        want = unpack_ref(codes, scales).float().to(t)  # code * scale is one fp32 product, then the type
        assert torch.equal(cat_unpack8(codes, scales, dtype=t).cpu(), want)


def test_ties_go_to_the_even_code():
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5]], device="cuda")
    assert cat_pack8(x)[0].tolist() == [[127, 0, 2, 2, 0, -2, -2, 126]]


def test_nan_and_infinity_stay_in_their_group():
    x = _rows(4, 300, "f32", 3)
    x[1, 130], x[2, 299] = float("nan"), float("-inf")
    y = cat_unpack8(*cat_pack8(x)).cpu()
    bad = torch.zeros(4, 300, dtype=torch.bool)
    bad[1, 128:256] = bad[2, 256:] = True
    assert torch.equal(torch.isnan(y), bad)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
def test_activation_backward(act, dtype):
    z, dy = _rows(37, 333, dtype, 5, 3.0), _rows(37, 333, dtype, 6)
    packed = cat_pack8(z)
    got = cat_activation_backward(dy, packed, act)
    d = dy.double().cpu()
    want = d * act_ref(unpack_ref(*packed), act)[1]
    zmag = 1.0 + unpack_ref(*packed).abs()
    assert_close(got, want, half_step(dy.dtype) * want.abs() + ACT_ERR * zmag * d.abs(), act)


def test_activations_far_out():
    """Arguments whose powers and exponentials leave fp32 saturate instead of giving 0 * inf."""
    z = torch.tensor([[3e38, -3e38, 1e20, -1e20, 200.0, -200.0, 40.0, -40.0]], device="cuda")
    for act in ACTS:
        for i in range(z.shape[1]):  # (a row each: in one group the small ones would be zero)
            packed = cat_pack8(z[:, i:i + 1].clone())
            got = float(cat_activation_backward(torch.ones(1, 1, device="cuda"), packed, act))
            want = 1.0 if act == "none" or float(z[0, i]) > 0 else 0.0
            assert abs(got - want) < 1e-6, (act, float(z[0, i]), got)


# ---------------------------------------------------------------------------
# layer norm
# ---------------------------------------------------------------------------
CHAIN = 64  # additions one after the other in a row's sum: 32 entries of a thread and the steps across threads; long rows more


def _chain(D):
    return CHAIN if D <= 8192 else CHAIN + D // 256


def _norm_bound(x, want, w, rstd, dtype):
    """The centred entry is off by the mean's error and a rounding, of numbers the size of the row's; then a few roundings."""
    D = x.shape[1]
    size = x.abs().mean(1, keepdim=True) * _chain(D) + x.abs()
    return half_step(dtype) * want.abs() + U32 * (2 * size * rstd[:, None] * w.abs() + _chain(D) * want.abs() + 4)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", LENGTHS)
@pytest.mark.parametrize("N", [1, 67])
def test_layer_norm(N, D, dtype):
    x = _rows(N, D, dtype, D + N)
    w, b = _params(D, D)
    y, mean, rstd, packed = cat_layer_norm(x, w, b, eps=1e-3, want_stats=True, pack=True)
    xd, wd, bd = x.double().cpu(), w.double().cpu(), b.double().cpu()
    want, m, r = norm_ref(xd, wd, bd, 1e-3)
    size = xd.abs().mean(1)
    assert_close(mean, m, U32 * _chain(D) * size, "mean")
    # (an error of the mean enters the variance squared, one of a centred entry twice)
    assert_close(rstd, r, U32 * r * (_chain(D) + 4 * _chain(D) * size * r), "rstd")
    assert_close(y, want, _norm_bound(xd, want, wd, r, x.dtype), "y")
    assert torch.equal(y, cat_layer_norm(x, w, b, eps=1e-3))
    assert all(torch.equal(p, q) for p, q in zip(packed, cat_pack8(x)))
    again = cat_layer_norm_packed(packed, mean, rstd, w, b, dtype=x.dtype)
    held = unpack_ref(*packed)
    want = (held - mean.double().cpu()[:, None]) * rstd.double().cpu()[:, None] * wd + bd
    assert_close(again, want, half_step(x.dtype) * want.abs() + U32 * (8 * (held.abs() + m.abs()[:, None]) * r[:, None] * wd.abs() + 4 * want.abs() + 4), "again")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_layer_norm_without_parameters(dtype):
    x = _rows(33, 515, dtype, 9)
    want, _, r = norm_ref(x.double().cpu(), torch.ones(515).double(), torch.zeros(515).double(), 1e-5)
    assert_close(cat_layer_norm(x), want, _norm_bound(x.double().cpu(), want, torch.ones(515), r, x.dtype), "y")


def test_layer_norm_of_rows_far_from_zero():
    """The variance comes from centred entries: a mean of a thousand deviations leaves them."""
    g = torch.Generator().manual_seed(0)
    x = (1000.0 + torch.randn(9, 1000, generator=g)).cuda()
    want, _, r = norm_ref(x.double().cpu(), torch.ones(1000).double(), torch.zeros(1000).double(), 1e-5)
    assert_close(cat_layer_norm(x), want, _norm_bound(x.double().cpu(), want, torch.ones(1000), r, x.dtype), "y")


def test_a_bad_row_is_its_own_affair():
    for D in (64, 515, 4100, 9000):
        x = _rows(9, D, "f32", D)
        clean = cat_layer_norm(x)
        x[3, D // 2] = float("nan")
        x[5, 0] = float("inf")
        y = cat_layer_norm(x)
        assert bool(torch.isnan(y[3]).all()) and bool(torch.isnan(y[5]).all())
        keep = [0, 1, 2, 4, 6, 7, 8]
        assert torch.equal(y[keep], clean[keep])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", LENGTHS)
@pytest.mark.parametrize("N,held,added", [(1, False, False), (67, False, True), (67, True, True), (1500, True, False)])
def test_layer_norm_backward(N, D, dtype, held, added):
    if N * D > 3_100_000:
        N = 150
    x, dy = _rows(N, D, dtype, D), _rows(N, D, dtype, D + 1)
    add = _rows(N, D, dtype, D + 2) if added else None
    w, b = _params(D, D)
    _, mean, rstd, packed = cat_layer_norm(x, w, b, eps=1e-3, pack=True)
    kw = dict(packed=packed) if held else dict(x=x)
    dx, dw, db = cat_layer_norm_backward(dy, mean, rstd, w, residual_grad=add, **kw)
    d, wd = dy.double().cpu(), w.double().cpu()
    m, r = mean.double().cpu(), rstd.double().cpu()
    rows = unpack_ref(*packed) if held else x.double().cpu()
    xh = (rows - m[:, None]) * r[:, None]
    want, want_w, want_b = norm_backward_ref(d, xh, r, wd)
    # xhat is off by a few roundings of (|x| + |mean|) rstd; the sums by their chains
    xh_err = 4 * U32 * (rows.abs() + m.abs()[:, None]) * r[:, None]
    g = (d * wd).abs()
    c = _chain(D)
    s1, s2 = g.mean(1, keepdim=True), (g * xh.abs()).mean(1, keepdim=True)
    s2_err = U32 * c * s2 + (g * xh_err).mean(1, keepdim=True)
    err = r[:, None] * (U32 * (8 * g + (c + 8) * s1 + 8 * xh.abs() * s2) + xh.abs() * s2_err + xh_err * (s2 + s2_err))
    if added:
        want = want + add.double().cpu()
        err = err + U32 * (want.abs() + add.double().cpu().abs())
    assert_close(dx, want, half_step(dx.dtype) * want.abs() + err, "dx")
    assert_close(dw, want_w, U32 * (N + 8) * (d * xh).abs().sum(0) + (d.abs() * xh_err).sum(0) + 1e-30, "dw")
    assert_close(db, want_b, U32 * (N + 8) * d.abs().sum(0), "db")
    again = cat_layer_norm_backward(dy, mean, rstd, w, residual_grad=add, **kw)
    assert all(torch.equal(p, q) for p, q in zip((dx, dw, db), again)), "the same bits on every run"
    alone, none_w, none_b = cat_layer_norm_backward(dy, mean, rstd, w, residual_grad=add, want_params=False, **kw)
    assert torch.equal(alone, dx) and none_w is None and none_b is None


def test_layer_norm_backward_against_differences():
    """Central differences of the definition in 64 bits: off by h^2 times third derivatives of a few units."""
    x, dy = _rows(3, 40, "f32", 1), _rows(3, 40, "f32", 2)
    w, b = _params(40, 3)
    _, mean, rstd = cat_layer_norm(x, w, b, want_stats=True)
    dx, dw, db = (t.double().cpu() for t in cat_layer_norm_backward(dy, mean, rstd, w, x=x))
    xd, wd, bd, d = (t.double().cpu() for t in (x, w, b, dy))
    h = 1e-4

    def slope(t, i):
        v = t.view(-1)[i].item()
        f = []
        for s in (h, -h):
            t.view(-1)[i] = v + s
            f.append(float((d * norm_ref(xd, wd, bd, 1e-5)[0]).sum()))
        t.view(-1)[i] = v
        return (f[0] - f[1]) / (2 * h)

    for got, t in ((dx, xd), (dw, wd), (db, bd)):
        want = torch.tensor([slope(t, i) for i in range(t.numel())], dtype=torch.float64).view(got.shape)
        assert_close(got, want, 1e-5 * (1.0 + want.abs().max()), "difference quotient")


def test_no_rows():
    for dtype in TYPES.values():
        x = torch.empty(0, 40, dtype=dtype, device="cuda")
        w, b = _params(40, 0)
        y, mean, rstd, packed = cat_layer_norm(x, w, b, pack=True)
        assert y.shape == (0, 40) and mean.shape == (0,) and packed[1].shape == (0, 1)
        assert cat_unpack8(*cat_pack8(x), dtype=dtype).shape == (0, 40)
        dx, dw, db = cat_layer_norm_backward(x, mean, rstd, w, packed=packed)
        assert dx.shape == (0, 40) and not dw.any() and not db.any()
        assert cat_activation_backward(x, packed, "gelu").shape == (0, 40)
