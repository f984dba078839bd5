"""Layer norm where a workgroup goes through several rows: the row requested ahead, the ragged last round and the sums over a
workgroup's rows, for every kernel that a row length takes.  Definitions in 64 bits, on the GPU."""
import pytest
import torch

from paper_2509_26277_amd import cat_layer_norm, cat_layer_norm_backward, cat_layer_norm_packed, cat_pack8, cat_unpack8

from block_util import TYPES, U32, half_step

pytestmark = pytest.mark.gpu

# One length for each of the kernels (threads a row x 16-byte groups a thread).  A workgroup holds 256 / threads rows, one at
# least, and there are 1024 of them forward, 512 backward: two and a half rounds forward, five or more backward.
LENGTHS = {"bf16": [(62, 8), (120, 16), (251, 32), (512, 64), (1000, 64), (2047, 64), (4001, 256), (8190, 256)],
           "f32": [(31, 8), (60, 16), (127, 32), (256, 64), (511, 64), (1001, 64), (2040, 64), (4001, 256), (8190, 256)]}
CASES = [(t, D, (1024 * 256 // threads) * 5 // 2 + 3) for t in LENGTHS for D, threads in LENGTHS[t]]
CHAIN = 64  # additions one after the other in a row's sum: 32 entries of a thread and the steps across threads


def _close(got, want, bound, what):
    assert got.shape == want.shape, what
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist())


def _rows(N, D, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(N, D, generator=g, device="cuda")
    return (x + 0.5 * torch.randn(D, generator=g, device="cuda")).to(TYPES[dtype])


def _params(D, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return 1.0 + 0.3 * torch.randn(D, generator=g, device="cuda"), 0.2 * torch.randn(D, generator=g, device="cuda")


@pytest.mark.parametrize("dtype,D,N", CASES)
def test_forward_and_again_from_the_checkpoint(dtype, D, N):
    x = _rows(N, D, dtype, D)
    w, b = _params(D, D + 1)
    y, mean, rstd, packed = cat_layer_norm(x, w, b, eps=1e-3, pack=True)
    xd, wd, bd = x.double(), w.double(), b.double()
    m = xd.mean(1)
    c = xd - m[:, None]
    r = 1.0 / torch.sqrt((c * c).mean(1) + 1e-3)
    size = xd.abs().mean(1)
    _close(mean, m, U32 * CHAIN * size, "mean")
    _close(rstd, r, U32 * r * (CHAIN + 4 * CHAIN * size * r), "rstd")
    want = c * r[:, None] * wd + bd
    err = U32 * (2 * (size[:, None] * CHAIN + xd.abs()) * r[:, None] * wd.abs() + CHAIN * want.abs() + 4)
    _close(y, want, half_step(x.dtype) * want.abs() + err, "y")
    assert torch.equal(y, cat_layer_norm(x, w, b, eps=1e-3))
    alone = cat_pack8(x)
    assert torch.equal(packed[0], alone[0]) and torch.equal(packed[1], alone[1])
    held = cat_unpack8(*packed).double()
    again = cat_layer_norm_packed(packed, mean, rstd, w, b, dtype=x.dtype)
    md, rd = mean.double()[:, None], rstd.double()[:, None]
    want = (held - md) * rd * wd + bd
    _close(again, want, half_step(x.dtype) * want.abs() + U32 * (8 * (held.abs() + md.abs()) * rd * wd.abs() + 4 * want.abs() + 4), "again")


@pytest.mark.parametrize("held", [False, True])
@pytest.mark.parametrize("dtype,D,N", CASES)
def test_backward(dtype, D, N, held):
    x, dy, add = _rows(N, D, dtype, D), _rows(N, D, dtype, D + 1), _rows(N, D, dtype, D + 2) if held else None
    w, b = _params(D, D + 3)
    _, mean, rstd, packed = cat_layer_norm(x, w, b, eps=1e-3, pack=True)
    kw = dict(packed=packed) if held else dict(x=x)
    dx, dw, db = cat_layer_norm_backward(dy, mean, rstd, w, residual_grad=add, **kw)
    d, wd, m, r = dy.double(), w.double(), mean.double()[:, None], rstd.double()[:, None]
    rows = cat_unpack8(*packed).double() if held else x.double()
    xh = (rows - m) * r
    xh_err = 4 * U32 * (rows.abs() + m.abs()) * r  # (a few roundings of its terms)
    g = d * wd
    s1, s2 = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    a1, a2 = g.abs().mean(1, keepdim=True), (g * xh).abs().mean(1, keepdim=True)
    a2_err = U32 * CHAIN * a2 + (g.abs() * xh_err).mean(1, keepdim=True)
    want = r * (g - s1 - xh * s2)
    err = r * (U32 * (8 * g.abs() + (CHAIN + 8) * a1 + 8 * xh.abs() * a2) + xh.abs() * a2_err + xh_err * (a2 + a2_err))
    if held:
        want = want + add.double()
        err = err + U32 * (want.abs() + add.double().abs())
    _close(dx, want, half_step(dx.dtype) * want.abs() + err, "dx")
    # A column's sum: up to 21 rounds in a register (where a row has a workgroup; 6 and 32 rows' slots in LDS where it has 8 lanes),
    # 512 parts as 16 and five halvings, each term's own rounding: no more than 64 additions one after the other.  A row left out,
    # or taken twice, is one term of N, more than the bound in most columns.
    _close(dw, (d * xh).sum(0), U32 * 64 * (d * xh).abs().sum(0) + (d.abs() * xh_err).sum(0), "dweight")
    _close(db, d.sum(0), U32 * 64 * d.abs().sum(0), "dbias")
    alone = cat_layer_norm_backward(dy, mean, rstd, w, residual_grad=add, want_params=False, **kw)[0]
    assert torch.equal(alone, dx)
