"""The weight's gradient behind a gate, dw = dy^T (act(g) v): its sums take act(g) v in more than a bfloat16 entry's bits."""
import pytest
import torch

from paper_2509_26277_amd import cat_gated_backward_weight, cat_pack8

from block_util import ACT_ERR, ACTS, U32, half_step
from test_gpu_gated import _close, _held, _matrix, act_ref

pytestmark = pytest.mark.gpu

# (M, F, N): one row, odd lengths, one tile and many, shares of k, large tiles whole and ragged, more tiles than workgroups
SHAPES = [(1, 16, 8), (3, 17, 33), (64, 257, 103), (129, 255, 136), (300, 513, 103), (777, 12, 63), (2000, 1001, 600), (256, 4096, 1024),
          (300, 8200, 2056), (4000, 1024, 512), (16384, 320, 256)]


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,F,N", SHAPES)
def test_bfloat16_gradients_round_once(M, F, N, act):
    """The only rounding to 16 bits is the result's: act(g) v is held to 2^-15 of itself (its upper 16 bits, and the rest rounded)."""
    dy = _matrix(M, N, "bf16", 5)
    packed, (g, v) = _held(M, F, "bf16", 7)
    u = act_ref(g, act)[0]
    h, d = u * v, dy.double()
    # the activation's own error is that of fp32 (GELU's tail: 2.4e-7 at most); the product with v rounds once
    off = 2.0 ** -15 * h.abs() + ACT_ERR * (1.0 + g.abs()) * v.abs() + U32 * h.abs()
    want, size = d.t() @ h, d.abs().t() @ h.abs()
    # two sums of M products, and of their shares
    bound = half_step(dy.dtype) * want.abs() + (1 + half_step(dy.dtype)) * (d.abs().t() @ off + U32 * (2 * M + 40) * size) + 1e-30
    dw, _ = cat_gated_backward_weight(dy, packed, act=act)
    _close(dw, want, bound, "dw")
    if want.numel() > 4096 and M > 16:  # 2^-15 of the terms is a 128th of half a step of 2^-8: beside the rounding's error, hardly anything
        rounded = want.to(dy.dtype).double() - want
        assert (dw.double() - want).norm() <= 1.02 * rounded.norm(), "more than the result's own rounding"
    again, _ = cat_gated_backward_weight(dy, packed, act=act, want_bias=False)
    assert torch.equal(again, dw)


@pytest.mark.parametrize("M", [5, 300])
def test_infinities_and_the_largest_values(M):
    """act(g) v that leaves the floats is an infinity in its row's sums, one below the largest float stays finite."""
    g, v = torch.zeros(M, 256), torch.zeros(M, 256)
    g[2, 0], v[2, 0] = 2.0 ** 70, 2.0 ** 70             # an infinity
    g[3, 128], v[3, 128] = 127 * 2.0 ** 60, 127 * 2.0 ** 53  # 127 * 127 * 2^113 = 2^126.98, upper 16 bits and a rest
    parts = [cat_pack8(t.cuda()) for t in (g, v)]
    packed = tuple(torch.stack(p) for p in zip(*parts))
    dy = torch.zeros(M, 8, dtype=torch.bfloat16, device="cuda")
    dy[2], dy[3] = 1.0, 2.0 ** -20
    dy[2, 1] = -1.0
    dw, _ = cat_gated_backward_weight(dy, packed, act="none")
    got = dw.double().cpu()
    assert got[0, 0] == float("inf") and got[1, 0] == float("-inf")
    want = 127.0 * 127.0 * 2.0 ** 93
    assert bool((got[:, 128] - want).abs().max() <= 2.0 ** -8 * want)
    got[:, 0] = got[:, 128] = 0.0
    assert not bool(got.any())


def test_a_nan_stays_in_the_columns_of_its_group():
    packed, _ = _held(300, 384, "bf16", 7)
    dy = _matrix(300, 40, "bf16", 5)
    clean, _ = cat_gated_backward_weight(dy, packed, act="silu")
    packed[1][0, 17, 1] = float("nan")  # the scale of a row's channels 128 .. 255
    dw, db = cat_gated_backward_weight(dy, packed, act="silu")
    assert bool(torch.isnan(dw[:, 128:256]).all()) and bool(torch.isfinite(db).all())
    assert torch.equal(dw[:, :128], clean[:, :128]) and torch.equal(dw[:, 256:], clean[:, 256:])
