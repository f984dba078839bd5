"""Products of 8-bit integers whose bfloat16 results have the longest rows that the calls take."""
import pytest
import torch

from paper_2509_26277_amd import cat_gated_linear8, cat_linear8

from block_util import U32, half_step
from test_gpu_linear8 import _close, _operands, _product

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,N,K", [(1, (1 << 21) + 16, 24), (40, (1 << 21) + 16, 33), (100, (1 << 21) + 16, 24), (100, (1 << 21) + 1, 33), (150, 1 << 22, 16)])
def test_rows_of_more_than_two_to_the_21_columns(M, N, K):
    x, xs, w, ws = _operands(M, 2 * N, K)
    res = torch.ones(M, N, dtype=torch.bfloat16, device="cuda")
    y, h = cat_linear8(x, xs, w[:N], ws[:N], act="relu", residual=res), cat_gated_linear8(x, xs, w, ws, act="relu")
    assert y.shape == h.shape == (M, N)
    half = half_step(y.dtype)
    for at in (0, N // 2, N - 3000):
        c, v = slice(at, at + 3000), slice(N + at, N + at + 3000)
        (g, ge), (u, ue) = _product(x, xs, w[c].contiguous(), ws[c], None), _product(x, xs, w[v].contiguous(), ws[v], None)
        g, want = g.clamp(min=0), g.clamp(min=0) + 1
        _close(y[:, c], want, half * want + (ge + 2 * U32 * want) * (1 + half), "y")
        want = g * u
        _close(h[:, c], want, half * want.abs() + (U32 * want.abs() + ge * (u.abs() + ue) + g * ue) * (1 + half), "gated")
