"""GELU of bfloat16 results far below zero: right to a step of its own value, not only of its argument."""
import math

import pytest
import torch

from paper_2509_26277_amd import cat_gated_linear, cat_gated_linear8, cat_linear8

from block_util import U32, half_step

pytestmark = pytest.mark.gpu
N = 8192


@pytest.mark.parametrize("M", [1, 40, 300, 2304])
def test_every_value_of_the_range(M):
    """Arguments by the bias alone, in every kernel.  The tail's fit is off by 3.8e-5 of its value and its evaluation in fp32 by 5.2e-5 (sums of
    9 roundings of numbers of up to 500, as an exponent), the exponential and the last three operations by 2 half steps of fp32 each."""
    z = torch.linspace(-13.2, 20.0, N, device="cuda")
    d = z.double()
    want = d * torch.special.erfc(-d / math.sqrt(2.0)) / 2
    held = want.abs() >= 2.0 ** -126  # the smallest normal number
    bound = want.abs() * (half_step(torch.bfloat16) * (1 + 1e-4) + 3.8e-5 + 5.2e-5 + 8 * U32)
    x8, w8, one = torch.zeros(M, 16, dtype=torch.int8, device="cuda"), torch.zeros(2 * N, 16, dtype=torch.int8, device="cuda"), torch.ones(2 * N, device="cuda")
    gate = torch.cat((z, one[:N]))
    got = [cat_linear8(x8, one[:M], w8[:N], one[:N], z, act="gelu"), cat_gated_linear8(x8, one[:M], w8, one, gate, act="gelu"),
           cat_gated_linear(x8.bfloat16(), w8.bfloat16(), gate, act="gelu"), cat_gated_linear(x8.bfloat16(), w8.bfloat16(), gate, act="gelu", pack=True)[0]]
    for i, y in enumerate(got):
        off = (y.double() - want).abs()
        bad = (off > bound) & held
        assert not bool(bad.any()), (i, int(bad.sum()), z[bad.any(0)].min().item(), z[bad.any(0)].max().item())
        assert bool((off[:, ~held] <= 2.0 ** -126).all())
