"""The derivative that float gradients behind a gate take, held to its own roundings: dh and the value exact, arguments of whole sixteenths."""
import math

import pytest
import torch

from paper_2509_26277_amd import cat_gated_backward_input, cat_pack8

from block_util import U32

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,F", [(5, 7), (40, 131), (300, 256), (300, 255)])  # joined from shares of rows, tiles of any alignment
def test_tanh_gelu(M, F):
    code = (torch.arange(M * F).view(M, F) * 37 % 255 - 127).float()
    code[:, ::128] = 127.0  # every group's scale is 1 / 16
    z, v = (code / 16).cuda(), torch.full((M, F), 127.0, device="cuda")
    parts = [cat_pack8(t) for t in (z, v)]
    packed = tuple(torch.stack(p) for p in zip(*parts))
    one = torch.ones(M, 1, device="cuda")
    dz, _ = cat_gated_backward_input(one, torch.ones(1, F, device="cuda"), packed, act="gelu_tanh")
    d = z.double()
    a = 2 * math.sqrt(2 / math.pi) * (d + 0.044715 * d ** 3)
    p, q = torch.sigmoid(a), torch.sigmoid(-a)
    slope = 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * d * d)
    want = p + d * p * q * slope
    # e = exp(-a): a rounds three times and its two constants once each, the exponential's argument again: 6 |a| half steps, and its own 2; p = 1 / (1 + e) moves by
    # p q of that, q by as much, p q by |p - q| of it.  p rounds by 3 (the sum, the reciprocal), p q by 5; slope, both products and the sum by 8
    e = 6 * a.abs() + 2
    bound = U32 * (p * q * e * (1 + d.abs() * slope) + 3 * p + (8 + 8) * d.abs() * p * q * slope + 2 * want.abs())
    got = dz[:, :F].double() / 127
    bad = ~((got - want).abs() <= bound + U32 * want.abs())
    assert not bool(bad.any()), (int(bad.sum()), z[bad].min().item(), z[bad].max().item())
    value = dz[:, F:].double()
    assert bool(((value - d * p).abs() <= U32 * (d.abs() * p * (q * e + 4)) + 1e-300).all())
