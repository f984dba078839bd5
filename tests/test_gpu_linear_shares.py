"""Shares of a weight's gradient: by rows in a workspace of the stated size, by tiles where the caller gives room for them; the same bits."""
import pytest
import torch

from paper_2509_26277_amd import binding, cat_linear_backward_weight, cat_pack8, cat_unpack8

from block_util import TYPES, U32, half_step

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(4096, 129, 129), (8192, 256, 1000), (16384, 257, 257), (300, 7, 9), (5000, 2000, 3000), (20000, 40, 33), (16384, 1024, 512)])
def test_either_layout_gives_the_same_bits(M, N, K, dtype):
    g = torch.Generator(device="cuda").manual_seed(M + N + K)
    dy, x = (torch.randn(M, D, generator=g, device="cuda").to(TYPES[dtype]) for D in (N, K))
    packed = cat_pack8(x)
    n = binding.load_library().cat_linear_backward_workspace_bytes(M, N, K, binding.CAT_F32 if dtype == "f32" else binding.CAT_BF16)
    for kw, u in ((dict(x=x), x.double()), (dict(packed=packed), cat_unpack8(*packed, dtype=torch.float32).to(x.dtype).double())):
        want, size = dy.double().t() @ u, dy.double().abs().t() @ u.abs()
        bound = half_step(x.dtype) * want.abs() + (1 + half_step(x.dtype)) * U32 * (M + 40) * size
        got = []
        for room in (n, n, 6 * n):
            buf = torch.full((room + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
            dw, db = cat_linear_backward_weight(dy, workspace=buf[:room], **kw)
            assert bool((buf[room:] == 0xA5).all())
            got.append(dw)
        assert bool(((got[0].double() - want).abs() <= bound).all())
        assert torch.equal(got[0], got[1]) and torch.equal(got[0], got[2])
        assert torch.equal(cat_linear_backward_weight(dy, **kw)[0], got[0])
