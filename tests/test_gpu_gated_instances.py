"""Every kernel of the gate's gradients: one is compiled for each activation, alignment of rows and tile size, and the shape picks it."""
import pytest
import torch

from paper_2509_26277_amd import binding

import test_gpu_gated
import test_gpu_linear8
from block_util import ACTS, TYPES, act_ref
from test_gated_host import A, B, C, D, E, FAKE

# what the shape is meant to pick: type, edge of a tile (None: shares of k, joined) and whether rows are whole groups of eight columns
CLASSES = {(4864, 2048, 64): ("bf16", 256, True), (6001, 2503, 130): ("bf16", 256, False), (300, 512, 136): ("bf16", 128, True), (300, 513, 136): ("bf16", 128, False),
           (4097, 1000, 256): ("f32", 128, True), (513, 1003, 130): ("f32", 128, False), (200, 96, 4096): ("bf16", None, True), (200, 97, 4096): ("f32", None, False)}


@pytest.mark.parametrize("M,F,N", list(CLASSES))
def test_the_shape_picks_its_kernel(M, F, N):
    """By the workspace that the call says it needs: sums over rows, four to a tile, and operands laid out in whole lines of 128 bytes."""
    dtype, edge, aligned = CLASSES[M, F, N]
    assert aligned == (F % 8 == 0)
    lib, dt, e = binding.load_library(), (0 if dtype == "f32" else 1), 4 if dtype == "f32" else 2
    assert lib.cat_gated_backward_input(A, B, C, D, M, N, F, dt, 0, E, None, FAKE, 16, None) == 3
    need = int(lib.cat_last_error().decode().split("need ")[1].split()[0])

    def up(n, to):
        return -(-n // to) * to

    laid = sum(up(rows * up(cols * e, 128), 256) for rows, cols in ((M, N), (N, F)) if cols * e % 16)
    sums = {tile: up(-(-M // tile) * 4 * 2 * F * 4, 256) for tile in (128, 256)}
    assert sums[128] != sums[256]
    if edge is None:
        assert need - laid not in sums.values() and need - laid >= 2 * M * F * 4  # two shares of dh at least
    else:
        assert need - laid == sums[edge]


@pytest.mark.gpu
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M,F,N", list(CLASSES))
def test_gradients_of_every_kernel(M, F, N, act):
    test_gpu_gated.test_gradients(M, F, N, CLASSES[M, F, N][0], act)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,M,F,K", [(d, M, F, K) for M in (17, 33, 64) for d, F, K in (("bf16", 8200, 2056), ("bf16", 8191, 2056), ("f32", 4100, 2052), ("f32", 4099, 2049))])
def test_few_rows_by_a_long_weight(dtype, M, F, K):
    """From 64 MB of weight on the tiles take 17 to 64 rows, too, without a checkpoint and with one."""
    assert 2 * F * K * (4 if dtype == "f32" else 2) >= 1 << 26
    test_gpu_gated.test_forward(M, F, K, dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("M", [2, 40, 300, 2304])
def test_every_row_has_the_same_values(M):
    """Rows that are alike, by a product of 8-bit integers over the activations' whole range: all M of them, NaN and values apart."""
    N = 4096
    x, xs = torch.ones(M, 1, dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda")
    w = torch.zeros(2 * N, 1, dtype=torch.int8, device="cuda")
    z = (torch.arange(N, device="cuda") - N // 2).float() / 64
    ends = [3e38, -3e38, 1e20, -1e20, 200.0, -200.0, float("inf"), float("-inf"), float("nan")]
    z[:len(ends)] = torch.tensor(ends, device="cuda")
    both = torch.cat((z, torch.ones(N, device="cuda")))
    one = torch.ones(2 * N, device="cuda")
    for act in ACTS:
        for t in TYPES.values():
            plain = test_gpu_linear8.cat_linear8(x, xs, w[:N], one[:N], z, act=act, dtype=t)
            gated = test_gpu_linear8.cat_gated_linear8(x, xs, w, one, both, act=act, dtype=t)
            for y in (plain, gated):
                nan = torch.isnan(y)
                assert torch.equal(nan, nan[:1].expand(M, N)) and torch.equal(torch.nan_to_num(y), torch.nan_to_num(y[:1]).expand(M, N)), act
                assert bool(nan[:, 8].all()) and not bool(nan[:, 9:].any())
            want = act_ref(z[9:].double(), act)[0]
            test_gpu_linear8._close(plain[:, 9:], want.expand(M, N - 9), test_gpu_linear8.half_step(t) * want.abs() + test_gpu_linear8.ACT_ERR * (1.0 + z[9:].double().abs()), act)
