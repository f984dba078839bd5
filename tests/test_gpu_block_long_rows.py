"""The norm's backward pass of rows beyond 8192 entries: few rows, more columns than a launch has threads for, no parameters."""
import pytest
import torch

from paper_2509_26277_amd import cat_layer_norm, cat_layer_norm_backward

from block_util import TYPES, U32, half_step

pytestmark = pytest.mark.gpu


def _close(got, want, bound, what):
    off = (got.double() - want).abs()
    assert bool((off <= bound).all()), (what, float((off - bound).max()))


def _case(N, D, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x, dy = ((torch.randn(N, D, generator=g, device="cuda") + 0.3).to(TYPES[dtype]) for _ in range(2))
    w = 1.0 + 0.2 * torch.randn(D, generator=g, device="cuda")
    return x, dy, w


# (2, 2^26 + 4): two sums for every column are more than 2^27, 32 of them a workgroup of 1024 threads
@pytest.mark.parametrize("dtype,N,D", [("f32", 2, (1 << 26) + 4), ("f32", 1, 9001), ("bf16", 3, 20002), ("bf16", 130, 8200), ("f32", 64, 8196)])
def test_sums_over_rows(dtype, N, D):
    """dweight and dbias: a column's N terms, each off by three roundings of xhat and one of its own, in a chain of N at most."""
    x, dy, w = _case(N, D, dtype, D)
    _, mean, rstd = cat_layer_norm(x, w, want_stats=True)
    dx, dw, db = cat_layer_norm_backward(dy, mean, rstd, w, x=x)
    want_w, want_b = torch.zeros(D, dtype=torch.float64, device="cuda"), torch.zeros(D, dtype=torch.float64, device="cuda")
    size_w, size_b = torch.zeros_like(want_w), torch.zeros_like(want_b)
    for r in range(N):
        m, s, d = mean[r].double(), rstd[r].double(), dy[r].double()
        xh = (x[r].double() - m) * s
        want_w += d * xh
        want_b += d
        size_w += d.abs() * (x[r].double().abs() + m.abs()) * s
        size_b += d.abs()
    _close(dw, want_w, U32 * (N + 6) * size_w, "dweight")
    _close(db, want_b, U32 * (N + 6) * size_b, "dbias")
    del want_w, want_b, size_w, size_b
    # dx, a row at a time; its two means are chains of D / 256 additions a thread
    chain = 64 + D // 256
    for r in range(0, N, max(1, N // 3)):
        m, s, d = mean[r].double(), rstd[r].double(), dy[r].double() * w.double()
        xh = (x[r].double() - m) * s
        want = s * (d - d.mean() - xh * (d * xh).mean())
        err = U32 * s * (8 * d.abs() + (chain + 8) * (d.abs().mean() + xh.abs() * (d * xh).abs().mean()) + 8 * (x[r].double().abs() + m.abs()) * s)
        _close(dx[r], want, half_step(dx.dtype) * want.abs() + err, "dx")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", [40, 1001, 5000, 9001])
def test_without_parameters_a_small_workspace_is_enough_and_stays_in_its_bounds(D, dtype):
    x, dy, w = _case(70, D, dtype, D)
    _, mean, rstd = cat_layer_norm(x, w, want_stats=True)
    want = cat_layer_norm_backward(dy, mean, rstd, w, x=x)[0]
    buf = torch.full((4096,), 0xA5, dtype=torch.uint8, device="cuda")
    dx, dw, db = cat_layer_norm_backward(dy, mean, rstd, w, x=x, want_params=False, workspace=buf[:256])
    assert dw is None and db is None and torch.equal(dx, want)
    assert bool((buf == 0xA5).all())
