"""The product with bias, activation and residual, and its gradients, against their definitions in 64 bits."""
import pytest
import torch

from paper_2509_26277_amd import (binding, cat_layer_norm, cat_layer_norm_backward, cat_linear, cat_linear_backward_input,
                                  cat_linear_backward_weight, cat_pack8, cat_unpack8)

from block_util import ACT_ERR, ACTS, SLOPE, TYPES, U32, act_ref, assert_close, half_step, unpack_ref

pytestmark = pytest.mark.gpu

# (M, N, K): single rows and few rows, tiles with ragged ends in every direction, lengths that are no whole 16-byte groups,
# shares of k, one entry; the last two fill the large tiles (bfloat16)
SHAPES = [(1, 1, 1), (1, 16, 8), (1, 1000, 2048), (3, 17, 33), (16, 100, 512), (17, 130, 300), (33, 64, 136), (64, 257, 1030),
          (65, 128, 64), (66, 1, 7), (100, 129, 100), (128, 128, 128), (129, 257, 136), (300, 513, 1030), (200, 300, 4096),
          (777, 24, 63), (1025, 640, 72), (3600, 3590, 72), (3584, 3840, 200)]


def _matrix(M, N, dtype, seed, scale=1.0):
    """A matrix whose memory is followed by NaN: nothing behind its last row may count."""
    g = torch.Generator().manual_seed(seed)
    buf = torch.full((M + 3, N), float("nan"), dtype=TYPES[dtype])
    buf[:M] = (torch.randn(M, N, generator=g) * scale).to(TYPES[dtype])
    return buf.cuda()[:M]


def _vector(N, seed):
    return 0.3 * torch.randn(N, generator=torch.Generator().manual_seed(seed)).cuda()


def _d(t):  # (double on the GPU: the references are products too)
    return t.double()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_forward(M, N, K, dtype):
    act = ACTS[(M + N + K) % len(ACTS)]
    x, w, b, res = _matrix(M, K, dtype, 1), _matrix(N, K, dtype, 2, K ** -0.5), _vector(N, 3), _matrix(M, N, dtype, 4)
    z = _d(x) @ _d(w).t() + _d(b)
    size = _d(x).abs() @ _d(w).t().abs() + _d(b).abs()
    z_err = U32 * (K + 8) * size
    u = act_ref(z, act)[0]
    err = SLOPE * z_err + ACT_ERR * (1.0 + z.abs())
    y, packed = cat_linear(x, w, b, act=act, residual=res, pack=True)
    want = u + _d(res)
    assert_close(y, want, (half_step(x.dtype) * want.abs() + err + U32 * want.abs()).cpu(), "y")
    # the checkpoint: half a step of 1 / 127 of the group's largest magnitude, on top of the product's error
    G = -(-N // 128)
    pad = torch.nn.functional.pad(z.abs(), (0, G * 128 - N)).view(M, G, 128)
    top = pad.amax(2)
    perr = torch.nn.functional.pad(z_err, (0, G * 128 - N)).view(M, G, 128).amax(2)
    assert_close(packed[1], top / 127, ((perr + 4 * U32 * top) / 127).cpu(), "scales")
    step = (top / 127).repeat_interleave(128, 1)[:, :N]
    held = unpack_ref(*packed)
    assert_close(held, z, (0.5 * step + 2 * z_err + 2 * perr.repeat_interleave(128, 1)[:, :N] + 256 * U32 * step).cpu(), "checkpoint")
    # without the checkpoint: the same bits; without anything: the product alone
    assert torch.equal(cat_linear(x, w, b, act=act, residual=res), y)
    z = _d(x) @ _d(w).t()
    assert_close(cat_linear(x, w), z, (half_step(x.dtype) * z.abs() + z_err).cpu(), "product")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [2, 150])
def test_every_activation(M, act, dtype):
    x, w, b = _matrix(M, 40, dtype, 1, 3.0), _matrix(70, 40, dtype, 2), _vector(70, 3)
    z = _d(x) @ _d(w).t() + _d(b)
    err = SLOPE * U32 * 48 * (_d(x).abs() @ _d(w).t().abs() + _d(b).abs()) + ACT_ERR * (1.0 + z.abs())
    want = act_ref(z, act)[0]
    assert_close(cat_linear(x, w, b, act=act), want, (half_step(x.dtype) * want.abs() + err).cpu(), act)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_gradients(M, N, K, dtype):
    act = ACTS[(M + N + K) % len(ACTS)]
    dy, w, z = _matrix(M, N, dtype, 5), _matrix(N, K, dtype, 6, N ** -0.5), _matrix(M, K, dtype, 7, 2.0)
    packed = cat_pack8(z)
    held = unpack_ref(*packed).cuda()
    u, du = act_ref(held, act)
    size = _d(dy).abs() @ _d(w).abs()
    want = (_d(dy) @ _d(w)) * du
    err = U32 * (N + 8) * size * SLOPE + ACT_ERR * (1.0 + held.abs()) * size
    dx = cat_linear_backward_input(dy, w, act=act, packed=packed)
    assert_close(dx, want, (half_step(dy.dtype) * want.abs() + err).cpu(), "dx")
    plain = _d(dy) @ _d(w)
    assert_close(cat_linear_backward_input(dy, w), plain, (half_step(dy.dtype) * plain.abs() + U32 * (N + 8) * size).cpu(), "dx, no activation")
    # the weight's gradient, from the checkpoint (bfloat16: u rounded for the matrix cores) and from rows
    dw, db = cat_linear_backward_weight(dy, packed=packed, act=act)
    want = _d(dy).t() @ u
    size = _d(dy).abs().t() @ u.abs()
    u_err = half_step(dy.dtype) * size + _d(dy).abs().t() @ (ACT_ERR * (1.0 + held.abs()))
    assert_close(dw, want, (half_step(dy.dtype) * want.abs() + U32 * (M + 8) * size + u_err).cpu() + 1e-30, "dw")
    assert_close(db, _d(dy).sum(0), (U32 * (M + 8) * _d(dy).abs().sum(0)).cpu(), "db")
    dw, none = cat_linear_backward_weight(dy, x=z, want_bias=False)
    want, size = _d(dy).t() @ _d(z), _d(dy).abs().t() @ _d(z).abs()
    assert none is None
    assert_close(dw, want, (half_step(dy.dtype) * want.abs() + U32 * (M + 8) * size).cpu(), "dw of rows")
    assert torch.equal(cat_linear_backward_weight(dy, x=z)[0], dw), "the same bits on every run"


def test_gradients_against_differences():
    """Central differences of act(x w^T + b) in 64 bits, for x, w and b; z is held exactly (integers up to 127)."""
    g = torch.Generator().manual_seed(0)
    z0 = torch.randint(-3, 4, (5, 24), generator=g).double()
    z0[:, 0] = 127.0
    dy, w = torch.randn(5, 9, generator=g).double(), torch.randn(9, 24, generator=g).double()
    dy, w = dy.float().double(), w.float().double()
    packed = cat_pack8(z0.float().cuda())
    assert torch.equal(unpack_ref(*packed), z0)
    h = 1e-5
    for act in ("gelu", "gelu_tanh", "silu"):
        def f(z, wv):
            return float((dy * (act_ref(z, act)[0] @ wv.t())).sum())

        dx = cat_linear_backward_input(dy.float().cuda(), w.float().cuda(), act=act, packed=packed).double().cpu()
        dw, db = (t.double().cpu() for t in cat_linear_backward_weight(dy.float().cuda(), packed=packed, act=act))
        for got, t, other in ((dx, z0, False), (dw, w, True)):
            want = torch.empty_like(t)
            for i in range(t.numel()):
                s = t.clone()
                s.view(-1)[i] += h
                hi = f(z0, s) if other else f(s, w)
                s.view(-1)[i] -= 2 * h
                lo = f(z0, s) if other else f(s, w)
                want.view(-1)[i] = (hi - lo) / (2 * h)
            assert_close(got, want, 1e-5 * (1.0 + want.abs().max()), act)
        assert_close(db, dy.sum(0), 1e-5, "db")


@pytest.mark.parametrize("M", [5, 200])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_and_infinity_go_where_the_formula_takes_them(M, dtype):
    x, w = _matrix(M, 200, dtype, 1), _matrix(150, 200, dtype, 2)
    clean = cat_linear(x, w, act="gelu")
    x[3, 100], w[140, 0] = float("nan"), float("inf")
    y = cat_linear(x, w, act="gelu")
    bad = torch.zeros(M, 150, dtype=torch.bool, device="cuda")
    bad[3] = bad[:, 140] = True
    assert torch.equal(y[~bad], clean[~bad])
    assert not bool(torch.isfinite(y[3]).any()) and bool(torch.isnan(y[3]).all())
    col = y[:, 140].float()
    rising = _d(x)[:, 0] > 0
    rising[3] = False
    assert bool((col[rising] == float("inf")).all())


def test_no_rows():
    for dtype in TYPES.values():
        x, w = torch.empty(0, 33, dtype=dtype, device="cuda"), torch.ones(7, 33, dtype=dtype, device="cuda")
        y, packed = cat_linear(x, w, pack=True)
        assert y.shape == (0, 7) and packed[0].shape == (0, 7)
        assert cat_linear_backward_input(y, w).shape == (0, 33)
        dw, db = cat_linear_backward_weight(y, x=x)
        assert dw.shape == (7, 33) and not dw.any() and not db.any()


def _block_step(x, dy, p, out):
    """Forward and backward through a block (norm, product, activation, product, residual), checkpoints in 8 bits."""
    h, mean, rstd, x8 = cat_layer_norm(x, p["g"], p["b"], pack=True)
    u, z8 = cat_linear(h, p["w1"], p["b1"], act="gelu", pack=True)
    y = cat_linear(u, p["w2"], p["b2"], residual=x)
    dw2, db2 = cat_linear_backward_weight(dy, packed=z8, act="gelu")
    dz = cat_linear_backward_input(dy, p["w2"], act="gelu", packed=z8)
    dw1, db1 = cat_linear_backward_weight(dz, x=h)
    dh = cat_linear_backward_input(dz, p["w1"])
    dx, dg, db = cat_layer_norm_backward(dh, mean, rstd, p["g"], packed=x8, residual_grad=dy)
    got = [y, dx, dw1, db1, dw2, db2, dg, db]
    if out is None:
        return got
    for o, v in zip(out, got):
        o.copy_(v)


def test_block_step_on_a_stream_and_in_a_graph():
    """On a stream of its own, and captured: every replay, on new inputs, gives the eager calls' bits."""
    M, D, F = 300, 96, 384
    x, dy = _matrix(M, D, "bf16", 1), _matrix(M, D, "bf16", 2, 0.1)
    p = dict(g=1.0 + _vector(D, 3), b=_vector(D, 4), w1=_matrix(F, D, "bf16", 5, 0.1), b1=_vector(F, 6), w2=_matrix(D, F, "bf16", 7, 0.1), b2=_vector(D, 8))
    eager = _block_step(x, dy, p, None)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        other = _block_step(x, dy, p, None)
    s.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, other))
    out = [torch.empty_like(t) for t in eager]
    with torch.cuda.stream(s):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=s):
            _block_step(x, dy, p, out)
    torch.cuda.synchronize()
    for k in range(4):
        x.copy_(_matrix(M, D, "bf16", 20 + k))
        want = _block_step(x, dy, p, None)
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(want, out)), f"replay {k}"


def test_a_workspace_of_the_stated_size_is_enough_and_stays_in_its_bounds():
    """The stated size for each call, with guard bytes behind it."""
    lib = binding.load_library()
    for dtype, dt in (("f32", 0), ("bf16", 1)):
        for M, N, K in [(1, 64, 2048), (300, 65, 1030), (150, 130, 4096)]:
            x, w, dy = _matrix(M, K, dtype, 1), _matrix(N, K, dtype, 2), _matrix(M, N, dtype, 3)
            packed = cat_pack8(x)
            for size, call in ((lib.cat_linear_workspace_bytes(M, N, K, dt), lambda ws: cat_linear(x, w, pack=True, workspace=ws)[0]),
                               (lib.cat_linear_backward_workspace_bytes(M, N, K, dt), lambda ws: cat_linear_backward_input(dy, w, workspace=ws)),
                               (lib.cat_linear_backward_workspace_bytes(M, N, K, dt),
                                lambda ws: cat_linear_backward_weight(dy, packed=packed, workspace=ws)[0])):
                buf = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
                call(buf[:size])
                assert bool((buf[size:] == 0xA5).all())


def test_checkpoint_of_a_product_decodes_in_either_type():
    x, w = _matrix(70, 64, "bf16", 1), _matrix(200, 64, "bf16", 2)
    _, packed = cat_linear(x, w, pack=True)
    assert torch.equal(cat_unpack8(*packed, dtype=torch.bfloat16), cat_unpack8(*packed).bfloat16())
