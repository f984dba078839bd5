"""The gated product and the gradients behind the gate, against their definitions in 64 bits."""
import pytest
import torch

from paper_2509_26277_amd import (binding, cat_gated_backward_input, cat_gated_backward_weight, cat_gated_linear, cat_pack8,
                                  cat_unpack8)

from block_util import ACT_ERR, ACTS, SLOPE, TYPES, U32, act_ref, half_step

pytestmark = pytest.mark.gpu

# (M, F, K): single rows and few rows, tiles with ragged ends in every direction, odd lengths (the value's rows, bias and gradients
# then start on any boundary), shares of k, one entry; large tiles (bfloat16) whole and ragged, with shares, and more than workgroups
SHAPES = [(1, 1, 1), (1, 16, 8), (1, 1001, 2048), (3, 17, 33), (16, 100, 512), (17, 65, 300), (33, 64, 136), (64, 257, 1030), (48, 40, 4096),
          (65, 64, 64), (66, 1, 7), (100, 129, 100), (128, 128, 128), (129, 255, 136), (300, 513, 1030), (200, 150, 4096), (777, 12, 63), (300, 9, 40), (2100, 7, 64), (513, 15, 128),
          (1025, 320, 72), (3600, 1795, 72), (3584, 1920, 200), (2000, 1001, 6000), (6144, 2560, 256), (6001, 2503, 130), (4864, 2048, 64)]
# a few rows behind the last whole tile, for which the tiles would need a round of workgroups more
TAILS = [("f32", 923, 2051, 130), ("f32", 4099, 1001, 513), ("bf16", 8200, 1001, 130), ("bf16", 8193, 1000, 128)]


def _matrix(M, N, dtype, seed, scale=1.0):
    """A matrix whose memory is followed by NaN: nothing behind its last row may count."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    buf = torch.full((M + 3, N), float("nan"), dtype=TYPES[dtype], device="cuda")
    buf[:M] = (torch.randn(M, N, generator=g, device="cuda") * scale).to(TYPES[dtype])
    return buf[:M]


def _vector(N, seed, scale=0.3):
    return _matrix(1, N, "f32", seed, scale)[0]


def _close(got, want, bound, what):
    assert got.shape == want.shape, what
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist())


def _groups(t, reduce):
    G = -(-t.shape[1] // 128)
    return reduce(torch.nn.functional.pad(t, (0, G * 128 - t.shape[1])).view(t.shape[0], G, 128))


def _held(M, F, dtype, seed, scale=2.0):
    """The checkpoints of a gate and a value, and what they stand for."""
    parts = [cat_pack8(_matrix(M, F, dtype, seed + i, scale)) for i in range(2)]
    packed = tuple(torch.stack(p) for p in zip(*parts))
    return packed, [cat_unpack8(c, s).double() for c, s in parts]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,F,K", SHAPES)
def test_forward(M, F, K, dtype):
    act = ACTS[(M + F + K) % len(ACTS)]
    x, w, b = _matrix(M, K, dtype, 1), _matrix(2 * F, K, dtype, 2, K ** -0.5), _vector(2 * F, 3)
    z = x.double() @ w.double().t() + b.double()
    z_err = U32 * (K + 8) * (x.double().abs() @ w.double().abs().t() + b.double().abs())
    (g, v), (ge, ve) = z.split(F, 1), z_err.split(F, 1)
    u = act_ref(g, act)[0]
    want, ue = u * v, SLOPE * ge + ACT_ERR * (1.0 + g.abs())
    bound = half_step(x.dtype) * want.abs() * (1 + U32) + U32 * want.abs() + (ue * (v.abs() + ve) + u.abs() * ve) * (1 + half_step(x.dtype))
    y, packed = cat_gated_linear(x, w, b, act=act, pack=True)
    _close(y, want, bound, "y")
    # the checkpoints: half a step of 1 / 127 of the group's largest magnitude, on top of the product's error
    for t, err, codes, scales in ((g, ge, packed[0][0], packed[1][0]), (v, ve, packed[0][1], packed[1][1])):
        top, perr = _groups(t.abs(), lambda a: a.amax(2)), _groups(err, lambda a: a.amax(2))
        _close(scales, top / 127, (perr + 4 * U32 * top) / 127, "scales")
        step, off = ((a.repeat_interleave(128, 1)[:, :F]) for a in (top / 127, perr))
        _close(cat_unpack8(codes, scales), t, 0.5 * step + 2 * err + 2 * off + 256 * U32 * step, "checkpoint")
    # again: the same bits; without the checkpoint (whose rounding of shares of k may be others): the same bounds
    again, packed2 = cat_gated_linear(x, w, b, act=act, pack=True)
    assert torch.equal(again, y) and all(torch.equal(p, q) for p, q in zip(packed, packed2))
    _close(cat_gated_linear(x, w, b, act=act), want, bound, "y without the checkpoint")
    z = x.double() @ w.double().t()
    (g, v), (ge, ve) = z.split(F, 1), z_err.split(F, 1)
    want = g * v
    _close(cat_gated_linear(x, w, act="none"), want,
           half_step(x.dtype) * want.abs() * (1 + U32) + U32 * want.abs() + (ge * (v.abs() + ve) + g.abs() * ve) * (1 + half_step(x.dtype)), "without bias")


@pytest.mark.parametrize("dtype,M,F,K", TAILS)
def test_rows_behind_the_last_tile(dtype, M, F, K):
    x, w, b = _matrix(M, K, dtype, 1), _matrix(2 * F, K, dtype, 2, K ** -0.5), _vector(2 * F, 3)
    z = x.double() @ w.double().t() + b.double()
    z_err = U32 * (K + 8) * (x.double().abs() @ w.double().abs().t() + b.double().abs())
    (g, v), (ge, ve) = z.split(F, 1), z_err.split(F, 1)
    u = act_ref(g, "gelu")[0]
    want, ue = u * v, SLOPE * ge + ACT_ERR * (1.0 + g.abs())
    bound = half_step(x.dtype) * want.abs() * (1 + U32) + U32 * want.abs() + (ue * (v.abs() + ve) + u.abs() * ve) * (1 + half_step(x.dtype))
    out = torch.full((M + 2, F), 7.0, dtype=x.dtype, device="cuda")
    _close(cat_gated_linear(x, w, b, act="gelu", out=out[:M]), want, bound, "y")
    assert bool((out[M:] == 7.0).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [2, 150, 2100])
def test_every_activation(M, act, dtype):
    F, K = (35, 40) if M < 1000 else (1032, 64)
    x, w, b = _matrix(M, K, dtype, 1, 3.0), _matrix(2 * F, K, dtype, 2, K ** -0.5), _vector(2 * F, 3)
    z = x.double() @ w.double().t() + b.double()
    z_err = U32 * (K + 8) * (x.double().abs() @ w.double().abs().t() + b.double().abs())
    (g, v), (ge, ve) = z.split(F, 1), z_err.split(F, 1)
    u = act_ref(g, act)[0]
    want, ue = u * v, SLOPE * ge + ACT_ERR * (1.0 + g.abs())
    _close(cat_gated_linear(x, w, b, act=act), want,
           half_step(x.dtype) * want.abs() * (1 + U32) + U32 * want.abs() + (ue * (v.abs() + ve) + u.abs() * ve) * (1 + half_step(x.dtype)), act)


@pytest.mark.parametrize("dtype,act", [(d, None) for d in TYPES] + [("bf16", "gelu"), ("f32", "silu")])
@pytest.mark.parametrize("M,F,N", SHAPES)
def test_gradients(M, F, N, dtype, act):
    act = act or ACTS[(M + F + N + 2) % len(ACTS)]
    dy, w = _matrix(M, N, dtype, 5), _matrix(N, F, dtype, 6, N ** -0.5)
    packed, (g, v) = _held(M, F, dtype, 7)
    u, du = act_ref(g, act)
    dh, size = dy.double() @ w.double(), dy.double().abs() @ w.double().abs()
    half = half_step(dy.dtype)
    want = torch.cat((dh * v * du, dh * u), 1)
    # dh sums N products; act and its derivative are off by ACT_ERR (1 + |g|), and the products round twice
    e = U32 * (N + 8) * size
    err = torch.cat((v.abs() * (SLOPE * e + ACT_ERR * (1.0 + g.abs()) * size), u.abs() * e + ACT_ERR * (1.0 + g.abs()) * (size + e)), 1) + 3 * U32 * want.abs()
    dz, db = cat_gated_backward_input(dy, w, packed, act=act)
    _close(dz, want, half * want.abs() + err * (1 + half), "dz")
    _close(db, want.sum(0), err.sum(0) + U32 * (M + 8) * want.abs().sum(0), "db")
    again, again_db = cat_gated_backward_input(dy, w, packed, act=act)
    assert torch.equal(again, dz) and torch.equal(again_db, db), "the same bits on every run"
    alone, none = cat_gated_backward_input(dy, w, packed, act=act, want_bias=False)
    assert none is None and torch.equal(alone, dz)
    # the last product's weight (bfloat16: act(g) v rounded for the matrix cores)
    dw, db = cat_gated_backward_weight(dy, packed, act=act)
    h = u * v
    want, size = dy.double().t() @ h, dy.double().abs().t() @ h.abs()
    h_err = dy.double().abs().t() @ (half * h.abs() + (1 + half) * (ACT_ERR * (1.0 + g.abs()) * v.abs() + U32 * h.abs()))
    _close(dw, want, half * want.abs() + U32 * (M + 8) * size + h_err + 1e-30, "dw")
    _close(db, dy.double().sum(0), U32 * (M + 8) * dy.double().abs().sum(0), "dw's bias")
    again, none = cat_gated_backward_weight(dy, packed, act=act, want_bias=False)
    assert none is None and torch.equal(again, dw)


def test_gradients_against_differences():
    """Central differences of dy . ((act(g) v) w^T) in 64 bits, for g, v and w; g and v are held exactly (integers up to 127)."""
    r = torch.Generator().manual_seed(0)
    g0, v0 = (torch.randint(-3, 4, (5, 24), generator=r).double() for _ in range(2))
    g0[:, 0] = v0[:, 0] = 127.0
    dy, w = torch.randn(5, 9, generator=r).float().double(), torch.randn(9, 24, generator=r).float().double()
    parts = [cat_pack8(t.float().cuda()) for t in (g0, v0)]
    packed = tuple(torch.stack(p) for p in zip(*parts))
    assert torch.equal(cat_unpack8(packed[0][0], packed[1][0]).double().cpu(), g0)
    h = 1e-5
    for act in ("none", "gelu", "gelu_tanh", "silu"):
        def f(g, v, wv):
            return float((dy * ((act_ref(g, act)[0] * v) @ wv.t())).sum())

        dz, db = (t.double().cpu() for t in cat_gated_backward_input(dy.float().cuda(), w.float().cuda(), packed, act=act))
        dw = cat_gated_backward_weight(dy.float().cuda(), packed, act=act)[0].double().cpu()
        for k, got in enumerate((dz[:, :24], dz[:, 24:], dw)):
            at = [g0, v0, w]
            want = torch.empty_like(at[k])
            for i in range(want.numel()):
                hi, lo = (t.clone() for t in (at[k], at[k]))
                hi.view(-1)[i] += h
                lo.view(-1)[i] -= h
                want.view(-1)[i] = (f(*at[:k], hi, *at[k + 1:]) - f(*at[:k], lo, *at[k + 1:])) / (2 * h)
            _close(got, want, 1e-5 * (1.0 + want.abs().max()), act)
        _close(db, dz.sum(0), 1e-5 * (1.0 + dz.abs().sum(0)), "db")


@pytest.mark.parametrize("M", [5, 200, 2100])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_nan_and_infinity_go_where_the_formula_takes_them(M, dtype):
    F = 75 if M < 1000 else 1032
    x, w = _matrix(M, 64, dtype, 1), _matrix(2 * F, 64, dtype, 2)
    clean, held = cat_gated_linear(x, w, act="gelu", pack=True)
    x[3, 10], w[F + 60, 0] = float("nan"), float("inf")
    y, packed = cat_gated_linear(x, w, act="gelu", pack=True)
    bad = torch.zeros(M, F, dtype=torch.bool, device="cuda")
    bad[3] = bad[:, 60] = True
    assert torch.equal(y[~bad], clean[~bad]) and bool(torch.isnan(y[3]).all()) and not bool(torch.isfinite(y[:, 60]).any())
    # the checkpoints: the gate's groups of row 3, the value's and with them all that share a scale with the infinity
    for i in range(2):
        g = cat_unpack8(packed[0][i], packed[1][i])
        assert bool(torch.isnan(g[3]).all())
        rows = torch.arange(M, device="cuda") != 3
        assert bool(torch.isnan(g[rows][:, :128]).all()) if i else torch.equal(g[rows], cat_unpack8(held[0][0], held[1][0])[rows])
        assert torch.equal(g[rows][:, 128:], cat_unpack8(held[0][i], held[1][i])[rows][:, 128:])


@pytest.mark.parametrize("M,F,K", [((1 << 20) + 300, 2056, 64), ((1 << 20) + 300, 8, 2056), ((1 << 20) + 300, 2051, 24)])
def test_more_than_two_to_the_31_entries(M, F, K):
    """Of the result, its checkpoints and gradients, or of x and dy (more than 4 GiB of them): first and last rows against the definitions."""
    x, w, w2 = _matrix(M, K, "bf16", 1), _matrix(2 * F, K, "bf16", 2, K ** -0.5), _matrix(K, F, "bf16", 3, K ** -0.5)
    half, ends = half_step(x.dtype), (slice(0, 400), slice(M - 400, M))
    y, packed = cat_gated_linear(x, w, act="relu", pack=True)
    alone = cat_gated_linear(x, w, act="relu")
    for rows in ends:
        z, z_err = x[rows].double() @ w.double().t(), U32 * (K + 8) * (x[rows].double().abs() @ w.double().abs().t())
        (g, v), (ge, ve) = z.split(F, 1), z_err.split(F, 1)
        want = g.clamp(min=0) * v
        bound = half * want.abs() * (1 + U32) + U32 * want.abs() + (ge * (v.abs() + ve) + g.abs() * ve) * (1 + half)
        _close(y[rows], want, bound, "y")
        _close(alone[rows], want, bound, "y without the checkpoint")
        for i, (t, err) in enumerate(((g, ge), (v, ve))):
            top, perr = _groups(t.abs(), lambda a: a.amax(2)), _groups(err, lambda a: a.amax(2))
            step, off = ((a.repeat_interleave(128, 1)[:, :F]) for a in (top / 127, perr))
            got = cat_unpack8(packed[0][i, rows].contiguous(), packed[1][i, rows].contiguous())
            _close(got, t, 0.5 * step + 2 * err + 2 * off + 256 * U32 * step, "checkpoint")
    del y, alone
    dz, _ = cat_gated_backward_input(x, w2, packed, act="relu")
    dy = torch.zeros_like(x)
    for rows in ends:
        dy[rows] = x[rows]
    dw, _ = cat_gated_backward_weight(dy, packed, act="relu", want_bias=False)
    want_w, size_w, err_w = 0, 0, 0
    for rows in ends:
        g, v = (cat_unpack8(packed[0][i, rows].contiguous(), packed[1][i, rows].contiguous()).double() for i in range(2))
        d = x[rows].double()
        dh, size = d @ w2.double(), d.abs() @ w2.double().abs()
        want, e = torch.cat((dh * v * (g > 0), dh * g.clamp(min=0)), 1), U32 * (K + 8) * size
        err = torch.cat((v.abs() * e, g.abs() * e), 1) + 3 * U32 * want.abs()
        _close(dz[rows], want, half * want.abs() + err * (1 + half), "dz")
        h = g.clamp(min=0) * v
        want_w, size_w = want_w + d.t() @ h, size_w + d.abs().t() @ h.abs()
        err_w = err_w + d.abs().t() @ (half * h.abs() + (1 + half) * U32 * h.abs())
    _close(dw, want_w, half * want_w.abs() + U32 * (M + 8) * size_w + err_w + 1e-30, "dw")


def test_no_rows():
    for dtype in TYPES.values():
        x, w = torch.empty(0, 33, dtype=dtype, device="cuda"), torch.ones(14, 33, dtype=dtype, device="cuda")
        y, packed = cat_gated_linear(x, w, pack=True)
        assert y.shape == (0, 7) and packed[0].shape == (2, 0, 7) and packed[1].shape == (2, 0, 1)
        dy, w2 = torch.empty(0, 5, dtype=dtype, device="cuda"), torch.ones(5, 7, dtype=dtype, device="cuda")
        dz, db = cat_gated_backward_input(dy, w2, packed)
        assert dz.shape == (0, 14) and db.shape == (14,) and not db.any()
        dw, db = cat_gated_backward_weight(dy, packed)
        assert dw.shape == (5, 7) and not dw.any() and not db.any()


def test_a_workspace_of_the_stated_size_is_enough_and_stays_in_its_bounds():
    lib = binding.load_library()
    for dtype, dt in (("f32", 0), ("bf16", 1)):
        for M, F, K in [(1, 64, 2048), (300, 65, 1030), (150, 130, 4096), (2000, 1001, 6000)]:
            x, w, dy, w2 = _matrix(M, K, dtype, 1), _matrix(2 * F, K, dtype, 2), _matrix(M, K, dtype, 3), _matrix(K, F, dtype, 4)
            packed = _held(M, F, dtype, 5)[0]
            size, back = lib.cat_gated_linear_workspace_bytes(M, F, K, dt), lib.cat_gated_backward_workspace_bytes(M, K, F, dt)
            for n, call in ((size, lambda ws: cat_gated_linear(x, w, pack=True, workspace=ws)[0]), (size, lambda ws: cat_gated_linear(x, w, workspace=ws)),
                            (back, lambda ws: cat_gated_backward_input(dy, w2, packed, workspace=ws)[0]),
                            (back, lambda ws: cat_gated_backward_weight(dy, packed, workspace=ws)[0])):
                buf = torch.full((n + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
                assert torch.equal(call(buf[:n]), call(None))
                assert bool((buf[n:] == 0xA5).all())
