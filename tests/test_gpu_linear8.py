"""Products of 8-bit integers, plain and gated, against their definitions in 64 bits."""
import pytest
import torch

from paper_2509_26277_amd import binding, cat_gated_linear8, cat_linear8

from block_util import ACT_ERR, ACTS, SLOPE, TYPES, U32, act_ref, half_step

pytestmark = pytest.mark.gpu

# (M, N, K): single rows and few rows, tiles with ragged ends in every direction, lengths that are no whole 16-byte groups, shares
# of k, one entry; rows of 128 entries a step and one more; large tiles
SHAPES = [(1, 1, 1), (1, 16, 16), (1, 1000, 2048), (3, 17, 33), (16, 100, 512), (17, 130, 300), (33, 64, 272), (64, 257, 1030), (48, 96, 8192),
          (65, 128, 128), (66, 1, 7), (100, 129, 129), (128, 128, 256), (129, 257, 144), (300, 513, 1030), (200, 300, 8192), (777, 24, 63),
          (1025, 640, 144), (3600, 3590, 144), (3584, 3840, 400), (2000, 2003, 12000)]


def _codes(M, N, seed, low=-128):
    g = torch.Generator().manual_seed(seed)
    return torch.randint(low, 128, (M, N), generator=g).to(torch.int8).cuda()


def _floats(*shape, seed, scale=1.0):
    return (scale * torch.randn(*shape, generator=torch.Generator().manual_seed(seed))).cuda()


def _operands(M, N, K, seed=0):
    """Codes and scales such that the products are of order one, some rows of much larger and smaller scale."""
    x, w = _codes(M, K, 1 + seed), _codes(N, K, 2 + seed)
    xs, ws = torch.exp(_floats(M, seed=3 + seed)) / 74, torch.exp(0.5 * _floats(N, seed=4 + seed)) / (74 * K ** 0.5)
    return x, xs, w, ws


def _close(got, want, bound, what):
    assert got.shape == want.shape, what
    bad = ~((got.double() - want).abs() <= bound)
    assert not bool(bad.any()), (what, int(bad.sum()), torch.nonzero(bad)[:3].tolist())


def _product(x, xs, w, ws, b):
    """z and its error: the sum, the scales' product and what comes of both round once each, z with the bias once more."""
    p = (x.double() @ w.double().t()) * xs.double()[:, None] * ws.double()
    z = p if b is None else p + b.double()
    return z, U32 * (3 * p.abs() + z.abs())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_product(M, N, K, dtype):
    act, t = ACTS[(M + N + K) % len(ACTS)], TYPES[dtype]
    x, xs, w, ws = _operands(M, N, K)
    b, res = _floats(N, seed=5, scale=0.3), _floats(M, N, seed=6).to(t)
    z, z_err = _product(x, xs, w, ws, b)
    u = act_ref(z, act)[0]
    want = u + res.double()
    err = SLOPE * z_err + ACT_ERR * (1.0 + z.abs()) + U32 * want.abs()
    y = cat_linear8(x, xs, w, ws, b, act=act, residual=res, dtype=t)
    assert y.dtype == t
    _close(y, want, half_step(t) * want.abs() + err, "y")
    assert torch.equal(cat_linear8(x, xs, w, ws, b, act=act, residual=res, dtype=t), y)
    z, z_err = _product(x, xs, w, ws, None)
    _close(cat_linear8(x, xs, w, ws, dtype=t), z, half_step(t) * z.abs() + z_err, "product")


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,F,K", [(M, (N + 1) // 2, K) for M, N, K in SHAPES])
def test_gated_product(M, F, K, dtype):
    act, t = ACTS[(M + F + K) % len(ACTS)], TYPES[dtype]
    x, xs, w, ws = _operands(M, 2 * F, K)
    b = _floats(2 * F, seed=5, scale=0.3)
    for bias in (b, None):
        z, z_err = _product(x, xs, w, ws, bias)
        (g, v), (ge, ve) = z.split(F, 1), z_err.split(F, 1)
        u = act_ref(g, act)[0]
        ue = SLOPE * ge + ACT_ERR * (1.0 + g.abs())
        want = u * v
        y = cat_gated_linear8(x, xs, w, ws, bias, act=act, dtype=t)
        _close(y, want, half_step(t) * want.abs() * (1 + U32) + U32 * want.abs() + ue * (v.abs() + ve) + u.abs() * ve, "y")
        assert torch.equal(cat_gated_linear8(x, xs, w, ws, bias, act=act, dtype=t), y)


@pytest.mark.parametrize("act", ACTS)
@pytest.mark.parametrize("M", [2, 150, 2100])
def test_every_activation(M, act):
    N, K = (70, 40) if M < 1000 else (2056, 64)
    x, xs, w, ws = _operands(M, N, K)
    z, z_err = _product(x, xs, w, ws, None)
    for t in TYPES.values():
        want = act_ref(z, act)[0]
        _close(cat_linear8(x, xs, w, ws, act=act, dtype=t), want, half_step(t) * want.abs() + SLOPE * z_err + ACT_ERR * (1.0 + z.abs()), act)


@pytest.mark.parametrize("M", [3, 200])
def test_the_longest_sums_are_exact(M):
    """131071 products of the largest magnitude, of either sign: the sums of all but the last entry stay whole."""
    K, N = 131071, 20
    x, w = torch.full((M, K), -128, dtype=torch.int8, device="cuda"), torch.full((N, K), -128, dtype=torch.int8, device="cuda")
    w[1] = 127
    one_x, one_w = torch.ones(M, device="cuda"), torch.ones(N, device="cuda")
    y = cat_linear8(x, one_x, w, one_w, dtype=torch.float32)
    want = (x[:1].double() @ w.double().t()).float().expand(M, N)  # (rounded once)
    assert torch.equal(y, want) and float(y[0, 0]) == float(torch.tensor(131071.0 * 16384.0))


def test_exact_in_integers():
    """Scales of one and sums below 2^24: whole numbers, of either kernel, whatever the order."""
    for M, N, K in [(5, 40, 100), (300, 400, 1000), (2100, 2050, 128)]:
        x, w = _codes(M, K, 7), _codes(N, K, 8)
        y = cat_linear8(x, torch.ones(M, device="cuda"), w, torch.ones(N, device="cuda"), dtype=torch.float32)
        assert torch.equal(y.double(), x.double() @ w.double().t())


# more tiles than workgroups, of several steps of k: what a workgroup carries from one tile to the next
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("M,N,K", [(6144, 5120, 1024), (6001, 5003, 600), (4864, 4096, 128), (4867, 4099, 133),
                                   (8193, 2048, 130), (4142, 4096, 130), (8200, 2002, 130)])  # (the last three: few rows behind the last tile)
def test_many_tiles(M, N, K, dtype):
    t = TYPES[dtype]
    x, xs, w, ws = _operands(M, N, K)
    b, res = _floats(N, seed=5, scale=0.3), _floats(M, N, seed=6).to(t)
    z, z_err = _product(x, xs, w, ws, b)
    want = act_ref(z, "silu")[0] + res.double()
    _close(cat_linear8(x, xs, w, ws, b, act="silu", residual=res, dtype=t), want,
           half_step(t) * want.abs() + SLOPE * z_err + ACT_ERR * (1.0 + z.abs()) + U32 * want.abs(), "y")
    if N % 2 == 0:
        F = N // 2
        (g, v), (ge, ve) = z.split(F, 1), z_err.split(F, 1)
        u = act_ref(g, "gelu")[0]
        want = u * v
        ue = SLOPE * ge + ACT_ERR * (1.0 + g.abs())
        _close(cat_gated_linear8(x, xs, w, ws, b, act="gelu", dtype=t), want,
               half_step(t) * want.abs() * (1 + U32) + U32 * want.abs() + ue * (v.abs() + ve) + u.abs() * ve, "gated")


def _apart(codes, ld):
    """The same codes in rows ld entries apart, everything between and behind them as large as it can be."""
    buf = torch.full((codes.shape[0], ld), -128, dtype=torch.int8, device="cuda")
    buf[:, :codes.shape[1]] = codes
    return buf[:, :codes.shape[1]]


@pytest.mark.parametrize("M,N,K", [(1, 40, 33), (5, 100, 1030), (40, 4100, 4097), (70, 96, 1), (130, 258, 1030), (300, 130, 144), (200, 300, 4001), (2304, 2050, 133)])
def test_rows_that_lie_apart(M, N, K):
    """Rows on 16-byte boundaries, whatever lies between them; as one operand's, the other's, both's: the same bits."""
    x, xs, w, ws = _operands(M, N, K)
    for call in (cat_linear8, cat_gated_linear8):
        want = call(x, xs, w, ws, act="silu")
        for ld in ((K + 15) // 16 * 16, (K + 15) // 16 * 16 + 48):
            far_x, far_w = _apart(x, ld), _apart(w, ld)
            for a, b in ((far_x, w), (x, far_w), (far_x, far_w)):
                assert torch.equal(call(a, xs, b, ws, act="silu"), want), ld
    wide = _apart(x, (K + 15) // 16 * 16 + 16)
    for bad in (torch.empty((M + 1, K + 1), dtype=torch.int8, device="cuda")[1:, :K] if M > 1 else None,  # rows on any byte
                torch.empty((K, M), dtype=torch.int8, device="cuda").t() if M > 1 and K > 1 else None):
        if bad is not None and not bad.is_contiguous() and bad.stride(0) % 16:
            with pytest.raises(ValueError):
                cat_linear8(bad, xs, w, ws)
    assert torch.equal(cat_linear8(wide, xs, w, ws), cat_linear8(x, xs, w, ws))


@pytest.mark.parametrize("M,N,K", [(17, 1030, 8208), (40, 4100, 8208), (64, 4100, 8208), (64, 8200, 8208)])
def test_few_rows_by_a_large_weight_whose_rows_lie_apart(M, N, K):
    """What lies between the rows of w counts for nothing: the same bits, in a workspace of the stated size."""
    x, xs, w, ws = _operands(M, N, K)
    z, z_err = _product(x, xs, w, ws, None)
    want = z.clamp(min=0)
    y = cat_linear8(x, xs, w, ws, act="relu", dtype=torch.float32)
    _close(y, want, z_err + U32 * want, "y")
    room = torch.empty(binding.load_library().cat_linear8_workspace_bytes(M, N, K), dtype=torch.uint8, device="cuda")
    assert torch.equal(cat_linear8(x, xs, _apart(w, 3 * K), ws, act="relu", dtype=torch.float32, workspace=room), y)
    far = cat_gated_linear8(x, xs, _apart(w, 3 * K), ws, act="silu")
    assert torch.equal(far, cat_gated_linear8(x, xs, w, ws, act="silu"))


def test_a_view_whose_last_row_ends_with_its_memory_is_refused():
    view = torch.zeros(63 * 48 + 45, dtype=torch.int8, device="cuda").as_strided((64, 45), (48, 1))  # 48 entries of its last row are not there
    with pytest.raises(ValueError):
        cat_linear8(view, torch.ones(64, device="cuda"), torch.zeros(8, 45, dtype=torch.int8, device="cuda"), torch.ones(8, device="cuda"))


@pytest.mark.parametrize("M", [5, 200])
def test_nan_and_infinity_go_where_the_formula_takes_them(M):
    x, xs, w, ws = _operands(M, 150, 200)
    clean, clean_gated = cat_linear8(x, xs, w, ws, act="relu"), cat_gated_linear8(x, xs, w, ws, act="relu")
    x[3], xs[3], ws[140] = 0, float("inf"), float("nan")  # a row that held an infinity: zeros times infinity
    y, h = cat_linear8(x, xs, w, ws, act="relu"), cat_gated_linear8(x, xs, w, ws, act="relu")
    bad = torch.zeros(M, 150, dtype=torch.bool, device="cuda")
    bad[3] = bad[:, 140] = True
    assert torch.equal(torch.isnan(y), bad) and torch.equal(y[~bad], clean[~bad])
    bad = torch.zeros(M, 75, dtype=torch.bool, device="cuda")
    bad[3] = bad[:, 65] = True
    assert torch.equal(torch.isnan(h), bad) and torch.equal(h[~bad], clean_gated[~bad])


@pytest.mark.parametrize("M", [1, 300, 2304])
def test_activations_over_their_whole_range(M):
    """A sweep of arguments by a product of one entry (exact: codes and scales are powers of two and whole numbers), in either type
    and kernel: steps of 1 / 64 up to 31.75 on both sides, then what leaves the exponentials' range, infinities and NaN."""
    N = 4096
    x, xs = torch.ones(M, 1, dtype=torch.int8, device="cuda"), torch.ones(M, device="cuda")
    w = torch.zeros(N, 1, dtype=torch.int8, device="cuda")
    z = (torch.arange(N, device="cuda") - N // 2).double() / 64
    ends = [3e38, -3e38, 1e20, -1e20, 200.0, -200.0, float("inf"), float("-inf"), float("nan")]
    z[:len(ends)] = torch.tensor(ends, device="cuda").double()
    b = z.float()
    z = b.double()
    for act in ACTS:
        for t in TYPES.values():
            y = cat_linear8(x, xs, w, torch.ones(N, device="cuda"), b, act=act, dtype=t)
            assert torch.equal(y, y[:1].expand(M, N).contiguous()) or bool((torch.isnan(y) == torch.isnan(y[:1])).all())
            got = y[M - 1].double()
            want = act_ref(z[9:], act)[0]
            _close(got[9:], want, half_step(t) * want.abs() + ACT_ERR * (1.0 + z[9:].abs()), act)
            far = [float(v) for v in got[:9]]
            assert far[6] == float("inf") and far[8] != far[8]
            if act == "none":
                assert far[7] == float("-inf")
            else:  # relu(-inf) is 0, of the others -inf * 0
                assert far[7] == 0.0 if act == "relu" else far[7] != far[7]
                assert far[1] == 0.0 and far[3] == 0.0 and far[5] == 0.0 and far[4] == 200.0


@pytest.mark.parametrize("M,N,K", [((1 << 22) + 300, 8, 1040), ((1 << 21) + 300, 1032, 16), ((1 << 21) + 300, 1031, 24)])
def test_more_than_two_to_the_31_entries(M, N, K):
    """Of x (more than 4 GiB of it), or of the result: first and last rows against the definition."""
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randint(-128, 128, (M, K), generator=g, device="cuda", dtype=torch.int8)
    w = torch.randint(-128, 128, (2 * N, K), generator=g, device="cuda", dtype=torch.int8)
    xs, ws = torch.rand(M, generator=g, device="cuda") / 74, torch.rand(2 * N, generator=g, device="cuda") / (74 * K ** 0.5)
    y, h = cat_linear8(x, xs, w[:N], ws[:N], act="relu"), cat_gated_linear8(x, xs, w, ws, act="relu")
    half = half_step(y.dtype)
    for rows in (slice(0, 400), slice(M - 400, M)):
        z, z_err = _product(x[rows], xs[rows], w, ws, None)
        want, err = z[:, :N].clamp(min=0), z_err[:, :N]
        _close(y[rows], want, half * want + err + U32 * want, "y")
        (a, v), (ae, ve) = z.split(N, 1), z_err.split(N, 1)
        u = a.clamp(min=0)
        _close(h[rows], u * v, half * (u * v).abs() * (1 + U32) + U32 * (u * v).abs() + ae * (v.abs() + ve) + u * ve, "gated")


def test_no_rows():
    x, w = torch.empty(0, 33, dtype=torch.int8, device="cuda"), torch.ones(8, 33, dtype=torch.int8, device="cuda")
    none, ws = torch.empty(0, device="cuda"), torch.ones(8, device="cuda")
    assert cat_linear8(x, none, w, ws).shape == (0, 8) and cat_gated_linear8(x, none, w, ws).shape == (0, 4)


def test_a_workspace_of_the_stated_size_is_enough_and_stays_in_its_bounds():
    lib = binding.load_library()
    for M, N, K in [(1, 64, 8192), (300, 66, 1030), (150, 130, 8192), (2000, 2004, 12000)]:
        x, xs, w, ws = _operands(M, N, K)
        for size, call in ((lib.cat_linear8_workspace_bytes(M, N, K), cat_linear8), (lib.cat_gated_linear8_workspace_bytes(M, N // 2, K), cat_gated_linear8)):
            buf = torch.full((size + 4096,), 0xA5, dtype=torch.uint8, device="cuda")
            assert torch.equal(call(x, xs, w, ws, act="none", workspace=buf[:size]), call(x, xs, w, ws, act="none"))
            assert bool((buf[size:] == 0xA5).all())
