"""Rows to 8-bit integers, as they are and through layer norm, against their definitions in 64 bits."""
import pytest
import torch

from paper_2509_26277_amd import binding, cat_layer_norm_quantize, cat_pack8, cat_quantize_rows

from block_util import TYPES, U32, assert_close, norm_ref

pytestmark = pytest.mark.gpu

# around every boundary of the kernels: 16-byte groups, lanes and waves of a row, the longest row held in registers (8192)
LENGTHS = [1, 2, 7, 8, 24, 33, 64, 65, 129, 200, 257, 500, 515, 1000, 1001, 1030, 2048, 2050, 4096, 4104, 8191, 8192, 8200, 20001]


def _rows(N, D, dtype, seed, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(N, D, generator=g) * torch.exp(0.5 * torch.randn(D, generator=g)) + 0.5 * torch.randn(D, generator=g)
    buf = torch.full((N + 2, D), float("nan"), dtype=TYPES[dtype])  # nothing behind the last row may count
    buf[:N] = (x * scale).to(TYPES[dtype])
    return buf.cuda()[:N]


def _reference(x):
    """Codes and scales by the definition; its three roundings to 32 bits made from 64."""
    v = x.double().cpu()
    a = v.abs().amax(1, keepdim=True)
    held = a >= 2.0 ** -100
    safe = torch.where(held, a, torch.ones_like(a))
    up, step = (127.0 / safe).float().double(), (safe / 127.0).float()
    code = torch.where(held, torch.round((v * up).float()), torch.zeros_like(v).float())
    return code.to(torch.int8), torch.where(held, step, torch.zeros_like(step))[:, 0]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", LENGTHS)
def test_rows_are_the_definitions(D, dtype):
    N = 5 if D > 4096 else 67
    x = _rows(N, D, dtype, D)
    x[0] = 0
    x[1] *= 1e-35  # below 2^-100: held as zeros
    if D > 2:
        x[2, D // 2] = 1000.0  # one large entry: codes of the others near zero
        x[3] = x[3].abs().max()  # all at the end of the range
    codes, scales = cat_quantize_rows(x)
    want_c, want_s = _reference(x)
    assert torch.equal(scales.cpu(), want_s)
    assert torch.equal(codes.cpu(), want_c)
    if D <= 128:  # a row is one group of a checkpoint
        c, s = cat_pack8(x)
        assert torch.equal(c, codes) and torch.equal(s[:, 0], scales)


def test_more_rows_than_workgroups():
    for D in (24, 300, 2050, 3000):
        x = _rows(5003, D, "bf16", D)
        codes, scales = cat_quantize_rows(x)
        want_c, want_s = _reference(x)
        assert torch.equal(scales.cpu(), want_s) and torch.equal(codes.cpu(), want_c)


def test_rows_lie_on_16_byte_boundaries_and_nothing_else_is_written():
    lib = binding.load_library()
    for D in (1, 13, 130, 3001, 9001):
        x = _rows(21, D, "bf16", D)
        codes, scales = cat_quantize_rows(x)
        assert codes.shape == (21, D) and codes.stride(0) % 16 == 0
        for ld in (D, D + 3, (D + 15) // 16 * 16 + 16):
            buf, s = torch.full((23, ld), 77, dtype=torch.int8, device="cuda"), torch.empty(21, device="cuda")
            assert lib.cat_quantize_rows(x.data_ptr(), 21, D, 1, buf.data_ptr(), ld, s.data_ptr(), binding._stream()) == 0
            assert torch.equal(buf[:21, :D], codes) and torch.equal(s, scales)
            assert bool((buf[21:] == 77).all()) and bool((buf[:, D:] == 77).all())


def test_ties_go_to_the_even_code_and_the_largest_float_stays_finite():
    x = torch.tensor([[127.0, 0.5, 1.5, 2.5, -0.5, -1.5, -2.5, 126.5]], device="cuda")
    assert cat_quantize_rows(x)[0].tolist() == [[127, 0, 2, 2, 0, -2, -2, 126]]
    x = torch.tensor([[torch.finfo(torch.float32).max, 1.0]], device="cuda")
    codes, scales = cat_quantize_rows(x)
    assert codes.tolist() == [[127, 0]] and bool(torch.isfinite(127.0 * scales).all())


@pytest.mark.parametrize("D", [8, 300, 3000, 9000])
def test_nan_and_infinity_stay_in_their_row(D):
    x = _rows(5, D, "f32", 3)
    clean = cat_quantize_rows(x)
    x[1, D // 2], x[3, D - 1] = float("nan"), float("-inf")
    codes, scales = cat_quantize_rows(x)
    y = codes.float() * scales[:, None]
    assert bool(torch.isnan(y[1]).all()) and bool(torch.isnan(y[3]).all())
    for r in (0, 2, 4):
        assert torch.equal(codes[r], clean[0][r]) and scales[r] == clean[1][r]
    for bad in (1, 3):
        c, s = cat_layer_norm_quantize(x)
        assert bool(torch.isnan(c[bad].float() * s[bad]).all())


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("D", LENGTHS)
def test_norm_to_8_bits(D, dtype):
    N = 5 if D > 4096 else 67
    x = _rows(N, D, dtype, D + 1)
    g = torch.Generator().manual_seed(D)
    w, b = 1.0 + 0.3 * torch.randn(D, generator=g), 0.2 * torch.randn(D, generator=g)
    eps = 1e-5
    xd, wd, bd = x.double().cpu(), w.double(), b.double()
    for ww, bb in ((w, b), (None, None)):
        wr, br = (wd, bd) if ww is not None else (torch.ones(D, dtype=torch.float64), torch.zeros(D, dtype=torch.float64))
        h, mean, rstd = norm_ref(xd, wr, br, eps)
        codes, scales = cat_layer_norm_quantize(x, None if ww is None else ww.cuda(), None if bb is None else bb.cuda(), eps=eps)
        # sums of a row: chains of 64 additions, of D / 256 in rows that are not held; the mean's error moves the variance by its square
        chain = 74 + D // 256
        e_mean = chain * U32 * xd.abs().mean(1, keepdim=True)
        c = (xd - mean[:, None]).abs()
        rel = (0.5 * chain + 8) * U32 + (e_mean * rstd[:, None]) ** 2
        err = wr.abs() * rstd[:, None] * (e_mean + U32 * c) + wr.abs() * c * rstd[:, None] * rel + 2 * U32 * (h.abs() + br.abs())
        top, worst = h.abs().amax(1, keepdim=True), err.amax(1, keepdim=True)
        assert_close(scales, top[:, 0] / 127, ((worst + 4 * U32 * top) / 127)[:, 0], "scales")
        held = codes.double().cpu() * scales.double().cpu()[:, None]
        assert_close(held, h, 0.5 * top / 127 + err + 2 * worst + 256 * U32 * top / 127, "rows")
        assert bool((codes.cpu().int().abs().amax(1) == 127).all() if D > 1 else True)


@pytest.mark.parametrize("D", [2056, 2051])
def test_more_than_two_to_the_31_entries(D):
    """First and last rows against the definition; a row's codes through the norm do not hang on the number of rows."""
    N = (1 << 20) + 300
    x = torch.randn(N, D, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda", dtype=torch.bfloat16)
    codes, scales = cat_quantize_rows(x)
    norm_codes, norm_scales = cat_layer_norm_quantize(x)
    for rows in (slice(0, 100), slice(N - 100, N)):
        want_c, want_s = _reference(x[rows])
        assert torch.equal(scales[rows].cpu(), want_s) and torch.equal(codes[rows].cpu(), want_c)
        c, s = cat_layer_norm_quantize(x[rows].contiguous())
        assert torch.equal(norm_codes[rows], c) and torch.equal(norm_scales[rows], s)


def test_no_rows():
    for call in (cat_quantize_rows, cat_layer_norm_quantize):
        codes, scales = call(torch.empty(0, 33, device="cuda"))
        assert codes.shape == (0, 33) and scales.shape == (0,)
