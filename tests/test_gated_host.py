"""What the gated operators and the products of 8-bit integers refuse, and their sizes of workspace: host code, nothing is launched."""
import os

import pytest
import torch

from paper_2509_26277_amd import binding

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
FAKE = 0x7F0000001000  # never dereferenced: every case below fails validation first
A, B, C, D, E = (FAKE + (k << 20) for k in range(5))


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.library_path()):
        from paper_2509_26277_amd import build
        build.build(verbose=False)
    return binding.load_library()


def _call(fn, defaults, **kw):
    a = dict(defaults)
    assert set(kw) <= set(a), kw
    a.update(kw)
    return fn(*a.values())


WS = dict(ws=FAKE, ws_bytes=1 << 40, stream=None)


def _quantize(lib, **kw):
    return _call(lib.cat_quantize_rows, dict(x=A, N=4, D=8, dt=0, codes=B, ld=8, scales=C, stream=None), **kw)


def _norm_quantize(lib, **kw):
    return _call(lib.cat_layer_norm_quantize, dict(x=A, N=4, D=8, dt=0, weight=None, bias=None, eps=1e-5, codes=B, ld=8, scales=C, stream=None), **kw)


def _linear8(lib, **kw):
    return _call(lib.cat_linear8, dict(x=A, ldx=16, xs=B, w=C, ldw=16, w_scales=D, bias=None, res=None, M=4, N=8, K=16, dt=1, act=0, y=E, **WS), **kw)


def _gated8(lib, **kw):
    return _call(lib.cat_gated_linear8, dict(x=A, ldx=16, xs=B, w=C, ldw=16, w_scales=D, bias=None, M=4, N=8, K=16, dt=1, act=0, y=E, **WS), **kw)


def _gated(lib, **kw):
    return _call(lib.cat_gated_linear, dict(x=A, w=B, bias=None, M=4, N=8, K=8, dt=1, act=0, y=C, codes=None, scales=None, **WS), **kw)


def _input(lib, **kw):
    return _call(lib.cat_gated_backward_input, dict(x=A, w=B, codes=C, scales=D, M=4, N=8, K=8, dt=1, act=0, y=E, db=None, **WS), **kw)


def _weight(lib, **kw):
    return _call(lib.cat_gated_backward_weight, dict(x=A, codes=C, scales=D, M=4, N=8, K=8, dt=1, act=0, y=E, db=None, **WS), **kw)


ROWS = [_quantize, _norm_quantize]
PRODUCTS = [_linear8, _gated8, _gated, _input, _weight]


@pytest.mark.parametrize("call", ROWS + PRODUCTS)
def test_types_pointers_and_alignment(lib, call):
    assert call(lib, dt=7) == INVALID and b"dtype" in lib.cat_last_error()
    assert call(lib, x=None) == INVALID and b"NULL" in lib.cat_last_error()
    assert call(lib, x=A + 8) == INVALID and b"aligned" in lib.cat_last_error()


@pytest.mark.parametrize("call,name", [(c, n) for c in ROWS for n in ("codes", "scales")] + [(c, n) for c in (_linear8, _gated8) for n in
                                       ("xs", "w", "w_scales", "y")] + [(_gated, "w"), (_gated, "y")] +
                         [(_input, n) for n in ("w", "codes", "scales", "y")] + [(_weight, n) for n in ("codes", "scales", "y")])
def test_every_array_is_needed(lib, call, name):
    assert call(lib, **{name: None}) == INVALID and b"NULL" in lib.cat_last_error()
    assert call(lib, **{name: E + 4}) == INVALID and b"aligned" in lib.cat_last_error()


@pytest.mark.parametrize("call,name", [(_norm_quantize, "weight"), (_norm_quantize, "bias"), (_linear8, "bias"), (_linear8, "res"), (_gated8, "bias"),
                                       (_gated, "bias"), (_input, "db"), (_weight, "db")])
def test_what_may_be_left_out_is_aligned_where_it_is_given(lib, call, name):
    assert call(lib, **{name: E + (1 << 20) + 4}) == INVALID and b"aligned" in lib.cat_last_error()


@pytest.mark.parametrize("call", ROWS)
def test_shapes_of_rows(lib, call):
    for kw in (dict(N=-1), dict(D=0), dict(D=-5), dict(N=1 << 31), dict(D=1 << 31)):
        assert call(lib, **kw) == INVALID


@pytest.mark.parametrize("call", PRODUCTS)
def test_shapes_of_products(lib, call):
    for kw in (dict(M=-1), dict(N=0), dict(K=0), dict(M=1 << 31), dict(N=1 << 31), dict(K=1 << 31)):
        assert call(lib, **kw) == INVALID
    assert call(lib, N=(1 << 22) + 8) == UNSUPPORTED  # bf16 rows of more than 8 MB


def test_long_sums(lib):
    for call in (_linear8, _gated8):
        assert call(lib, K=131072, ldx=131072, ldw=131072) == UNSUPPORTED and b"131071" in lib.cat_last_error()
    for call in (_gated, _input, _weight):
        assert call(lib, K=(1 << 22) + 8) == UNSUPPORTED


@pytest.mark.parametrize("call", PRODUCTS)
def test_activations(lib, call):
    for act in (-1, 5, 99):
        assert call(lib, act=act) == INVALID and b"activation" in lib.cat_last_error()


def test_distances_of_rows(lib):
    for call in ROWS:
        for ld in (7, 0, -8, 1 << 31):
            assert call(lib, ld=ld) == INVALID and b"apart" in lib.cat_last_error()
        assert call(lib, N=0, ld=8) == 0 and call(lib, N=0, ld=9) == 0
    for call in (_linear8, _gated8):
        for name in ("ldx", "ldw"):
            for ld in (0, 15, 17, 24, 40, (1 << 23) + 16):
                assert call(lib, **{name: ld}) == INVALID and b"apart" in lib.cat_last_error()
            assert call(lib, M=0, **{name: 32}) == 0
        assert call(lib, M=0, K=13, ldx=13, ldw=16) == 0 and call(lib, M=0, K=13, ldx=14, ldw=16) == INVALID


def test_codes_and_scales_come_together(lib):
    assert _gated(lib, codes=D) == INVALID and b"scales" in lib.cat_last_error()
    assert _gated(lib, scales=D) == INVALID and b"codes" in lib.cat_last_error()


def test_aliases(lib):
    for call in ROWS:
        assert call(lib, codes=A) == INVALID and call(lib, scales=A) == INVALID
    for call in (_linear8, _gated8):
        assert all(call(lib, y=p) == INVALID for p in (A, B, C, D)) and call(lib, bias=E) == INVALID
    assert _linear8(lib, res=E) == INVALID
    assert _gated(lib, y=A) == INVALID and _gated(lib, y=B) == INVALID and _gated(lib, bias=C) == INVALID
    assert all(_input(lib, y=p) == INVALID for p in (A, B, C, D)) and all(_weight(lib, y=p) == INVALID for p in (A, C, D))


def test_eps(lib):
    for eps in (-1e-5, float("nan"), float("inf")):
        assert _norm_quantize(lib, eps=eps) == INVALID and b"eps" in lib.cat_last_error()


@pytest.mark.parametrize("call", PRODUCTS)
def test_workspace(lib, call):
    assert call(lib, ws=None) == WORKSPACE
    assert call(lib, ws=FAKE + 16) == WORKSPACE
    assert call(lib, ws_bytes=16) == WORKSPACE and b"need" in lib.cat_last_error()


def test_no_rows_need_no_arrays(lib):
    for call in ROWS:
        assert call(lib, N=0, x=None, codes=None, scales=None) == 0
    for call in (_linear8, _gated8):
        assert call(lib, M=0, x=None, xs=None, y=None) == 0
    assert _gated(lib, M=0, x=None, y=None) == 0 and _input(lib, M=0, x=None, codes=None, scales=None, y=None) == 0


def test_sizes_of_workspace(lib):
    f, g, b, i, j = (lib.cat_gated_linear_workspace_bytes, lib.cat_gated_linear8_workspace_bytes, lib.cat_gated_backward_workspace_bytes,
                     lib.cat_linear8_workspace_bytes, lib.cat_gated_linear8_workspace_bytes)
    assert f(-1, 8, 8, 0) == 0 and f(8, 0, 8, 0) == 0 and f(8, 8, 8, 3) == 0 and b(8, 8, 0, 0) == 0 and i(8, 8, 0) == 0 and j(8, 8, 131072) == 0
    for M, N, K in [(0, 1, 1), (1, 8192, 2048), (4096, 1000, 512), (16384, 4096, 2048)]:
        for n in [i(M, N, K), g(M, N, K)] + [h(M, N, K, dt) for h in (f, b) for dt in (0, 1)]:
            assert n > 0 and n % 256 == 0
    # 256 bytes are stated where nothing is written (all calls may share them): a call that writes there, be it less, states more
    assert i(1, 8192, 2048) == 256 and g(1, 4096, 2048) == 256 and i(4096, 1024, 512) == 256
    for M in (1, 4, 100, 300):
        for N in (1, 8, 16):
            assert all(f(M, N, 8, dt) > 256 and b(M, 8, N, dt) > 256 for dt in (0, 1))  # a checkpoint's sums, sums over rows
            assert i(M, N, 1030) == 256 or i(M, N, 1030) > 256 and M > 64  # (laid out anew)
    for M, N, K in [(1, 1, 131071), (1, 2, 8192), (4, 16, 8192)]:  # shares of k of few rows: 4 bytes of sums and more
        assert i(M, N, K) > 256 and g(M, N, K) > 256
    # rows that are no whole number of 16-byte groups are laid out anew
    assert i(4096, 1000, 513) >= (4096 + 1000) * 528 and g(4096, 1000, 513) >= (4096 + 2000) * 528 and f(4096, 1000, 513, 0) >= (4096 + 2000) * 516 * 4


def test_python_refuses_before_the_library(lib):
    x, c, s = torch.zeros(4, 8), torch.zeros(4, 8, dtype=torch.int8), torch.zeros(4)
    for call in (lambda: binding.cat_quantize_rows(x), lambda: binding.cat_layer_norm_quantize(x), lambda: binding.cat_linear8(c, s, c, s),
                 lambda: binding.cat_gated_linear(x, x), lambda: binding.cat_gated_linear8(c, s, c, s)):
        with pytest.raises(ValueError):  # no device tensors
            call()
    with pytest.raises(ValueError, match="two rows for every channel"):
        binding.cat_gated_linear(x, x[:3])
    with pytest.raises(ValueError, match="two dimensions"):
        binding.cat_linear8(c[0], s, c, s)
    with pytest.raises(ValueError, match="three dimensions"):
        binding._gate(0, (c, s), 4)
    with pytest.raises(TypeError):
        binding.cat_linear8(c, s, c, s, dtype=torch.float16)
    with pytest.raises(TypeError):
        binding.cat_quantize_rows(x.half())


class _On:
    """As much of a tensor as the checks look at."""
    dtype, shape = torch.int8, torch.Size([4, 8])

    def __init__(self, index):
        self.index = index

    def get_device(self):
        return self.index

    def is_contiguous(self):
        return True

    def data_ptr(self):
        return FAKE


def test_tensors_of_another_device_are_refused(monkeypatch):
    monkeypatch.setattr(torch.cuda, "current_device", lambda: 1)
    assert binding._here(_On(1), "x") == 1 and binding._at(1, _On(1), torch.int8, (4, 8), "w") == FAKE and binding._at(1, None, None, None, "w") is None
    with pytest.raises(ValueError, match="current device"):
        binding._here(_On(0), "x")
    for other in (0, -1):
        with pytest.raises(ValueError, match="cuda:1"):
            binding._at(1, _On(other), torch.int8, (4, 8), "w")
        with pytest.raises(ValueError, match="cuda:1"):
            binding._room(1, _On(other), 256, None)
