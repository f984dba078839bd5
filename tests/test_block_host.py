"""What the operators of a block's training step refuse, and their sizes of workspace: host code, nothing is launched."""
import ctypes
import os

import pytest
import torch

from paper_2509_26277_amd import binding

INVALID, UNSUPPORTED, WORKSPACE = 1, 2, 3
FAKE = 0x7F0000001000  # never dereferenced: every case below fails validation first
A, B, C, D = (FAKE + (k << 20) for k in range(4))


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


def _pack(lib, **kw):
    return _call(lib.cat_pack8, dict(x=A, N=4, D=8, dt=0, codes=B, scales=C, stream=None), **kw)


def _unpack(lib, **kw):
    return _call(lib.cat_unpack8, dict(codes=A, scales=B, N=4, D=8, dt=0, x=C, stream=None), **kw)


def _norm(lib, **kw):
    return _call(lib.cat_layer_norm, dict(x=A, N=4, D=8, dt=0, weight=None, bias=None, eps=1e-5, y=B, mean=None, rstd=None, codes=None,
                                          scales=None, stream=None), **kw)


def _norm_packed(lib, **kw):
    return _call(lib.cat_layer_norm_packed, dict(codes=A, scales=B, mean=C, rstd=C, N=4, D=8, dt=0, weight=None, bias=None, y=D, stream=None), **kw)


def _norm_backward(lib, **kw):
    return _call(lib.cat_layer_norm_backward, dict(dy=A, x=B, codes=None, scales=None, mean=C, rstd=C, N=4, D=8, dt=0, weight=None, radd=None, dx=D,
                                                   dw=None, db=None, ws=FAKE, ws_bytes=1 << 30, stream=None), **kw)


def _linear(lib, **kw):
    return _call(lib.cat_linear, dict(x=A, w=B, bias=None, res=None, M=4, N=8, K=8, dt=1, act=0, y=C, codes=None, scales=None, ws=FAKE,
                                      ws_bytes=1 << 30, stream=None), **kw)


def _backward_input(lib, **kw):
    return _call(lib.cat_linear_backward_input, dict(dy=A, w=B, codes=None, scales=None, M=4, N=8, K=8, dt=1, act=0, dx=C, ws=FAKE,
                                                     ws_bytes=1 << 30, stream=None), **kw)


def _backward_weight(lib, **kw):
    return _call(lib.cat_linear_backward_weight, dict(dy=A, x=B, codes=None, scales=None, M=4, N=8, K=8, dt=1, act=0, dw=C, db=None, ws=FAKE,
                                                      ws_bytes=1 << 30, stream=None), **kw)


def _activation_backward(lib, **kw):
    return _call(lib.cat_activation_backward, dict(dy=A, codes=B, scales=C, N=4, D=8, dt=0, act=2, dz=D, stream=None), **kw)


ROWS = [(_pack, "x"), (_unpack, "x"), (_norm, "x"), (_norm_packed, "y"), (_norm_backward, "dy"), (_activation_backward, "dy")]
PRODUCTS = [(_linear, "x"), (_backward_input, "dy"), (_backward_weight, "dy")]


@pytest.mark.parametrize("call,rows", ROWS + PRODUCTS)
def test_types_pointers_and_alignment(lib, call, rows):
    assert call(lib, dt=7) == INVALID and b"dtype" in lib.cat_last_error()
    assert call(lib, **{rows: None}) == INVALID and b"NULL" in lib.cat_last_error()
    assert call(lib, **{rows: A + 8}) == INVALID and b"aligned" in lib.cat_last_error()


@pytest.mark.parametrize("call", [c for c, _ in ROWS])
def test_shapes_of_rows(lib, call):
    for kw in (dict(N=-1), dict(D=0), dict(D=-5), dict(N=1 << 31), dict(D=1 << 31)):
        assert call(lib, **kw) == INVALID


@pytest.mark.parametrize("call", [c for c, _ in PRODUCTS])
def test_shapes_of_products(lib, call):
    for kw in (dict(M=-1), dict(N=0), dict(K=0), dict(M=1 << 31), dict(N=1 << 31), dict(K=1 << 31)):
        assert call(lib, **kw) == INVALID
    assert call(lib, K=(1 << 22) + 8) == UNSUPPORTED  # bf16 rows of more than 8 MB
    assert call(lib, N=(1 << 22) + 8) == UNSUPPORTED


@pytest.mark.parametrize("call", [_linear, _backward_input, _backward_weight, _activation_backward])
def test_activations(lib, call):
    for act in (-1, 5, 99):
        assert call(lib, act=act) == INVALID and b"activation" in lib.cat_last_error()


@pytest.mark.parametrize("call", [_norm, _linear, _backward_input])
def test_codes_and_scales_come_together(lib, call):
    assert call(lib, codes=D) == INVALID and b"scales" in lib.cat_last_error()
    assert call(lib, scales=D) == INVALID and b"codes" in lib.cat_last_error()


@pytest.mark.parametrize("call", [_norm_backward, _backward_weight])
def test_rows_or_a_checkpoint(lib, call):
    assert call(lib, codes=D, scales=D) == INVALID and b"one of the two" in lib.cat_last_error()
    assert call(lib, x=None) == INVALID and b"one of the two" in lib.cat_last_error()
    assert call(lib, x=None, codes=D) == INVALID


@pytest.mark.parametrize("call", [_backward_input, _backward_weight])
def test_a_derivative_needs_its_argument(lib, call):
    assert call(lib, act=2) == INVALID and b"checkpoint" in lib.cat_last_error()


def test_aliases(lib):
    assert _norm(lib, y=A) == INVALID
    assert _norm_backward(lib, dx=A) == INVALID and _norm_backward(lib, dx=B) == INVALID and _norm_backward(lib, radd=D) == INVALID
    assert _linear(lib, y=A) == INVALID and _linear(lib, y=B) == INVALID and _linear(lib, res=C) == INVALID
    assert _backward_input(lib, dx=A) == INVALID and _backward_input(lib, dx=B) == INVALID
    assert _backward_weight(lib, dw=A) == INVALID and _backward_weight(lib, dw=B) == INVALID
    assert _activation_backward(lib, dz=A) == INVALID


def test_eps(lib):
    for eps in (-1e-5, float("nan"), float("inf")):
        assert _norm(lib, eps=eps) == INVALID and b"eps" in lib.cat_last_error()


@pytest.mark.parametrize("call", [_norm_backward, _linear, _backward_input, _backward_weight])
def test_workspace(lib, call):
    assert call(lib, ws=None) == WORKSPACE
    assert call(lib, ws=FAKE + 16) == WORKSPACE
    assert call(lib, ws_bytes=16) == WORKSPACE and b"need" in lib.cat_last_error()


def test_sizes_of_workspace(lib):
    f, g, h = lib.cat_linear_workspace_bytes, lib.cat_linear_backward_workspace_bytes, lib.cat_layer_norm_backward_workspace_bytes
    assert f(-1, 8, 8, 0) == 0 and f(8, 0, 8, 0) == 0 and f(8, 8, 8, 3) == 0 and g(8, 8, 0, 0) == 0 and h(4, 0, 0) == 0
    for M, N, K in [(0, 1, 1), (1, 8192, 2048), (4096, 1000, 512), (16384, 8192, 2048)]:
        for dt in (0, 1):
            assert f(M, N, K, dt) % 256 == 0 and f(M, N, K, dt) > 0 and g(M, N, K, dt) % 256 == 0 and g(M, N, K, dt) > 0
    # rows that are no whole number of 16-byte groups are laid out anew
    assert f(4096, 1000, 513, 0) >= (4096 + 1000) * 516 * 4
    assert h(1 << 20, 1024, 1) <= 1024 * 2 * 1024 * 4


def test_python_refuses_before_the_library(lib):
    x = torch.zeros(4, 8)
    for call in (lambda: binding.cat_pack8(x), lambda: binding.cat_layer_norm(x), lambda: binding.cat_linear(x, x)):
        with pytest.raises(ValueError):  # no device tensors
            call()
    with pytest.raises(TypeError):
        binding.cat_pack8(x.half())
    with pytest.raises(ValueError):
        binding.cat_pack8(x[0])
    with pytest.raises(ValueError):
        binding._act("tanh")
    assert ctypes.c_int(binding.ACTIVATIONS["silu"]).value == 4
