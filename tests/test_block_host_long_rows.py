"""The norm's backward pass of long rows: what it asks of its workspace.  Host code, nothing is launched."""
import os

import pytest

from paper_2509_26277_amd import binding

OK, WORKSPACE = 0, 3
FAKE = 0x7F0000001000  # never dereferenced: no rows, or a call that fails validation


@pytest.fixture(scope="module")
def lib():
    if not os.path.exists(binding.library_path()):
        from paper_2509_26277_amd import build
        build.build(verbose=False)
    return binding.load_library()


def _up(b):
    return (b + 255) // 256 * 256


def test_parts_are_no_more_than_rows(lib):
    size = lib.cat_layer_norm_backward_workspace_bytes
    for dt in (0, 1):
        assert size(1, 1 << 26, dt) == 2 * 4 << 26  # one part of dweight and dbias, half a gigabyte
        assert size(1, 1 << 30, dt) == 2 * 4 << 30
        assert size(3, 9001, dt) == _up(3 * 2 * 9001 * 4)
        assert size(1000, 9001, dt) == _up(64 * 2 * 9001 * 4)
        assert size(0, 9001, dt) >= 256


def test_without_the_parameters_gradients_a_small_workspace_is_enough(lib):
    def call(N, D, dw, db, ws_bytes):
        return lib.cat_layer_norm_backward(FAKE, FAKE + 4096, None, None, FAKE, FAKE, N, D, 0, None, None, FAKE + 8192, dw, db, FAKE, ws_bytes, None)

    for D in (8, 4000, 9001, 1 << 26):
        assert call(0, D, None, None, 256) == OK
        assert call(0, D, None, None, 128) == WORKSPACE
    for D in (4000, 9001, 1 << 26):
        assert call(2, D, FAKE + 16384, None, 256) == WORKSPACE and call(2, D, None, FAKE + 16384, 256) == WORKSPACE
