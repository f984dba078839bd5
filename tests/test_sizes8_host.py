"""Sizes of workspace of the products of 8-bit integers: every shape that a call takes has one.  Host code, nothing is launched."""
import pytest
import torch

from paper_2509_26277_amd import binding

from test_gated_host import INVALID, UNSUPPORTED, WORKSPACE, _gated8, _linear8, lib  # noqa: F401

LONGEST = 1 << 22  # columns of bfloat16 rows of 8 MB
SHAPES = [(M, N, K) for M in (1, 48, 100, 300) for N in ((1 << 21) - 8, 1 << 21, (1 << 21) + 1, (1 << 21) + 16, LONGEST - 1, LONGEST) for K in (1, 16, 24, 33)]


@pytest.mark.parametrize("call,size", [(_linear8, "cat_linear8_workspace_bytes"), (_gated8, "cat_gated_linear8_workspace_bytes")])
def test_long_rows_of_bfloat16_results(lib, call, size):  # noqa: F811
    size = getattr(lib, size)
    for M, N, K in SHAPES:
        n = size(M, N, K)
        assert n >= 256 and n % 256 == 0, (M, N, K)
        # a byte less is refused for its size: the shape itself is taken, and so, being larger, is the stated size
        assert call(lib, M=M, N=N, K=K, ldx=K, ldw=K, ws_bytes=255) == WORKSPACE, (M, N, K)
        if n > 512:
            assert call(lib, M=M, N=N, K=K, ldx=K, ldw=K, ws_bytes=256) == WORKSPACE
            need = int(lib.cat_last_error().decode().split("need ")[1].split()[0])
            assert need <= n, (M, N, K)
    # float rows end at half as many columns, whatever the workspace
    assert call(lib, N=(1 << 21) + 8, dt=0) == UNSUPPORTED
    for N in (LONGEST + 1, LONGEST + 8):
        assert size(100, N, 33) == 0 and call(lib, M=100, N=N, K=33, ldx=33, ldw=33) == UNSUPPORTED


def test_a_size_of_0_gives_no_memory(lib):  # noqa: F811
    """A refused shape's call is not lent the bytes that calls without a workspace share."""
    room = binding._room(0, None, 0, torch.device("cpu"))
    assert room.numel() == 0
    assert _linear8(lib, N=LONGEST + 8, ws=room.data_ptr(), ws_bytes=room.numel()) == UNSUPPORTED
    assert _linear8(lib, ws=room.data_ptr(), ws_bytes=room.numel()) == WORKSPACE
    assert _linear8(lib, dt=9, ws=room.data_ptr(), ws_bytes=room.numel()) == INVALID
