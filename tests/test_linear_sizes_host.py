"""The sizes of workspace of the products' gradients, which a program may have kept: what they were when the calls came.  Host code."""
import pytest

from test_gated_host import lib  # noqa: F401

# M, N, K, type, bytes
SIZES = [(129, 129, 129, 0, 168192), (129, 129, 129, 1, 102144), (4096, 129, 129, 0, 7439104), (4096, 129, 129, 1, 4276992), (16384, 1024, 4096, 0, 269484032),
         (16384, 1024, 4096, 1, 202375168), (8192, 256, 1000, 0, 50200576), (8192, 256, 1000, 1, 30351360), (16384, 257, 257, 0, 45145344),
         (16384, 257, 257, 1, 28103936), (300, 7, 9, 0, 77824), (300, 7, 9, 1, 77312), (5000, 2000, 3000, 0, 109160192), (5000, 2000, 3000, 1, 31336192),
         (5003, 1030, 1001, 0, 71140864), (5003, 1030, 1001, 1, 34152192), (65536, 129, 129, 0, 86148352), (65536, 129, 129, 1, 52593920), (1, 1, 1, 0, 768),
         (20000, 40, 33, 0, 5329664), (20000, 40, 33, 1, 2769664)]


@pytest.mark.parametrize("M,N,K,dt,size", SIZES)
def test_gradients_ask_for_no_more_than_they_did(lib, M, N, K, dt, size):  # noqa: F811
    assert lib.cat_linear_backward_workspace_bytes(M, N, K, dt) <= size
