"""The addresses that the products' tile ends form, on the host: the kernels' own functions, every lane of every tile, under an address
sanitizer."""
import os
import re
import shutil
import subprocess

import pytest

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2509_26277_amd", "csrc")
COMPILER = shutil.which("amdclang++") or "/opt/rocm/bin/amdclang++"

# whole tiles and ragged ones, rows of any alignment, fewer columns than a lane's eight; the shapes of the gradient tests' large tiles
SHAPES = [(1, 1), (1, 8), (1, 9), (17, 15), (300, 7), (255, 127), (256, 128), (257, 129), (129, 1001), (130, 1000), (255, 1003), (513, 1096), (100, 1032),
          (6001, 2503), (4864, 2048), (6144, 2560)]


@pytest.fixture(scope="module")
def program(tmp_path_factory):
    if not os.path.exists(COMPILER):
        pytest.skip("no compiler")
    d = tmp_path_factory.mktemp("ends")
    source = open(os.path.join(CSRC, "cat_gemm_kernel.h")).read()
    ends = source[source.index("// The epilogue of a wave's MT x 16 rows by 128 columns."):source.index("// Workgroups stay for all of their tiles")]
    ends = re.sub(r'asm volatile\(.*?\);', ";", ends, flags=re.S).replace("#pragma unroll\n", "")
    (d / "tile_ends.inc").write_text(ends)
    (d / "hip").mkdir()
    (d / "hip" / "hip_runtime.h").write_text('#include "host_device.h"\n')
    out = str(d / "tile_ends")
    subprocess.run([COMPILER, "-x", "c++", "-std=c++17", "-O1", "-w", "-Xarch_host", "-fsanitize=address", "-I", str(d), "-I", HERE,
                    "-I", os.path.join(os.path.dirname(HERE), "include"), "-I", CSRC, os.path.join(HERE, "tile_ends.cpp"), "-o", out], check=True)
    return out


@pytest.mark.parametrize("M,N", SHAPES)
def test_every_access_lies_in_its_array_and_every_entry_is_written(program, M, N):
    r = subprocess.run([program, str(M), str(N)], capture_output=True, text=True, env=dict(os.environ, ASAN_OPTIONS="detect_leaks=0"))
    assert r.returncode == 0, (r.stdout + r.stderr)[:2000]
