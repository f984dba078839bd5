"""The tile kernel's loads go straight into LDS and its turning reads are assembly: the compiler does not see that one reads what
the other writes, so no barrier between them may stand without the kernel's own wait.  Reads the source; nothing is launched."""
import os
import re

SOURCE = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2509_26277_amd", "csrc", "cat_gemm_kernel.h")


def test_every_barrier_of_the_tile_kernel_stands_behind_a_wait():
    with open(SOURCE) as f:
        text = f.read()
    body = re.sub(r"//[^\n]*", "", text[text.index("void k_gemm("):text.index("cat_status launch_gemm_tiles")])
    statements = [s.strip() for s in body.split(";")]
    barriers = [i for i, s in enumerate(statements) if s.endswith("__syncthreads()")]
    assert len(barriers) == 2  # behind the first step's loads, and in a step
    for i in barriers:
        assert statements[i] == "__syncthreads()" and re.search(r'"s_waitcnt vmcnt\(0\)" ::: "memory"', statements[i - 1]), statements[i - 1]
