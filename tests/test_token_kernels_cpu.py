"""What the token kernels' sources have to hold whatever the compiler does with them."""
import os
import re

import paper_1911_00472_b200

CSRC = os.path.join(os.path.dirname(paper_1911_00472_b200.__file__), "csrc")


def test_tables_read_as_vectors_say_so():
    """Weights in shared memory are read as vectors of eight floats: their table asks for that alignment itself, and stands
    behind whole vectors of it."""
    with open(os.path.join(CSRC, "pcr_heads.cuh")) as f:
        text = f.read()
    alignment = int(re.search(r"struct alignas\((\d+)\) HeadTables", text)[1])
    assert alignment % (4 * 8) == 0
    pairs = int(re.search(r"kMaxHeadDim = (\d+);", text)[1]) // 2
    assert pairs * 8 % alignment == 0 and pairs * 4 % alignment == 0
