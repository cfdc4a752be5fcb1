"""Arguments of the token operators at the ends of their ranges."""
import struct

import pytest

from paper_1911_00472_b200 import binding as B

E = B.PCR_E_ARG


@pytest.mark.parametrize("std", [1e-45, 1e-41, 1.4e36, 3e38])
def test_deviations_that_no_scale_of_single_precision_stands_for(std):
    """Values are scaled by 1 / (255 std): 0 * inf would be no number, and nothing would be left of 1 / inf."""
    args = [1 << 20, 1000, 2 << 20, 2, 3 << 20, 10, 14, 2, struct.pack("3f", 0.5, 0.5, 0.5), struct.pack("3f", 0.2, std, 0.2), B.PCR_BF16, 4 << 20, None]
    assert B.lib().pcr_patch_tokens(*args) == E
