"""Numbers at the ends of their ranges, which the operators on device memory refuse before any device is asked for (no GPU needed)."""
import ctypes as C

import pytest

import paper_2604_07609_amd as B
from tests.test_operators_refusals import attend, cache, store  # noqa: F401


@pytest.mark.parametrize("scale", [2.4e38, 3.4e38])
def test_a_scale_that_overflows_in_units_of_powers_of_two(scale):
    """exp(x) is computed as 2^(x log2(e)): the scale times log2(e) has to be a number as well, or a score of 0 would be NaN."""
    lib = B.load_library()
    assert lib.blink_paged_attention(0, C.byref(attend(scale=scale)), None) == B.ERR_INVAL
    assert b"scale" in lib.blink_last_error()
