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


def test_more_threads_than_a_launch_has():
    """A launch counts its threads in 32 bits. (The numbers below are just beyond; none of the addresses is read.)"""
    lib, P = B.load_library(), 1 << 20
    assert lib.blink_kv_cache_read(0, C.byref(cache()), P, 1 << 28, P, P, None) == B.ERR_TOO_LARGE               # 2 heads of 64: 16 threads a token
    assert lib.blink_kv_cache_read(0, C.byref(cache(n_kv_heads=64, head_dim=128, bits=4)), P, 1 << 22, P, P, None) == B.ERR_TOO_LARGE
    assert lib.blink_qk_norm_rope(0, C.byref(store(n_tokens=1 << 27)), None) == B.ERR_TOO_LARGE                  # 2^24 workgroups of 256
    assert lib.blink_qk_norm_rope(0, C.byref(store(n_tokens=1 << 26, cache=cache(bits=4, head_dim=128), q_stride=512, k_stride=256, v_stride=256, q_out_stride=512)), None) == B.ERR_TOO_LARGE
