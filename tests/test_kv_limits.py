"""Calls at the ends of the cache operators' ranges, on the host: of no tokens,
of more than a launch or an argument can count, on several devices."""
import ctypes

import numpy as np
import pytest

import paper_2601_22787_amd as eq

FAKE = np.zeros(4096, dtype=np.uint8)
P = (FAKE.ctypes.data + 255) // 256 * 256


@pytest.mark.parametrize("rope", [False, True])
def test_norm_of_no_tokens(rope):
    """What torch gives for an empty tensor's address is 0."""
    r = eq.eq_rope(P, P, 10, 128, 0)
    at = ctypes.addressof(r) if rope else None
    for tokens, hq, hk, rc in ((0, 64, 8, eq.EQ_OK), (3, 0, 0, eq.EQ_OK), (1, 64, 0, eq.EQ_EINVAL)):
        assert eq.lib().eq_qk_norm_rope(None, hq * 128, hq, P, None, None, hk * 128, hk, P, None, 0,
                                        tokens, 128, 1e-5, None, at, None) == rc
    # what is no size of a head stays refused
    assert eq.lib().eq_qk_norm_rope(None, 8, 64, None, None, None, 8, 8, None, None, 0, 0, 72, 1e-5,
                                    None, None, None) == eq.EQ_EINVAL
