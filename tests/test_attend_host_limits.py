"""Host-side limits of the attention and mass-eviction entry points that the
basic refusals do not reach.  Only calls that fail validation are made: the
addresses stand in for device memory and are never dereferenced."""
import ctypes

import pytest

import paper_2609_04971_amd as bkv
from test_attend_host import attend, shared


@pytest.mark.parametrize("call", [attend, shared])
def test_a_scale_that_leaves_fp32_in_log2_units(call):
    # kernels work in log2 units: scale * log2(e) is finite up to 2.3587e38 (2^128 / log2(e))
    for scale in (2.36e38, 3.0e38, 3.4e38):
        assert ctypes.c_float(scale).value != float("inf")
        assert call(scale=scale, n=16) == bkv.ERR_INVALID
    assert call(scale=2.35e38, n=16) == bkv.ERR_WORKSPACE  # the next check
