"""The largest sizes that the operators around a decode step's attention take: a call beyond them is refused for its shape before anything is
launched, not by the launch.  (On the CPU; what is within them is asked of functions that launch nothing.)"""
from ctypes import c_int64

import pytest

from paper_2601_12698_amd import binding as B
from paper_2601_12698_amd import serving as S
from test_serving_checks import cache_read, cache_write


@pytest.mark.parametrize("call", [cache_write, cache_read])
@pytest.mark.parametrize("heads,d,lanes", [(8, 256, 32), (1, 144, 32), (3, 128, 16), (7, 96, 16), (8, 64, 8), (16, 16, 2)])
def test_a_cache_call_has_fewer_than_2_to_32_threads(call, heads, d, lanes):
    """A row of d elements takes `lanes` threads; a write rounds the tokens up to eight."""
    most = min((1 << 32) // (heads * lanes), (1 << 31) // heads)
    st = (c_int64 * 2)(heads * d, d)
    for tokens in (most, most + 1, most + 1000, (1 << 31) // heads - 9):
        if tokens >= most:
            assert call(tokens=tokens, heads=heads, d=d, ks=st, vs=st) == B.ERR_UNSUPPORTED_SHAPE, tokens
    fits = most - 300                                          # of whole workgroups of 256 threads
    assert S.load().kvcache_algorithmic_bytes(fits, heads, d, 0, 1) == 2 * fits * heads * (3 * d + 1) + 8 * fits
