"""CPU: what the query for the 8-bit cache's way refuses."""
import ctypes

import pytest

from paper_2609_25869_b200 import bsa
from tests.test_cache_host import INVALID, UNSUPPORTED, _built, cache, window  # noqa: F401


def way(w=None, c=None):
    a, b = ctypes.c_int(-1), ctypes.c_int(-1)
    return bsa.lib().bsa_debug_cache_way(w or window(), c or cache(), ctypes.byref(a), ctypes.byref(b))


@pytest.mark.parametrize("bad", [dict(batch=1), dict(heads_kv=4), dict(d=64), dict(N_kv=199), dict(heads=5), dict(left=-2), dict(N=0), dict(dtype=7)], ids=str)
def test_descriptions_that_a_forward_refuses(bad):
    assert way(window(**bad)) == INVALID


def test_caches_that_a_forward_refuses_and_missing_places():
    assert way(c=cache(block=8)) == INVALID and way(c=cache(ks=0)) == INVALID
    assert way(window(d=96), cache(d=96)) == UNSUPPORTED
    n = ctypes.c_int(0)
    L = bsa.lib()
    assert L.bsa_debug_cache_way(window(), cache(), None, ctypes.byref(n)) == INVALID
    assert L.bsa_debug_cache_way(window(), cache(), ctypes.byref(n), None) == INVALID
    assert L.bsa_debug_cache_way(None, cache(), ctypes.byref(n), ctypes.byref(n)) == INVALID
    assert L.bsa_debug_cache_way(window(), None, ctypes.byref(n), ctypes.byref(n)) == INVALID
