"""CPU: what the query for the 8-bit cache's way refuses, and places of LSE and of the workspace that a forward refuses."""
import ctypes

import pytest

from paper_2609_25869_b200 import bsa
from tests import test_window_host as W
from tests.test_cache_host import FAKE, INVALID, UNSUPPORTED, _built, cache, forward, window  # noqa: F401


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


def test_an_lse_or_a_workspace_in_the_place_of_another_tensor():
    """Outputs that begin where another tensor of the call does are refused (Q 1, O 2, LSE 3, workspace 4, codes 5 and 6, scales 7 and 8)."""
    for at in (1, 2):
        assert forward(lse=at * FAKE) == INVALID
    for at in (1, 2, 3, 5, 6, 7, 8):
        assert forward(ws=at * FAKE) == INVALID
    q, k, v, o = (W.view(i * FAKE) for i in (1, 2, 3, 4))
    for at in (1, 2, 3, 4):
        assert W.forward(window(), q, k, v, o, at * FAKE) == INVALID
    for args in ((q, k, v, o), (q, k, v, q)):  # (O may take the place of Q)
        assert W.forward(window(), *args, 5 * FAKE) != INVALID


def test_a_forward_without_such_overlaps_is_not_refused_on_the_host():
    assert forward() != INVALID and forward(o=W.view(FAKE)) != INVALID
