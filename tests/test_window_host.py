"""CPU: what the entry points for positions and windows refuse, before anything touches a device."""
import ctypes

import pytest
import torch

from paper_2609_25869_b200 import bsa
from paper_2609_25869_b200 import build as bsa_build

INVALID, UNSUPPORTED = 1, 2
FAKE = 0x10000  # never dereferenced: the checks come first


@pytest.fixture(scope="module", autouse=True)
def _built():
    bsa_build.build()


def view(data=FAKE, batch=1 << 20, head=1 << 16, row=128):
    return bsa._VIEW.pack(data, batch, head, row)


def window(batch=2, heads=4, heads_kv=2, d=128, N=100, N_kv=200, left=10, right=0, sinks=4, dtype=0, scale=0.0, start=0, length=0):
    return bsa._WINDOW.pack(batch, heads, heads_kv, d, N, N_kv, left, right, sinks, dtype, scale, start, length)


def forward(desc, q=None, k=None, v=None, o=None, lse=FAKE):
    vs = [x if x is not None else view() for x in (q, k, v, o)]
    return bsa.lib().bsa_window_forward(desc, *vs, lse, None)


def backward(desc, views=None, ws=FAKE, n=1 << 40):
    vs = views or [view()] * 8
    return bsa.lib().bsa_window_backward(desc, *vs[:4], FAKE, *vs[4:], ws, n, None)


def rope(**kw):
    c = dict(batch=2, heads=4, heads_kv=2, d=128, N=100, dtype=0, axes=(32, 48, 48), pairs=0, shared=0, inverse=0, theta=1e4, freq=0, pos=FAKE,
             pos_batch=300, first=0, grid=(0, 0, 0), origin=(0, 0, 0), q=None, k=None, qo=None, ko=None)
    c.update(kw)
    n = len(c["axes"])
    pad = (0,) * (4 - n)
    desc = bsa._ROPE.pack(c["batch"], c["heads"], c["heads_kv"], c["d"], c["N"], c["dtype"], n, *c["axes"], *pad, c["pairs"], c["shared"], c["inverse"], 0,
                          c["theta"], c["freq"], c["pos"], c["pos_batch"], c["first"], *c["grid"], *pad, *c["origin"], *pad)
    vs = [c[x] if c[x] is not None else view() for x in ("q", "k", "qo", "ko")]
    return bsa.lib().bsa_rope(desc, *vs, None)


@pytest.mark.parametrize("bad", [dict(batch=0), dict(heads=0), dict(heads_kv=0), dict(heads=5), dict(N=0), dict(N_kv=0), dict(N=-1),
                                 dict(left=-2), dict(right=-2), dict(sinks=-1), dict(dtype=2), dict(scale=-1.0), dict(scale=float("inf")),
                                 dict(scale=float("nan")), dict(start=FAKE + 2), dict(length=FAKE + 1)])
def test_window_descriptions_that_make_no_sense(bad):
    assert forward(window(**bad)) == INVALID and backward(window(**bad)) == INVALID
    assert bsa.lib().bsa_window_workspace_bytes(window(**bad)) == 0


@pytest.mark.parametrize("bad", [dict(d=256), dict(d=96), dict(d=32), dict(N=(1 << 29) + 1), dict(N_kv=1 << 40), dict(batch=40000, heads=2)])
def test_window_sizes_beyond_the_kernels(bad):
    assert forward(window(**bad)) == UNSUPPORTED and backward(window(**bad)) == UNSUPPORTED


@pytest.mark.parametrize("bad", [dict(data=0), dict(data=FAKE + 8), dict(row=0), dict(row=100), dict(head=-8), dict(batch=4), dict(row=1 << 38)])
def test_views_that_the_copies_cannot_follow(bad):
    for i in range(4):
        assert forward(window(), *[view(**bad) if j == i else view() for j in range(4)]) == INVALID
    for i in range(8):
        assert backward(window(), [view(**bad) if j == i else view() for j in range(8)]) == INVALID
    assert forward(window(), lse=None) == INVALID and forward(window(), lse=FAKE + 2) == INVALID
    for x in ("q", "k", "qo", "ko"):
        assert rope(**{x: view(**bad)}) == INVALID


def test_null_arguments():
    L = bsa.lib()
    assert L.bsa_window_forward(None, view(), view(), view(), view(), FAKE, None) == INVALID
    assert L.bsa_window_forward(window(), None, view(), view(), view(), FAKE, None) == INVALID
    assert L.bsa_window_backward(None, *[view()] * 4, FAKE, *[view()] * 4, FAKE, 1 << 40, None) == INVALID
    assert L.bsa_window_backward(window(), *[view()] * 4, None, *[view()] * 4, FAKE, 1 << 40, None) == INVALID
    assert L.bsa_rope(None, view(), view(), view(), view(), None) == INVALID
    assert L.bsa_window_status(None) == INVALID and L.bsa_window_workspace_bytes(None) == 0


@pytest.mark.parametrize("bad", [dict(batch=0), dict(heads=0), dict(heads_kv=-1), dict(N=0), dict(d=0), dict(dtype=5), dict(pairs=2),
                                 dict(axes=(31, 48, 48)), dict(axes=(-2, 48, 48)), dict(axes=(64, 64, 2)), dict(axes=(0, 0, 0)), dict(theta=0.0),
                                 dict(theta=float("nan")), dict(pos=FAKE + 2), dict(pos_batch=-1), dict(pos=0, grid=(1, 2, 0)),
                                 dict(pos=0, grid=(5, 5, 5)), dict(pos=0, grid=(4, 5, 5), first=1), dict(pos=0, grid=(1, 1, 1), first=-1),
                                 dict(pos=0, grid=(1 << 30, 1 << 30, 1 << 30))])
def test_rotations_that_make_no_sense(bad):
    assert rope(**bad) == INVALID


@pytest.mark.parametrize("origin", [(0, 0, (1 << 31) - 5), ((1 << 31) - 1, 0, 0), (0, (1 << 31) - 4, -(1 << 31))])
def test_a_grid_that_reaches_beyond_int32_positions(origin):
    assert rope(pos=0, grid=(4, 5, 6), N=120, origin=origin) == INVALID


def test_rotations_beyond_the_kernel():
    assert rope(d=100, axes=(16,), grid=(0,), origin=(0,)) == UNSUPPORTED
    assert rope(d=264, axes=(16,), grid=(0,), origin=(0,)) == UNSUPPORTED
    assert rope(N=(1 << 29) + 1) == UNSUPPORTED
    freqs = (ctypes.c_double * 64)(*([1.0] * 63 + [float("inf")]))
    assert rope(freq=ctypes.addressof(freqs)) == INVALID


def test_the_binding_refuses_what_does_not_fit_together():
    x = torch.zeros(2, 10, 64, dtype=torch.bfloat16)
    with pytest.raises(ValueError):  # no CUDA tensors
        bsa.rope(x, axes=[64], grid=[10])
    with pytest.raises(ValueError):
        bsa.window_forward(x, x, x, left=1)
    with pytest.raises(ValueError):
        bsa.window_backward(x, x, x, x, x, x, left=1)
    assert (bsa._VIEW.size, bsa._ROPE.size, bsa._WINDOW.size) == (32, 136, 80)


# d = 128 of 2 x 4 x 100 entries: rows that share elements, heads inside each other's rows, batches inside heads, one stride for two dimensions
@pytest.mark.parametrize("bad", [dict(row=64), dict(row=120), dict(head=64), dict(head=128 * 99), dict(batch=1 << 16), dict(batch=128 * 50, head=1 << 20),
                                 dict(row=1 << 16), dict(head=1 << 20), dict(batch=3 * (1 << 16) + 128 * 99), dict(row=(1 << 16) + 120)])
def test_outputs_whose_entries_overlap(bad):
    assert forward(window(N_kv=100), o=view(**bad)) == INVALID
    for i in (5, 6, 7):
        assert backward(window(N_kv=100, heads_kv=4), [view(**bad) if j == i else view() for j in range(8)]) == INVALID
    assert rope(qo=view(**bad), heads_kv=0) == INVALID and rope(ko=view(**bad), heads_kv=4) == INVALID


def test_outputs_in_the_place_of_what_is_still_read():
    """Q, K, V, O, dO, dQ, dK, dV by their numbers: dQ over Q, K, V, dO, dK, dV; dK over Q, dO, dV; dV over Q, dO; O over K, V."""
    own = [FAKE * (i + 1) for i in range(8)]
    square = window(N=100, N_kv=100, heads=4, heads_kv=4)  # so that any tensor can stand in for any other
    for out, others in ((5, (0, 1, 2, 4, 6, 7)), (6, (0, 4, 7)), (7, (0, 4))):
        for other in others:
            assert backward(square, [view(data=own[other if i == out else i]) for i in range(8)], n=1 << 50) == INVALID
    for other in (1, 2):
        assert forward(square, *[view(data=own[other if i == 3 else i]) for i in range(4)]) == INVALID
