"""CPU: what the 8-bit cache's entry points refuse before anything touches a device, and the reference that its GPU tests compare with."""
import pytest
import torch

from paper_2609_25869_b200 import bsa
from paper_2609_25869_b200 import build as bsa_build
from tests import cache_reference as C

INVALID, UNSUPPORTED = 1, 2
FAKE = 0x10000  # never dereferenced: the checks come first


@pytest.fixture(scope="module", autouse=True)
def _built():
    bsa_build.build()


def view(data=FAKE, batch=1 << 20, head=1 << 16, row=128):
    return bsa._VIEW.pack(data, batch, head, row)


def cache(k=None, v=None, ks=7 * FAKE, vs=8 * FAKE, scale_batch=64, scale_head=4, N=200, batch=2, heads=2, d=128, block=64):
    k, v = (dict(dict(data=a, batch=1 << 20, head=1 << 16, row=128), **(x or {})) for a, x in ((5 * FAKE, k), (6 * FAKE, v)))
    return bsa._CACHE.pack(*(k[n] for n in ("data", "batch", "head", "row")), *(v[n] for n in ("data", "batch", "head", "row")), ks, vs, scale_batch,
                           scale_head, N, batch, heads, d, block)


def rows(N=100, dtype=0, reserved=0, start=0, count=0):
    return bsa._ROWS.pack(N, dtype, reserved, start, count)


def window(batch=2, heads=4, heads_kv=2, d=128, N=100, N_kv=200, left=10, right=0, sinks=4, dtype=0, scale=0.0, start=0, length=0):
    return bsa._WINDOW.pack(batch, heads, heads_kv, d, N, N_kv, left, right, sinks, dtype, scale, start, length)


def write(c=None, r=None, k=None, v=None):
    return bsa.lib().bsa_cache_write(c or cache(), r or rows(), k or view(FAKE), v or view(2 * FAKE), None)


def read(c=None, r=None, k=None, v=None):
    return bsa.lib().bsa_cache_read(c or cache(), r or rows(), k or view(FAKE), v or view(2 * FAKE), None)


def forward(w=None, c=None, q=None, o=None, lse=3 * FAKE, ws=4 * FAKE, n=1 << 40):
    return bsa.lib().bsa_cache_forward(w or window(), c or cache(), q or view(FAKE), o or view(2 * FAKE), lse, ws, n, None)


CACHES = [dict(batch=0), dict(heads=0), dict(N=0), dict(d=0), dict(block=0), dict(block=8), dict(block=48), dict(block=256), dict(ks=0), dict(vs=0),
          dict(scale_batch=0), dict(scale_head=-1), dict(k=dict(data=0)), dict(v=dict(data=5 * FAKE + 8)), dict(k=dict(row=120)), dict(v=dict(row=8)),
          dict(k=dict(head=-16)), dict(v=dict(batch=(1 << 20) + 8)), dict(k=dict(row=1 << 38))]


@pytest.mark.parametrize("bad", CACHES, ids=str)
def test_caches_that_make_no_sense(bad):
    assert write(cache(**bad)) == INVALID and read(cache(**bad)) == INVALID and forward(c=cache(**bad)) == INVALID
    assert bsa.lib().bsa_cache_workspace_bytes(window(), cache(**bad)) == 0


@pytest.mark.parametrize("bad", [dict(d=96), dict(d=256), dict(N=(1 << 29) + 1), dict(batch=40000, heads=2)], ids=str)
def test_caches_beyond_the_kernels(bad):
    wide = dict(row=256, head=1 << 40, batch=1 << 50) if bad.get("N") else dict(row=256)
    for st in (write(cache(**bad)), read(cache(**bad))):
        assert st == UNSUPPORTED
    shape = dict(d=bad.get("d", 128), N_kv=bad.get("N", 200), batch=bad.get("batch", 2))
    assert forward(window(**shape), cache(**bad)) == UNSUPPORTED, wide


@pytest.mark.parametrize("bad", [dict(N=0), dict(N=-5), dict(dtype=2), dict(reserved=1), dict(start=FAKE + 2), dict(count=FAKE + 1)], ids=str)
def test_rows_that_make_no_sense(bad):
    assert write(r=rows(**bad)) == INVALID and read(r=rows(**bad)) == INVALID


def test_rows_beyond_the_kernels():
    assert write(r=rows(N=(1 << 29) + 1)) == UNSUPPORTED
    assert read(r=rows(N=(1 << 29) + 1), k=view(FAKE, 1 << 37, 1 << 37, 128)) in (INVALID, UNSUPPORTED)


@pytest.mark.parametrize("bad", [dict(data=0), dict(data=FAKE + 8), dict(row=0), dict(row=100), dict(head=-8), dict(batch=4), dict(row=1 << 38)], ids=str)
def test_views_that_the_kernels_cannot_follow(bad):
    for f in (write, read):
        assert f(k=view(**bad)) == INVALID and f(v=view(**bad)) == INVALID
    assert forward(q=view(**bad)) == INVALID and forward(o=view(**bad)) == INVALID


def test_null_arguments():
    L = bsa.lib()
    for f in (L.bsa_cache_write, L.bsa_cache_read):
        assert f(None, rows(), view(FAKE), view(2 * FAKE), None) == INVALID and f(cache(), None, view(FAKE), view(2 * FAKE), None) == INVALID
        assert f(cache(), rows(), None, view(FAKE), None) == INVALID and f(cache(), rows(), view(FAKE), None, None) == INVALID
    for i in range(4):
        args = [window(), cache(), view(FAKE), view(2 * FAKE)]
        args[i] = None
        assert L.bsa_cache_forward(*args, 3 * FAKE, 4 * FAKE, 1 << 40, None) == INVALID
    assert forward(lse=None) == INVALID and forward(lse=3 * FAKE + 2) == INVALID
    assert L.bsa_cache_workspace_bytes(None, cache()) == 0 and L.bsa_cache_workspace_bytes(window(), None) == 0


@pytest.mark.parametrize("bad", [dict(batch=1), dict(heads_kv=4), dict(d=64), dict(N_kv=199), dict(heads=5), dict(left=-2), dict(right=-2), dict(sinks=-1),
                                 dict(dtype=7), dict(scale=-1.0), dict(start=FAKE + 1), dict(N=0)], ids=str)
def test_descriptions_that_disagree_with_the_cache_or_make_no_sense(bad):
    assert forward(window(**bad)) == INVALID
    assert bsa.lib().bsa_cache_workspace_bytes(window(**bad), cache()) == 0


def test_outputs_in_the_place_of_another_tensor():
    """K, V and the scales are written by a write, K and V by a read, O by a forward."""
    for at in (5, 6, 7, 8):
        assert write(k=view(at * FAKE)) == INVALID and write(v=view(at * FAKE)) == INVALID
        assert read(k=view(at * FAKE)) == INVALID and read(v=view(at * FAKE)) == INVALID
        assert forward(o=view(at * FAKE)) == INVALID and forward(lse=at * FAKE) == INVALID
    assert read(k=view(FAKE), v=view(FAKE)) == INVALID
    assert write(cache(v=dict(data=5 * FAKE))) == INVALID and write(cache(vs=7 * FAKE)) == INVALID and write(cache(ks=5 * FAKE)) == INVALID


# codes of 2 x 2 x 200 tokens: rows that share elements, heads inside each other's rows, one stride for two dimensions; scales of four blocks
@pytest.mark.parametrize("bad", [dict(k=dict(row=64)), dict(v=dict(row=112)), dict(k=dict(head=64)), dict(v=dict(batch=1 << 16)), dict(scale_head=3),
                                 dict(scale_batch=4), dict(scale_batch=6)], ids=str)
def test_caches_whose_entries_overlap_are_not_written(bad):
    assert write(cache(**bad)) == INVALID
    assert read(k=view(row=64)) == INVALID and read(v=view(data=2 * FAKE, head=128)) == INVALID and forward(o=view(data=2 * FAKE, row=64)) == INVALID


def test_the_binding_refuses_what_does_not_fit_together():
    x = torch.zeros(2, 10, 64, dtype=torch.float8_e4m3fn)
    s = torch.zeros(2, 1, dtype=torch.uint8).view(torch.float8_e8m0fnu)
    with pytest.raises(ValueError):  # no CUDA tensors
        bsa.Cache(x, x, s, s)
    with pytest.raises(ValueError):
        bsa.cache_create(1, 2, 100, 64, device="cpu")
    assert (bsa._CACHE.size, bsa._ROWS.size) == (120, 32)


def test_the_reference_rounds_to_the_nearest_code():
    """Against torch's conversion, which rounds 32-bit values the same way; all halfway points among them."""
    t = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    x = torch.cat([t, (t[1:] + t[:-1]) / 2, torch.nextafter((t[1:] + t[:-1]) / 2, t[1:]), torch.rand(5000, dtype=torch.float64) * 448])
    x = torch.cat([x, -x]).float()
    a, b = C.nearest_code(x.double()), x.to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(a & 127, b & 127) and torch.equal((a | b)[x < 0] & 128, b[x < 0] & 128)
    assert (C.nearest_code(torch.tensor([float("inf"), float("nan")], dtype=torch.float64)) == 127).all()


def test_the_reference_takes_the_smallest_scale_and_keeps_what_is_there():
    x = torch.zeros(1, 1, 3, 64, dtype=torch.float64)
    x[0, 0, 0, 0], x[0, 0, 1, 1], x[0, 0, 2, 2] = 448.0, 1.0, 449.0
    codes, scales = torch.zeros(1, 1, 32, 64, dtype=torch.uint8), torch.zeros(1, 1, 2, dtype=torch.uint8)
    c, s = C.write(x[:, :, :2], codes, scales, 16, [0], [2])
    assert s[0, 0].tolist() == [127, 0]
    c2, s2 = C.write(x[:, :, 2:], c, s, 16, [2], [1])
    assert s2[0, 0].tolist() == [128, 0] and torch.equal(C.values(c2, s2, 16)[0, 0, :2], C.values(c, s, 16)[0, 0, :2])
    c3, s3 = C.write(x[:, :, 1:2], c2, s2, 16, [3], [1])
    assert s3[0, 0].tolist() == [128, 0] and float(C.values(c3, s3, 16)[0, 0, 3, 1]) == 1.0
