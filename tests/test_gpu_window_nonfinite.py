"""NaN and infinities where a row of windowed attention sees them: they belong to that row's outputs, and to no other row's."""
import math

import pytest
import torch

from paper_2609_25869_b200 import bsa
from tests import window_reference as R

pytestmark = pytest.mark.gpu


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def tensors(seed, b, h, hk, n, nk, d, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [torch.empty(s, device="cuda", dtype=dtype).normal_(0, 1, generator=g) for s in ((b, h, n, d), (b, hk, nk, d), (b, hk, nk, d))]


def check(q, k, v, clean, hit, **kw):
    """Rows of ``hit`` [batch, heads, N] are NaN in O and LSE; the others have the bits of the clean call."""
    O, L = bsa.window_forward(q, k, v, **kw)
    assert torch.isnan(O[hit]).all() and torch.isnan(L[hit]).all()
    assert torch.equal(O[~hit], clean[0][~hit]) and torch.equal(L[~hit], clean[1][~hit])


# (batch, heads, key heads, rows, keys): one CTA, clusters of several sizes, of sixteen; rows of several heads and windows in one block
FEW = [(1, 1, 1, 1, 40), (2, 8, 2, 1, 700), (1, 4, 1, 8, 900), (1, 8, 2, 4, 20000), (1, 1, 1, 1, 110000)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", FEW, ids=lambda s: "x".join(map(str, s)))
def test_a_row_of_few_that_sees_a_nan(size, d):
    b, h, hk, n, nk = size
    q, k, v = tensors(31, b, h, hk, n, nk, d)
    kw = dict(left=nk - 20, right=0, sinks=3)
    clean = bsa.window_forward(q, k, v, **kw)
    sees = R.sees(n, nk, b, nk - 20, 0, 3, None, None, "cuda")
    bad = q.clone()  # a query with one NaN
    bad[-1, -1, -1, 5] = math.nan
    hit = torch.zeros(b, h, n, dtype=torch.bool, device="cuda")
    hit[-1, -1, -1] = True
    check(bad, k, v, clean, hit, **kw)
    for j in (0, nk // 2, nk - n, nk - 1):  # one key of one key head
        bad = k.clone()
        bad[0, 0, j, -1] = math.nan
        hit = torch.zeros(b, h, n, dtype=torch.bool, device="cuda")
        hit[0, :h // hk] = sees[0, :, j]
        check(q, bad, v, clean, hit, **kw)
    bad = torch.full_like(k, math.nan)  # nothing but NaN: no maximum at all
    check(q, bad, v, clean, torch.ones(b, h, n, dtype=torch.bool, device="cuda"), **kw)
    bad = torch.where(torch.arange(nk, device="cuda")[:, None] == nk - n, math.inf, k.abs())  # an infinite score of every row
    check(q.abs(), bad, v, clean, torch.ones(b, h, n, dtype=torch.bool, device="cuda"), **kw)
    part = dict(kw, kv_len=ints([nk] * (b - 1) + [0]))  # no keys: still nothing seen, whatever the query holds
    O, L = bsa.window_forward(torch.full_like(q, math.nan), k, v, **part)
    assert not O[-1].any() and (L[-1] == -math.inf).all()


# (batch, heads, key heads, rows, keys, left, right, sinks): whole tiles, edges on every tile, several items per CTA
TILES = [(1, 2, 1, 300, 300, -1, 0, 0), (2, 4, 2, 400, 1000, 200, 60, 5), (1, 40, 40, 900, 900, 130, 0, 140)]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", TILES, ids=lambda s: "x".join(map(str, s)))
def test_a_row_of_a_tile_that_sees_a_nan(size, d, dtype):
    b, h, hk, n, nk, left, right, sinks = size
    q, k, v = tensors(32, b, h, hk, n, nk, d, dtype)
    kw = dict(left=left, right=right, sinks=sinks)
    clean = bsa.window_forward(q, k, v, **kw)
    sees = R.sees(n, nk, b, left, right, sinks, None, None, "cuda")
    bad = q.clone()
    hit = torch.zeros(b, h, n, dtype=torch.bool, device="cuda")
    for row in (0, 130, n - 1):
        bad[-1, -1, row, 5] = math.nan
        hit[-1, -1, row] = True
    check(bad, k, v, clean, hit, **kw)
    for j in (0, nk // 2, nk - 1):
        bad = k.clone()
        bad[0, 0, j, -1] = math.nan
        hit = torch.zeros(b, h, n, dtype=torch.bool, device="cuda")
        hit[0, :h // hk] = sees[0, :, j]
        check(q, bad, v, clean, hit, **kw)
    check(q, torch.full_like(k, math.nan), v, clean, torch.ones(b, h, n, dtype=torch.bool, device="cuda"), **kw)
    part = dict(kw, q_start=ints([0] * b), kv_len=ints([nk] * (b - 1) + [150]))  # rows behind the length: nothing seen, whatever they hold
    O, L = bsa.window_forward(torch.full_like(q, math.nan), k, v, **part)
    assert not O[-1, :, 150:].any() and (L[-1, :, 150:] == -math.inf).all() and torch.isnan(L[-1, :, :150]).all()


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("size", FEW, ids=lambda s: "x".join(map(str, s)))
def test_an_infinite_value_that_a_row_of_few_sees(size, d):
    """In its own column only, with its sign: the weights of all keys are above zero, so the sum is infinite, not NaN."""
    b, h, hk, n, nk = size
    q, k, v = tensors(33, b, h, hk, n, nk, d)
    kw = dict(left=-1, right=-1, scale=1e-3)
    O, L = bsa.window_forward(q, k, v, **kw)
    for j in (0, nk - 1):
        bad = v.clone()
        bad[0, 0, j, 3], bad[0, 0, j, d - 2] = math.inf, -math.inf
        want = O.clone()
        want[0, :h // hk, :, 3], want[0, :h // hk, :, d - 2] = math.inf, -math.inf
        O2, L2 = bsa.window_forward(q, k, bad, **kw)
        assert torch.equal(O2, want) and torch.equal(L2, L)


# batch, heads, key heads, rows, keys, left, right, sinks, starts, lengths: the sequences go on behind the last query
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("case", [(1, 1, 1, 8, 54, 1, 0, 0, [0], [21]), (2, 3, 1, 13, 118, 129, 1, 1, [65, 54], [118, 67]),
                                  (1, 8, 2, 153, 1174, 1, 0, 4, [0], [747]), (3, 16, 16, 249, 2687, 128, 30, 1, [0, 700, 2400], [771, 2687, 2500]),
                                  (1, 2, 2, 38, 1367, -1, 0, 0, [0], [1367])], ids=lambda c: "x".join(map(str, c[:8])))
def test_keys_behind_the_last_query_may_hold_anything(case, d):
    """Keys that only rows of the last tile behind the last query would see change no bit of the gradients, and have none of their own."""
    b, h, hk, n, nk, left, right, sinks, starts, lengths = case
    q, k, v = tensors(34, b, h, hk, n, nk, d)
    g = torch.randn_like(q)
    kw = dict(left=left, right=right, sinks=sinks, q_start=ints(starts), kv_len=ints(lengths))
    O, L = bsa.window_forward(q, k, v, **kw)
    G = bsa.window_backward(q, k, v, O, L, g, **kw)
    hidden = ~R.sees(n, nk, b, left, right, sinks, kw["q_start"], kw["kv_len"], "cuda").any(1)
    for value in (math.nan, math.inf):
        k2, v2 = k.clone(), v.clone()
        k2.transpose(1, 2)[hidden], v2.transpose(1, 2)[hidden] = value, value
        O2, L2 = bsa.window_forward(q, k2, v2, **kw)
        G2 = bsa.window_backward(q, k2, v2, O2, L2, g, **kw)
        assert torch.equal(O, O2) and torch.equal(L, L2) and all(torch.equal(x, y) for x, y in zip(G, G2))
    assert not G[1].transpose(1, 2)[hidden].any() and not G[2].transpose(1, 2)[hidden].any()
