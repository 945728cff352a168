"""The 8-bit cache's attention way by way: what one call leaves for the next, and how far each way's roundings and NaN reach."""
import pytest
import torch

from paper_2609_25869_b200 import bsa
from tests import cache_bounds as B
from tests import cache_reference as C
from tests import window_reference as R
from tests.test_gpu_cache import check_forward, check_write, filled, garbage, generator, parts, queries
from tests.test_gpu_window import DT, ints

pytestmark = pytest.mark.gpu


class Call:
    """bsa_cache_forward through the C ABI, with the positions, the outputs and the workspace in the caller's hands."""

    def __init__(self, q, cache, left, right=0, sinks=0):
        self.q, self.cache, self.window = q, cache, (left, right, sinks)
        some = ints([0] * cache.batch)
        self.need = bsa.lib().bsa_cache_workspace_bytes(self.desc(some, some), cache._packed)

    def desc(self, start, length):
        b, h, n, d = self.q.shape if self.cache.layout == "hnd" else (self.q.shape[i] for i in (0, 2, 1, 3))
        return bsa._WINDOW.pack(b, h, self.cache.heads, d, n, self.cache.N, *self.window, bsa._tensor_of(self.q, "Q")[0], 0.0,
                                start.data_ptr(), length.data_ptr())

    def __call__(self, start, length, O, LSE, ws):
        nhd, dev = self.cache.layout == "nhd", self.q.get_device()
        vq, vo = (bsa._view(x, nhd, self.q.dtype, dev, "Q")[4] for x in (self.q, O))
        assert bsa.lib().bsa_cache_forward(self.desc(start, length), self.cache._packed, vq, vo, LSE.data_ptr(), ws.data_ptr(), ws.numel(),
                                           torch.cuda.current_stream().cuda_stream or None) == 0


@pytest.mark.parametrize("n,nk,left", [(300, 5000, 200), (300, 9000, -1), (1, 40000, -1)])
@pytest.mark.parametrize("d", [64, 128])
def test_a_workspace_used_again_holds_nothing_of_the_call_before(n, nk, left, d):
    """Calls one right behind the other with one workspace, each at other positions (which the 16-bit way keeps there, written by a kernel that is
    still running when the attention kernel starts): the bits of calls alone."""
    cache, _ = filled(31, 2, 2, nk, d, "bf16", "hnd", 64)
    q = queries(31, 2, 4, n, d, "bf16", "hnd")
    call = Call(q, cache, left, 3, 5)
    places = [([nk - n, 1000], [nk, 1000 + n]), ([0, 2222], [n, 3000]), ([700, nk - n - 1], [701 + n, nk]), ([1500, -3], [4000, 90])]
    places = [(ints(a), ints(b)) for a, b in places]

    def outputs():
        return torch.empty_like(q), torch.empty(2, 4, n, device="cuda")
    alone = []
    for start, length in places:
        O, L = outputs()
        call(start, length, O, L, torch.full((max(call.need, 256),), 255, dtype=torch.uint8, device="cuda"))
        torch.cuda.synchronize()
        alone.append((O, L))
    ws = torch.full((max(call.need, 256),), 255, dtype=torch.uint8, device="cuda")
    got = [(i % 4, *outputs()) for i in range(40)]
    torch.cuda.synchronize()
    for i, O, L in got:
        call(*places[i], O, L, ws)
    torch.cuda.synchronize()
    for i, O, L in got:
        assert torch.equal(O, alone[i][0]) and torch.equal(L, alone[i][1])
    assert bsa.window_status() == 0


def tiny(cache, g, size):
    """Writes normal keys, and values around `size`, all of one sign, so that nothing cancels; both in 64 bits."""
    shape = cache.K.shape
    k = torch.empty(shape, device="cuda").normal_(0, 1, generator=g).bfloat16()
    v = torch.empty(shape, device="cuda").uniform_(0.5, 1.0, generator=g).double().mul_(size).bfloat16()
    bsa.cache_write(cache, k, v)
    return [C.values(c, s, cache.block).cuda() for c, s in parts(cache)]


# one row; few rows in parts; through 16 bits; from the codes, uncut and in parts
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("b,h,hk,n,nk", [(1, 4, 2, 1, 700), (1, 4, 2, 1, 40000), (2, 2, 1, 300, 700), (5, 14, 14, 64, 6000), (1, 4, 2, 300, 6000)])
def test_values_near_the_types_smallest(b, h, hk, n, nk, d):
    """Scales of V down to the smallest there is: the reciprocal of a row's sum times such a scale is no normal number, the outputs are."""
    cache = bsa.cache_create(b, hk, nk, d)
    values = tiny(cache, generator(32), 2.0 ** -117)
    assert int(cache.V_scale.view(torch.uint8).max()) <= 2
    q = queries(32, b, h, n, d, "bf16", "hnd")
    O, L = bsa.cache_forward(q, cache, left=-1, right=-1, q_start=ints([0] * b))
    wO, wL, tO, tL = C.forward(q, *values, left=-1, right=-1, q_start=ints([0] * b))
    up = 2.0 ** 117  # (the comparison's own least number is far above these)
    R.assert_within(O.double() * up, wO * up, tO * up, "O")
    R.assert_within(L, wL, tL, "LSE")
    assert bsa.window_status() == 0


@pytest.mark.parametrize("block,d", [(16, 64), (32, 64), (16, 128)])  # of 32 threads each
def test_a_scale_that_grows_under_one_warp(block, d):
    """Tokens one by one, each twice as loud as the one before: every lane of a block's warp has to see the scale as it was."""
    g = generator(33)
    cache = bsa.cache_create(4, 9, 3 * block, d, block=block)
    for i in range(block + 5):
        k, v = (torch.empty(4, 9, 1, d, device="cuda").normal_(0, 1, generator=g).mul_(2.0 ** (i % 23 - 11)).bfloat16() for _ in range(2))
        check_write(cache, k, v, [i, i + block - 5, max(0, i - 7), 0])


@pytest.mark.parametrize("block,start", [(16, 5), (64, 100), (128, 64)])
@pytest.mark.parametrize("foreign", [0, 90, 254, 255])
def test_a_first_write_inside_a_block(foreign, block, start):
    """Memory that held another sequence (codes of any byte, NaN among them): with the block's scales zeroed the new tokens get the smallest scale that takes them,
    and rows that see them alone are finite; a scale left there counts as that of tokens in front."""
    b, h, n, d = 2, 2, 150, 64
    g = generator(34)
    cache = garbage(34, b, h, 512, d, block, scales=(foreign, foreign + 1))
    for i in range(b):  # both sequences' slots, as a user clears them
        cache.K_scale.view(torch.uint8)[i].zero_()
        cache.V_scale.view(torch.uint8)[i].zero_()
    k, v = (torch.empty(b, h, n, d, device="cuda").normal_(0, 1, generator=g).bfloat16() for _ in range(2))
    check_write(cache, k, v, [start, start], None)
    alone = bsa.cache_create(b, h, 512, d, block=block)
    bsa.cache_write(alone, k, v, start=ints([start, start]))
    first, last = start // block, (start + n - 1) // block
    for mine, want in zip(parts(cache), parts(alone)):
        assert torch.equal(mine[1][..., first:last + 1], want[1][..., first:last + 1])
        assert torch.equal(mine[0][:, :, start:start + n] & 127, want[0][:, :, start:start + n] & 127)
    for rows in (1, 40):
        q = queries(34, b, 4, rows, d, "bf16", "hnd")
        kw = dict(left=30, q_start=ints([start + n - rows] * b), kv_len=ints([start + n] * b))
        O, L = bsa.cache_forward(q, cache, **kw)
        O2, L2 = bsa.cache_forward(q, alone, **kw)
        assert torch.isfinite(O).all() and torch.equal(O, O2) and torch.equal(L, L2)
    if foreign:
        cache.K_scale.view(torch.uint8)[0, :, first] = foreign
        check_write(cache, k, v, [start, start], None)
        assert int(cache.K_scale.view(torch.uint8)[0, 0, first]) == max(foreign, int(parts(alone)[0][1][0, 0, first]))


# ------------------------------------------------------------------ which way, and each way's own
def test_every_way_is_taken_by_the_sizes_that_the_tests_use():
    """The rule's constants may change; then the sizes of the tests in this file and its neighbour have to follow."""
    for d in (64, 128):
        for n, nk, left, want in [(1, 600, -1, "rows"), (1, 40000, -1, "rows"), (300, 700, -1, "unpacked"), (300, 5000, 200, "unpacked"), (300, 6000, -1, "tiles")]:
            cache = bsa.cache_create(2, 2, nk, d)
            q = torch.empty(2, 4, n, d, device="cuda", dtype=torch.bfloat16)
            way, parts_ = bsa.debug_cache_way(q, cache, left=left)
            assert way == want and (parts_ > 1) == (nk >= 6000 and n > 1 or nk == 40000)


#       b  h   hk  n    nk    left  right sinks starts                  lengths                   at least so many items for each of the GPU's pairs of CTAs
MANY = [
    (5, 40, 40, 200, 2000, -1, 0, 0, None, None, 3),
    (5, 40, 40, 200, 2000, -1, 7, 0, [1800, -200, 50, 1900, -70], [2000, 0, 250, 1999, 130], 3),      # no key; rows behind, rows in front of the sequence
    (5, 40, 40, 200, 2000, 1200, 5, 130, [1800, 0, 1000, 1900, 300], [2000, 200, 1100, 2000, 0], 3),  # a window, first tokens, rows behind, no key
    (4, 37, 37, 200, 3000, -1, -1, 0, None, None, 2),
    (3, 9, 3, 100, 9000, -1, 0, 0, None, None, 2),                                                    # in parts
    (3, 9, 3, 100, 9000, 8500, 0, 40, [8900, -100, 600], [9000, 0, 700], 2),                          # parts without a tile
    (3, 5, 5, 520, 12000, -1, 0, 0, [11480, 4000, 11000], [12000, 4520, 11520], 2),                   # three tiles of rows
    (5, 14, 14, 64, 6000, -1, 0, 0, [5936, 1, 0, 600, 5000], [6000, 65, 0, 664, 5064], 1),            # uncut, an item a pair
    (4, 12, 12, 64, 300, 500, 0, 0, None, None, 1),
]


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (64, "fp16"), (128, "bf16"), (128, "fp16")])
@pytest.mark.parametrize("block,layout", [(16, "hnd"), (64, "nhd")])
@pytest.mark.parametrize("case", MANY, ids=lambda c: "x".join(str(x) for x in c[:8]))
def test_rows_by_the_tile_item_after_item(case, block, layout, d, dtype):
    """The kernel that reads the codes with several items for each pair of CTAs, whole ones and parts: what one item hands to the next."""
    b, h, hk, n, nk, left, right, sinks, starts, lengths, rounds = case
    cache, values = filled(sum(case[1:5]) + d, b, hk, nk, d, dtype, layout, block, 0.8)
    q = queries(n + nk, b, h, n, d, dtype, layout)
    kw = dict(left=left, right=right, sinks=sinks, q_start=ints(starts), kv_len=ints(lengths))
    way, cut = bsa.debug_cache_way(q, cache, **kw)
    assert way == "tiles"
    pairs = torch.cuda.get_device_properties(0).multi_processor_count // 2
    assert -(-n // 256) * b * h * cut > (rounds - 1) * pairs
    check_forward(q, cache, values, **kw)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("way,b,h,hk,n,nk", [("rows", 1, 4, 2, 3, 500), ("rows", 1, 4, 2, 3, 40000), ("unpacked", 2, 2, 1, 300, 700), ("tiles", 1, 4, 2, 300, 6000),
                                             ("tiles", 5, 14, 14, 64, 6000)])
def test_queries_at_the_ends_of_their_type(way, b, h, hk, n, nk, dtype):
    """Rows up to the type's largest numbers and down to its smallest, with a scale that takes their scores back; a row of zeros sees its keys evenly."""
    cache, values = filled(35, b, hk, nk, 128, dtype, "hnd", 64)
    kw = dict(left=-1, right=-1, q_start=ints([0] * b))
    ends = ((2.0 ** 120, 2.0 ** -124), (2.0 ** -115, 2.0 ** 111)) if dtype == "bf16" else ((2.0 ** 12, 2.0 ** -16), (2.0 ** -12, 2.0 ** 8))
    q = queries(35, b, h, n, 128, dtype, "hnd")
    assert bsa.debug_cache_way(q, cache, **kw)[0] == way
    for f, scale in (*ends, (0.0, 0.0)):
        check_forward((q.float() * f).to(q.dtype), cache, values, scale=scale, **kw)


@pytest.mark.parametrize("way,b,h,hk,n,nk", [("rows", 1, 4, 2, 3, 500), ("unpacked", 2, 2, 1, 300, 700), ("tiles", 1, 4, 2, 300, 6000)])
@pytest.mark.parametrize("scale,loud", [(2.0 ** 120, 2.0 ** 20), (2.0 ** -80, 2.0 ** -20)])
def test_factors_beyond_32_bits(scale, loud, way, b, h, hk, n, nk):
    """Scores of zero, or so small that they are none, under a factor that has no number in 32 bits: every key that is seen has the same weight, none besides."""
    g = generator(36)
    cache = bsa.cache_create(b, hk, nk, 64)
    k, v = (torch.empty(b, hk, nk, 64, device="cuda").normal_(0, 1, generator=g).mul_(f).bfloat16() for f in (loud, 1.0))
    q = torch.zeros(b, h, n, 64, dtype=torch.bfloat16, device="cuda")
    k[..., 0] = 0
    q[..., 0] = loud
    bsa.cache_write(cache, k, v)
    V = C.values(*parts(cache)[1], 64).cuda().repeat_interleave(h // hk, 1)
    start = nk - n - 7
    kw = dict(left=-1, q_start=ints([start] * b))
    assert bsa.debug_cache_way(q, cache, **kw)[0] == way
    O, L = bsa.cache_forward(q, cache, scale=scale, **kw)
    count = torch.arange(start + 1, start + n + 1, device="cuda").double()
    want = V.cumsum(2)[:, :, start:start + n] / count[:, None]
    assert (L.double() - count.log()).abs().max() <= 2.0 ** -17
    # P is one for every key: the mean of V in 32 bits (2^-19 of its absolute values), rounded once
    assert ((O.double() - want).abs() <= 2.0 ** -8 * want.abs() * 1.01 + 2.0 ** -18 * V.abs().amax()).all()


@pytest.mark.parametrize("what", ["K", "V", "K_scale", "V_scale"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("way,h,n,nk,tile", [("rows", 8, 3, 705, 2), ("rows", 8, 3, 40001, 2), ("unpacked", 2, 600, 700, 128), ("tiles", 2, 600, 6000, 256)])
def test_a_nan_that_some_rows_see(way, h, n, nk, tile, d, what):
    """Causal rows: those that see a NaN code, or any of a block whose scale is 255, are NaN; those of other tiles keep every bit."""
    block = 16
    cache, _ = filled(37, 1, 1, nk, d, "bf16", "hnd", block)
    q = queries(37, 1, h, n, d, "bf16", "hnd")
    key = -(-(nk - n + (2 if n == 3 else 530)) // block) * block  # the first key of a block, at the position of row 530 or a little behind it
    sees = key - (nk - n)                                         # the first row that sees it
    apart = sees // tile * tile
    assert 0 < apart <= sees < n
    kw = dict(left=-1)
    assert bsa.debug_cache_way(q, cache, **kw)[0] == way
    for s in (cache.K_scale, cache.V_scale):  # the block is none of the largest scale, which the others' roundings go by
        s.view(torch.uint8)[..., key // block] = 1
    O, L = bsa.cache_forward(q, cache, **kw)
    if what in ("K", "V"):
        getattr(cache, what).view(torch.uint8)[0, 0, key, 5] = 127
    else:
        getattr(cache, what).view(torch.uint8)[0, 0, key // block] = 255
    O2, L2 = bsa.cache_forward(q, cache, **kw)
    assert torch.equal(O[:, :, :apart], O2[:, :, :apart]) and torch.equal(L[:, :, :apart], L2[:, :, :apart])
    if what == "V":
        assert O2[:, :, sees:, 5].isnan().all() and torch.equal(L, L2)
        assert torch.equal(O[..., :5], O2[..., :5]) and torch.equal(O[..., 6:], O2[..., 6:])
    else:
        assert O2[:, :, sees:].isnan().all() and (what == "V_scale" or L2[:, :, sees:].isnan().all())
    assert bsa.window_status() == 0


WAYS = [("rows", 1, 12, 3, 3, 700), ("rows", 2, 6, 3, 2, 40000), ("unpacked", 2, 6, 3, 300, 700), ("tiles", 1, 6, 3, 300, 6000), ("tiles", 5, 14, 14, 64, 6000)]


def check_by_row(way, q, cache, **kw):
    assert bsa.debug_cache_way(q, cache, **kw)[0] == way
    O, L = bsa.cache_forward(q, cache, **kw)
    (kc, ks), (vc, vs) = parts(cache)
    wO, wL, tO, tL = B.forward(way, q, C.values(kc, ks, cache.block).cuda(), C.values(vc, vs, cache.block).cuda(), vs, cache.block, **kw)
    R.assert_within(L, wL, tL, "LSE")
    R.assert_within(O, wO, tO, "O")
    assert bsa.window_status() == 0


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (64, "fp16"), (128, "bf16"), (128, "fp16")])
@pytest.mark.parametrize("block", [16, 64])
@pytest.mark.parametrize("way,b,h,hk,n,nk", WAYS)
def test_quiet_rows_and_heads_beside_loud_ones(way, b, h, hk, n, nk, block, d, dtype):
    """Each key head's K and V of another size, each row of Q, blocks as different as a louder token makes them: every row within what its own numbers allow."""
    g = generator(38)
    cache = bsa.cache_create(b, hk, nk, d, block=block)
    by = lambda low, high, shape: torch.pow(2.0, torch.randint(low, high, shape, device="cuda", generator=g).float())  # noqa: E731
    k, v = (torch.empty(b, hk, nk, d, device="cuda").normal_(0, 1, generator=g) for _ in range(2))
    k *= by(-6, 2, (b, hk, 1, 1))
    v *= by(-12, 8 if dtype == "bf16" else 3, (b, hk, 1, 1)) * torch.empty(b, hk, nk, 1, device="cuda").normal_(0, 1.2, generator=g).exp_()
    bsa.cache_write(cache, k.to(DT[dtype]), v.to(DT[dtype]))
    q = (queries(38, b, h, n, d, "bf16", "hnd").float() * by(-10, 3, (b, h, n, 1))).to(DT[dtype])
    check_by_row(way, q, cache, left=-1, right=0)
    check_by_row(way, q, cache, left=nk - n - 5, right=3, sinks=20)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (64, "fp16"), (128, "bf16"), (128, "fp16")])
@pytest.mark.parametrize("block", [16, 64])
@pytest.mark.parametrize("way,b,h,hk,n,nk", WAYS)
def test_a_window_behind_a_louder_token(way, b, h, hk, n, nk, block, d, dtype):
    """The window begins inside a block whose first token, seen by nobody, is far louder than all that is seen: its scale is the largest there is."""
    g = generator(39)
    cache = bsa.cache_create(b, hk, nk, d, block=block)
    k, v = (torch.empty(b, hk, nk, d, device="cuda").normal_(0, 1, generator=g) for _ in range(2))
    left = nk - n - 2 * block - 3  # so row 0, at nk - n, sees keys from 2 block + 3 on
    k[:, :, 2 * block] *= 32
    v[:, :, 2 * block] *= 2.0 ** (20 if dtype == "bf16" else 12)
    bsa.cache_write(cache, k.to(DT[dtype]), v.to(DT[dtype]))
    check_by_row(way, queries(39, b, h, n, d, dtype, "hnd"), cache, left=left)
