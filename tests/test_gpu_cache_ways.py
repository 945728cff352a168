"""The 8-bit cache's attention way by way: what one call leaves for the next, and how far each way's roundings and NaN reach."""
import pytest
import torch

from paper_2609_25869_b200 import bsa
from tests import cache_reference as C
from tests import window_reference as R
from tests.test_gpu_cache import check_write, filled, garbage, generator, parts, queries
from tests.test_gpu_window import ints

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
