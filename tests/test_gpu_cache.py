"""The 8-bit cache through the C ABI: bytes written against the definition, values read, attention against the formulas in 64 bits, element by
element within what the roundings allow (cache_reference.py has the bounds)."""
import math

import pytest
import torch

from paper_2609_25869_b200 import bsa
from tests import cache_reference as C
from tests import window_reference as R
from tests.test_gpu_window import CASES, DT, FEW, ints

pytestmark = pytest.mark.gpu


def generator(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def garbage(seed, batch, heads, N, d, block, layout="hnd", scales=None):
    """A cache of random bytes (codes: NaN among them), scales too or one."""
    g = generator(seed)
    shape = (batch, heads, N, d) if layout == "hnd" else (batch, N, heads, d)
    K, V = (torch.randint(0, 256, shape, dtype=torch.uint8, device="cuda", generator=g).view(torch.float8_e4m3fn) for _ in range(2))
    s = (batch, heads, -(-N // block))
    S = [torch.randint(*((0, 256) if scales is None else scales), s, dtype=torch.uint8, device="cuda", generator=g).view(torch.float8_e8m0fnu) for _ in range(2)]
    return bsa.Cache(K, V, *S, block=block, layout=layout)


def parts(cache):
    """((codes, scales) of K, of V) as bytes on the CPU, heads first."""
    first = lambda x: (x if cache.layout == "hnd" else x.transpose(1, 2)).contiguous().cpu()  # noqa: E731
    return [(first(x.view(torch.uint8)), s.view(torch.uint8).cpu().contiguous()) for x, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale))]


def by_head(x, layout):
    return x if layout == "hnd" else x.transpose(1, 2)


def tokens(g, batch, heads, N, d, dtype, layout, spread=1.0):
    shape = (batch, heads, N, d) if layout == "hnd" else (batch, N, heads, d)
    x = torch.empty(shape, device="cuda").normal_(0, 1, generator=g)
    loud = torch.empty((*shape[:-1], 1), device="cuda").normal_(0, spread, generator=g).exp_()
    return (x * loud).to(DT[dtype])


def same_codes(a, b):
    """Byte by byte, any NaN for any NaN and zero for minus zero."""
    nan = ((a & 127) == 127) & ((b & 127) == 127)
    zero = ((a & 127) == 0) & ((b & 127) == 0)
    return bool(((a == b) | nan | zero).all())


def check_write(cache, K, V, start=None, count=None):
    before = parts(cache)
    bsa.cache_write(cache, K, V, start=ints(start), count=ints(count))
    torch.cuda.synchronize()
    for (codes, scales), (c0, s0), x in zip(parts(cache), before, (K, V)):
        want_c, want_s = C.write(by_head(x, cache.layout).cpu(), c0, s0, cache.block, start, count)
        assert torch.equal(scales, want_s)
        assert same_codes(codes, want_c)
        untouched = want_c == c0
        assert torch.equal(codes[untouched] & 127, c0[untouched] & 127)


#        b  h  N    cap   starts            counts
WRITES = [
    (1, 1, 1, 1, None, None),
    (1, 2, 128, 128, None, None),
    (2, 3, 1, 300, [17, 299], None),                   # one token inside a block, the cache's last
    (3, 2, 77, 200, [0, 100, 190], [77, 40, 77]),      # a count below the rows; the last runs over the cache's end
    (2, 1, 40, 90, [-13, -40], None),                  # rows in front of the cache; all of them
    (4, 1, 5, 64, [60, 64, 1000, 3], [4, 5, 5, 0]),    # behind the cache; nothing
    (2, 2, 300, 513, [1, 128], [300, -7]),
    (1, 4, 9, 50, [2 ** 31 - 1], None),
    (1, 1, 9, 50, [-2 ** 31], [2 ** 31 - 1]),
]


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("d,dtype", [(64, "fp16"), (128, "bf16"), (64, "bf16"), (128, "fp16")])
@pytest.mark.parametrize("block", [16, 32, 64, 128])
def test_written_bytes(block, d, dtype, layout):
    for i, (b, h, n, cap, start, count) in enumerate(WRITES):
        g = generator(100 * block + d + i)
        cache = garbage(i, b, h, cap, d, block, layout, scales=(110, 140))
        check_write(cache, tokens(g, b, h, n, d, dtype, layout), tokens(g, b, h, n, d, dtype, layout, 3.0), start, count)


@pytest.mark.parametrize("block,d", [(16, 128), (64, 64), (128, 128)])
def test_token_by_token(block, d):
    """Scales that grow under what is there: the bytes after every token are the definition's."""
    g = generator(5)
    cache = bsa.cache_create(2, 2, 150, d, block=block)
    for i in range(0, 140, 1):
        loud = 2.0 ** ((i * 7) % 23 - 11)
        check_write(cache, tokens(g, 2, 2, 1, d, "bf16", "hnd") * loud, tokens(g, 2, 2, 1, d, "bf16", "hnd") / loud, [i, i + 3], None)


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
def test_extremes_written(dtype):
    """Zeros, the type's largest and smallest values, infinities and NaN, scales that were NaN or differ by all there is."""
    g = generator(6)
    fin = torch.finfo(DT[dtype])
    x = tokens(g, 1, 1, 128, 64, dtype, "hnd")
    x[0, 0, :16] = 0
    x[0, 0, 16:32] = fin.smallest_normal * 0.25
    x[0, 0, 32, 5], x[0, 0, 33, 6] = fin.max, -fin.max
    x[0, 0, 48, 0], x[0, 0, 49, 1], x[0, 0, 50, 2] = math.inf, -math.inf, math.nan
    x[0, 0, 64:80] = math.nan
    x[0, 0, 80:96] *= fin.smallest_normal
    x[0, 0, 96, 0] = 448.0
    x[0, 0, 97] = x[0, 0, 97].clamp(-1, 1)
    x[0, 0, 112:] = 2.0 ** torch.arange(-8, 8, device="cuda").view(16, 1).double().to(x.dtype)
    for scales in ((0, 1), (255, 256), (247, 255), (100, 140)):
        for start in (0, 7):
            cache = garbage(7, 1, 1, 160, 64, 16, scales=scales)
            check_write(cache, x, x.flip(2).contiguous(), [start], None)


def test_memory_around_is_left_alone():
    """A cache that is a view of a longer one with more heads, scales of more blocks: every byte outside stays."""
    g = generator(8)
    big = torch.randint(0, 256, (2, 3, 6, 300, 128), dtype=torch.uint8, device="cuda", generator=g)
    sc = torch.randint(0, 256, (2, 3, 6, 40), dtype=torch.uint8, device="cuda", generator=g)
    b0, s0 = big.clone(), sc.clone()
    K, V = (big[i, 1:, 1:5, 32:232].view(torch.float8_e4m3fn) for i in range(2))
    Ks, Vs = (sc[i, 1:, 1:5, 3:16].view(torch.float8_e8m0fnu) for i in range(2))
    cache = bsa.Cache(K, V, Ks, Vs, block=16)
    x, y = (tokens(g, 2, 4, 60, 128, "bf16", "nhd") for _ in range(2))
    wide = torch.zeros(2, 60, 3 * 4 * 128, dtype=torch.bfloat16, device="cuda")  # as a fused projection leaves them
    wide[..., 512:1024], wide[..., 1024:] = x.flatten(2), y.flatten(2)
    k, v = (wide[..., i * 512:(i + 1) * 512].unflatten(-1, (4, 128)).transpose(1, 2) for i in (1, 2))
    check_write(cache, k, v, [150, 21], [60, 44])
    for t in (big, sc):  # what lies inside is checked above
        t0 = b0 if t is big else s0
        inside = torch.zeros(t.shape, dtype=torch.bool, device="cuda")
        inside[:, 1:, 1:5, slice(32, 232) if t is big else slice(3, 16)] = True
        assert torch.equal(t[~inside], t0[~inside])


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
def test_read(d, dtype, layout):
    """Exact, zero outside, the type's largest number beyond its range."""
    for i, (b, h, n, cap, start, count) in enumerate(WRITES):
        block = (16, 32, 64, 128)[i % 4]
        cache = garbage(i + 20, b, h, cap, d, block, layout, scales=(80, 160) if dtype == "bf16" else (112, 140))
        for t, (codes, scales), (want_t) in zip(bsa.cache_read(cache, n, start=ints(start), count=ints(count), dtype=DT[dtype]), parts(cache), "KV"):
            want = C.read(codes, scales, block, n, start, count)
            top = torch.finfo(DT[dtype]).max
            want = want.clamp(-top, top).to(DT[dtype])
            got = by_head(t, layout).cpu()
            assert torch.equal(got.isnan(), want.isnan()) and torch.equal(got.nan_to_num(0.0), want.nan_to_num(0.0)), want_t


def test_read_into_views_and_scales_at_their_ends():
    cache = garbage(30, 1, 2, 64, 64, 16)
    cache.K_scale.view(torch.uint8)[0, 0] = torch.tensor([0, 255, 254, 1], dtype=torch.uint8)
    out = torch.full((2, 80, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    K, V = out[:1, :70].transpose(1, 2), out[1:, :70].transpose(1, 2)
    bsa.cache_read(cache, 70, K=K, V=V)
    for t, (codes, scales) in zip((K, V), parts(cache)):
        top = torch.finfo(torch.bfloat16).max
        want = C.read(codes, scales, 16, 70, None, None).clamp(-top, top).to(torch.bfloat16)
        assert torch.equal(t.cpu().isnan(), want.isnan()) and torch.equal(t.cpu().nan_to_num(0.0), want.nan_to_num(0.0))
    assert (out[:, 70:] == 7).all()


# ------------------------------------------------------------------ attention
def filled(seed, batch, heads, N, d, dtype, layout, block, spread=0.3):
    """A cache of normal tokens and its values in 64 bits, laid out as the cache (batch always there)."""
    g = generator(seed)
    cache = bsa.cache_create(batch, heads, N, d, block=block, layout=layout)
    bsa.cache_write(cache, *(tokens(g, batch, heads, N, d, dtype, layout, spread) for _ in range(2)))
    return cache, [by_head(C.values(c, s, block).cuda(), layout) for c, s in parts(cache)]


def without_batch(cache):
    return bsa.Cache(cache.K[0], cache.V[0], cache.K_scale[0], cache.V_scale[0], block=cache.block, layout=cache.layout)


def check_forward(q, cache, values, **kw):
    O, L = bsa.cache_forward(q, cache, **kw)
    torch.cuda.synchronize()
    assert bsa.window_status() == 0
    wO, wL, tO, tL = C.forward(q, *values, layout=cache.layout, **kw)
    R.assert_within(L, wL, tL, "LSE")
    R.assert_within(O, wO, tO, "O")
    return O, L


def queries(seed, b, h, n, d, dtype, layout):
    s = (b, h, n, d) if layout == "hnd" else (b, n, h, d)
    return torch.empty(s if b else s[1:], device="cuda").normal_(0, 1, generator=generator(seed + 99)).to(DT[dtype])


# Few row tiles over long windows: the kernel that reads the codes, keys cut into parts
#       b  h  hk   n    nk   left right sinks  starts           lengths
LONG = [
    (1, 2, 1, 300, 6000, -1, 0, 0, None, None),
    (0, 2, 2, 513, 3333, -1, 10, 0, None, None),
    (2, 2, 2, 257, 5000, -1, -1, 0, [0, -100], [5000, 3000]),                # rows in front of the sequence
    (1, 4, 2, 600, 9000, 6000, 100, 200, None, None),                        # a window, its ends inside tiles, first tokens
    (2, 3, 1, 400, 4000, 3500, 0, 7, [3600, 100], [4000, 450]),              # rows behind the sequence; parts without a tile
    (3, 2, 1, 270, 7000, -1, 0, 40, [6730, 30, 0], [7000, 300, 0]),          # a short sequence, one without a key
    (1, 1, 1, 1000, 4096, -1, 63, 0, None, None),
    (2, 8, 2, 65, 20000, 15000, 0, 1, [19000, 19935], [19065, 20000]),       # 260 rows per key head
    (1, 3, 3, 290, 30000, 4000, 500, 129, [25000], [25100]),                 # most rows at no position
]


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (64, "fp16"), (128, "bf16"), (128, "fp16")])
@pytest.mark.parametrize("case", CASES + FEW + LONG, ids=lambda c: "x".join(str(x) for x in c[:8]))
def test_forward(case, d, dtype, layout):
    """The windowed kernels' own cases, tiles and few rows, and long windows of few tiles, over caches of every block size."""
    b, h, hk, n, nk, left, right, sinks, starts, lengths = case
    block = (16, 32, 64, 128)[(n + nk + d // 64 + (layout == "nhd")) % 4]
    cache, values = filled(sum(case[1:5]) + d, max(b, 1), hk, nk, d, dtype, layout, block)
    if not b:
        cache, values = without_batch(cache), [x[0] for x in values]
    q = queries(n + nk, b, h, n, d, dtype, layout)
    check_forward(q, cache, values, left=left, right=right, sinks=sinks, q_start=ints(starts), kv_len=ints(lengths))


@pytest.mark.parametrize("block", [16, 64])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,nk,left", [(1, 1000, 150), (3, 1000, 150), (200, 1000, 150), (200, 9000, 5150)])
def test_what_no_row_sees_may_hold_anything(n, nk, left, d, block):
    """Behind the length, in front of the window, between the sinks and the window: codes of NaN and scales of any byte there change no bit."""
    cache, values = filled(11, 2, 2, nk, d, "bf16", "hnd", block)
    q = queries(3, 2, 4, n, d, "bf16", "hnd")
    starts, lengths = [nk - 400, 130], [nk - 400 + n, 130 + n]
    kw = dict(left=left, right=0, sinks=7, q_start=ints(starts), kv_len=ints(lengths))
    O, L = check_forward(q, cache, values, **kw)
    for b in range(2):
        for lo, hi in ((lengths[b], nk), (7, starts[b] - left)):
            if lo >= hi:
                continue
            for t, s in ((cache.K, cache.K_scale), (cache.V, cache.V_scale)):
                t.view(torch.uint8)[b, :, lo:hi, ::2] = 127
                t.view(torch.uint8)[b, :, lo:hi, 1::2] = 255
                a, z = -(-lo // block), hi // block if hi < nk else s.shape[-1]
                s.view(torch.uint8)[b, :, a:z:3], s.view(torch.uint8)[b, :, a + 1:z:3], s.view(torch.uint8)[b, :, a + 2:z:3] = 255, 0, 254
    O2, L2 = bsa.cache_forward(q, cache, **kw)
    assert torch.equal(O, O2) and torch.equal(L, L2)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,nk", [(2, 700), (300, 700), (300, 6000)])
@pytest.mark.parametrize("what", ["K", "V", "K_scale", "V_scale", "Q"])
def test_a_nan_that_a_row_sees_reaches_its_outputs(what, n, nk, d):
    cache, values = filled(13, 1, 1, nk, d, "bf16", "hnd", 32)
    q = queries(4, 1, 2, n, d, "bf16", "hnd")
    kw = dict(left=-1, right=-1, q_start=ints([100]))
    clean = check_forward(q, cache, values, **kw)
    if what == "Q":
        q[0, 1, n - 1, 3] = math.nan
    elif what in ("K", "V"):
        getattr(cache, what).view(torch.uint8)[0, 0, 333, 5] = 127
    else:
        getattr(cache, what).view(torch.uint8)[0, 0, 9] = 255
    O, L = bsa.cache_forward(q, cache, **kw)
    if what == "Q":
        assert O[0, 1, n - 1].isnan().all() and L[0, 1, n - 1].isnan()
        assert torch.equal(O[0, 0], clean[0][0, 0]) and torch.equal(L[0, 0], clean[1][0, 0])
    elif what == "V":
        assert O[..., 5].isnan().all() and not O[..., :5].isnan().any() and torch.equal(L, clean[1])
    else:
        assert O.isnan().all() and (what == "V_scale" or L.isnan().all())
    assert bsa.window_status() == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,nk,block", [(1, 900, 16), (260, 900, 16), (260, 6000, 16), (260, 6000, 64)])
def test_blocks_of_very_different_size(n, nk, block, d, dtype):
    """Scales from 2^-20 to 2^6 side by side, and queries whose elements differ as much."""
    g = generator(14)
    cache = bsa.cache_create(1, 2, nk, d, block=block)
    e = torch.randint(-20, 7 if dtype == "bf16" else 4, (1, 2, -(-nk // block)), generator=g, device="cuda")
    f = torch.pow(2.0, e.float()).repeat_interleave(block, 2)[:, :, :nk, None]
    K, V = (tokens(g, 1, 2, nk, d, "bf16", "hnd", 0.1) for _ in range(2))
    bsa.cache_write(cache, (K * f * 0.05).to(DT[dtype]), (V * f).to(DT[dtype]))
    values = [C.values(c, s, block).cuda() for c, s in parts(cache)]
    q = queries(5, 1, 4, n, d, dtype, "hnd")
    q[..., ::3] *= 2.0 ** -12
    check_forward(q, cache, values, left=-1, right=-1, q_start=ints([200]), kv_len=ints([nk - 10]))
    check_forward(q, cache, values, left=nk - 860, right=3, sinks=5, q_start=ints([nk - 300]), kv_len=ints([nk - 10]))


@pytest.mark.parametrize("n,nk", [(1, 500), (300, 500), (300, 5000)])
def test_large_and_small_queries(n, nk):
    """Rows of bf16 up to its largest numbers and down to its smallest; a row of zeros sees its keys evenly."""
    cache, values = filled(15, 1, 1, nk, 128, "bf16", "hnd", 64)
    q = queries(6, 1, 1, n, 128, "bf16", "hnd")
    kw = dict(left=-1, right=-1, q_start=ints([0]))
    for f, scale in ((2.0 ** 100, 2.0 ** -104), (2.0 ** -110, 2.0 ** 106), (0.0, 0.0)):
        check_forward((q.float() * f).bfloat16(), cache, values, scale=scale, **kw)


@pytest.mark.parametrize("n,left", [(1, 300), (200, 300), (200, -1)])
def test_views(n, left):
    """Q out of a fused projection, O into one, a cache that is a stretch of a longer one, no batch; LSE given."""
    g = generator(16)
    end = 896 if left > 0 else 9056
    big = bsa.cache_create(3, 4, end + 128, 128, block=32)
    bsa.cache_write(big, *(tokens(g, 3, 4, end + 128, 128, "bf16", "hnd") for _ in range(2)))
    cache = bsa.Cache(big.K[1:, 1:3, 96:end], big.V[1:, 1:3, 96:end], big.K_scale[1:, 1:3, 3:end // 32], big.V_scale[1:, 1:3, 3:end // 32], block=32)
    values = [C.values(c, s, 32)[1:, 1:3, 96:end].cuda() for c, s in parts(big)]
    wide = torch.empty(2, n, 3, 4, 128, device="cuda", dtype=torch.bfloat16).normal_(0, 1, generator=g)
    q = wide[:, :, 1].transpose(1, 2)
    kw = dict(left=left, right=0, sinks=10, q_start=ints([500, 20]), kv_len=ints([700, 600]))
    O, L = check_forward(q, cache, values, **kw)
    out = torch.zeros_like(wide)
    lse = torch.empty_like(L)
    O2, L2 = bsa.cache_forward(q, cache, O=out[:, :, 2].transpose(1, 2), LSE=lse, **kw)
    assert L2 is lse and torch.equal(L, lse) and torch.equal(O, O2) and not out[:, :, :2].any()
    bsa.cache_forward(q, cache, O=q, LSE=lse, **kw)  # in the place of Q
    assert torch.equal(O, q)


def test_tokens_of_a_stream():
    """As a model runs them: rotate, write, attend, token by token and by the chunk; against attention over what is read back."""
    g = generator(17)
    b, h, hk, d, n = 2, 8, 2, 128, 200
    cache = bsa.cache_create(b, hk, 300, d, block=32)
    kw = dict(left=63, right=0, sinks=4)
    x = [torch.empty(b, m, n, d, device="cuda", dtype=torch.bfloat16).normal_(0, 1, generator=g) for m in (h, hk, hk)]
    at = 0
    for step in (130, 1, 1, 7, 1, 40, 1, 19):
        q, k, v = (t[:, :, at:at + step] for t in x)
        pos = (at + torch.arange(step, device="cuda", dtype=torch.int32)).view(-1, 1)
        q, k = bsa.rope(q, k, axes=[d], positions=pos)
        start, length = ints([at] * b), ints([at + step] * b)
        bsa.cache_write(cache, k, v, start=start)
        O, L = bsa.cache_forward(q, cache, q_start=start, kv_len=length, **kw)
        K, V = bsa.cache_read(cache, 300)
        wO, wL, tO, tL = C.forward(q, K.double(), V.double(), q_start=start, kv_len=length, **kw)
        R.assert_within(O, wO, tO, "O")
        R.assert_within(L, wL, tL, "LSE")
        O16, L16 = bsa.window_forward(q, K, V, q_start=start, kv_len=length, **kw)
        R.assert_within(O16, wO, tO, "O of the 16-bit cache")
        at += step
    assert at == n and bsa.window_status() == 0


def test_a_plan_over_what_is_read():
    """The block-sparse forward takes a cache's window in 16 bits."""
    g = generator(18)
    cache, _ = filled(18, 1, 2, 512, 64, "bf16", "hnd", 64)
    K, V = bsa.cache_read(cache, 256, start=ints([128]))
    q = torch.empty(2, 256, 64, device="cuda", dtype=torch.bfloat16).normal_(0, 1, generator=g)
    with bsa.plan_create(torch.ones(2, 4, 4, dtype=torch.uint8, device="cuda"), 64, 64, 256, 2, 64) as plan:
        O, L = plan.forward(q, K[0], V[0])
    wO, wL, tO, tL = R.forward(q, K[0], V[0], left=-1, right=-1, u=R.HALF_STEP[q.dtype])
    R.assert_within(O, wO, tO, "O")


@pytest.mark.parametrize("n,left", [(1, 200), (300, 200), (300, -1)])
def test_captured_and_replayed(n, left):
    """A step in a graph follows the positions in device memory; two graphs and an eager call side by side."""
    g = generator(19)
    b, h, hk, d = 2, 4, 2, 64
    cap = 1000 if left > 0 else 9000  # (the sizes decide which way rows by the tile go)
    caches = [bsa.cache_create(b, hk, cap, d, block=16) for _ in range(3)]
    x = [torch.empty(b, m, 900, d, device="cuda", dtype=torch.float16).normal_(0, 1, generator=g) for m in (h, hk, hk)]
    kw = dict(left=left, right=0, sinks=3)
    start, length = ints([0, 0]), ints([n, n])
    ins = [t[:, :, :n].contiguous() for t in x]

    def step(cache, st=None, le=None):
        bsa.cache_write(cache, ins[1], ins[2], start=start if st is None else st)
        return (*bsa.cache_forward(ins[0], cache, q_start=start if st is None else st, kv_len=length if le is None else le, **kw),
                *bsa.cache_read(cache, 50, start=start if st is None else st, dtype=torch.float16))
    step(caches[2])  # first calls of the process outside of a capture
    graphs, outs = [], []
    for i in range(2):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            outs.append(step(caches[i]))
        graphs.append(graph)
    caches[2] = bsa.cache_create(b, hk, cap, d, block=16)
    for c in caches[:2]:
        c.K_scale.view(torch.uint8).zero_()
    side = torch.cuda.Stream()
    for i in range(3):
        at = i * n
        start.fill_(at)
        length.fill_(at + n)
        for t, src in zip(ins, x):
            t.copy_(src[:, :, at:at + n])
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            graphs[1].replay()
        graphs[0].replay()
        want = step(caches[2])
        torch.cuda.synchronize()
        for got in outs:
            assert all(torch.equal(a, w) for a, w in zip(got, want))
    assert bsa.window_status() == 0


@pytest.mark.parametrize("n,nk", [(1, 600), (300, 600), (300, 6000)])
def test_other_streams(n, nk):
    """stream=: a torch stream or a handle, with the default stream busy; outputs come from that stream's pool."""
    cache, values = filled(20, 1, 2, nk, 128, "bf16", "hnd", 64)
    q = queries(7, 1, 4, n, 128, "bf16", "hnd")
    kw = dict(left=-1, right=0, sinks=0, q_start=ints([nk - 350]), kv_len=ints([nk - 350 + n]))
    O, L = check_forward(q, cache, values, **kw)
    K, V = bsa.cache_read(cache, nk)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    torch.cuda._sleep(20_000_000)
    other = bsa.cache_create(1, 2, nk, 128, device="cuda")
    side.wait_stream(torch.cuda.current_stream())
    for s in (side, side.cuda_stream):
        O2, L2 = bsa.cache_forward(q, cache, stream=s, **kw)
        bsa.cache_write(other, K, V, stream=s)
        K2, V2 = bsa.cache_read(other, nk, stream=s)
    side.synchronize()
    assert torch.equal(O, O2) and torch.equal(L, L2) and torch.equal(K, K2) and torch.equal(V, V2)


class withheld_tiles:
    """First tiles never arrive, and a wait lasts about 10 ms of SM clocks."""

    def __enter__(self):
        bsa.debug_set_wait_limit(20_000_000)
        bsa.debug_withhold_arrival(True)

    def __exit__(self, *exc):
        bsa.debug_withhold_arrival(False)
        bsa.debug_set_wait_limit(0)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n,nk,left", [(1, 100, -1), (2, 5000, -1), (300, 300, -1), (700, 700, 200), (300, 40000, -1)])
def test_a_wait_that_runs_out_ends_in_a_status_not_a_hang(n, nk, left, d):
    cache, values = filled(21, 1, 2, nk, d, "bf16", "hnd", 64)
    q = queries(8, 1, 4, n, d, "bf16", "hnd")
    kw = dict(left=left, right=0, sinks=2)
    O, L = bsa.cache_forward(q, cache, **kw)
    assert bsa.window_status() == 0
    with withheld_tiles():
        bsa.cache_forward(q, cache, **kw)
        assert bsa.window_status() == 6 and bsa.window_status() == 0
    O2, L2 = bsa.cache_forward(q, cache, **kw)
    assert bsa.window_status() == 0 and torch.equal(O, O2) and torch.equal(L, L2)


def test_offsets_beyond_32_bits():
    """Codes, rows and outputs that lie more than 4 GB from their tensor's beginning."""
    g = generator(22)
    hk, cap, d = 36, 1_000_000, 128
    K, V = (torch.empty(1, hk, cap, d, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for _ in range(2))
    s = [torch.empty(1, hk, cap // 16, dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu) for _ in range(2)]
    cache = bsa.Cache(K, V, *s, block=16)
    start = cap - 80  # the beginning of a block
    k, v = (tokens(g, 1, hk, 60, d, "bf16", "hnd") for _ in range(2))
    bsa.cache_write(cache, k, v, start=ints([start]))
    small = bsa.cache_create(1, hk, 80, d, block=16)
    bsa.cache_write(small, k, v)
    for a, b in zip(bsa.cache_read(cache, 60, start=ints([start])), bsa.cache_read(small, 60)):
        assert torch.equal(a, b)
    for n in (1, 40):
        q = queries(9, 1, hk * 4, n, d, "bf16", "hnd")
        kw = dict(left=30 - n // 2, right=0)
        O, L = bsa.cache_forward(q, cache, q_start=ints([start + 60 - n]), kv_len=ints([start + 60]), **kw)
        O2, L2 = bsa.cache_forward(q, small, q_start=ints([60 - n]), kv_len=ints([60]), **kw)
        assert (O.float() - O2.float()).abs().max() <= 4 * 2.0 ** -8 * O2.float().abs().max() and (L - L2).abs().max() <= 1e-4
    assert bsa.window_status() == 0


def test_the_same_bits_every_time():
    cache, _ = filled(23, 2, 4, 5000, 128, "bf16", "nhd", 64)
    for n in (1, 5, 400):
        q = queries(10, 2, 8, n, 128, "bf16", "nhd")
        a = bsa.cache_forward(q, cache, left=-1)
        for _ in range(3):
            b = bsa.cache_forward(q, cache, left=-1)
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_the_binding_refuses_what_does_not_fit():
    cache, _ = filled(24, 2, 2, 100, 64, "bf16", "hnd", 64)
    x = torch.zeros(2, 2, 10, 64, dtype=torch.bfloat16, device="cuda")
    for bad in (x[:1], x[:, :1], x[..., :32], x.float(), x[0], x.cpu(), x.transpose(2, 3)):
        with pytest.raises((ValueError, bsa.BsaError)):
            bsa.cache_write(cache, bad, bad)
        with pytest.raises((ValueError, bsa.BsaError)):
            bsa.cache_read(cache, 10, K=bad, V=bad)
    for bad in (x[:1], x[..., :32], x.float(), x[0], x.cpu(), x.repeat(1, 2, 1, 1)[:, :3]):
        with pytest.raises((ValueError, bsa.BsaError)):
            bsa.cache_forward(bad, cache, left=1)
    with pytest.raises(ValueError):
        bsa.cache_write(cache, x, x, start=torch.zeros(2, dtype=torch.int64, device="cuda"))
    with pytest.raises(ValueError):
        bsa.cache_read(cache, 10, K=x)
    with pytest.raises(ValueError):
        bsa.cache_read(cache, 11, K=x, V=x.clone())
    with pytest.raises(ValueError):
        bsa.cache_forward(x, cache, left=1, O=x[:, :, :5])
    with pytest.raises(ValueError):
        bsa.Cache(cache.K, cache.V, cache.K_scale, cache.V_scale, block=48)
    with pytest.raises(ValueError):
        bsa.Cache(cache.K, cache.V, cache.K_scale, cache.V_scale, block=16)
    with pytest.raises(ValueError):
        bsa.Cache(cache.K, cache.V[:1], cache.K_scale, cache.V_scale)
    with pytest.raises(ValueError):
        bsa.Cache(cache.K, cache.V, cache.K_scale, cache.V_scale.view(torch.uint8))


def test_first_calls_in_a_captured_graph():
    """Nothing that a first call sets up (attributes, addresses, module loading) is refused while a stream is being captured."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2609_25869_b200 import bsa
cache = bsa.cache_create(1, 2, 6000, 64, block=16)
x = [torch.randn(1, h, 6000, 64, device='cuda').bfloat16() for h in (4, 2, 2)]
calls = [(1, -1), (300, 200), (300, -1), (3, -1)]
def run():
    out = []
    bsa.cache_write(cache, x[1], x[2])
    for n, left in calls:
        out += bsa.cache_forward(x[0][:, :, -n:], cache, left=left, sinks=2)
    return out + list(bsa.cache_read(cache, 100))
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    got = run()
g.replay()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(got, run())) and bsa.window_status() == 0
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("n,nk,left", [(300, 700, 100), (300, 6000, -1), (1, 40000, -1)])
def test_workspaces(n, nk, left):
    """Too small, misaligned or missing ones are refused; calls that overlap bring their own, and bytes behind one stay."""
    cache, _ = filled(25, 1, 2, nk, 64, "bf16", "hnd", 64)
    q = queries(11, 1, 4, n, 64, "bf16", "hnd")
    O, L = bsa.cache_forward(q, cache, left=left)
    lib = bsa.lib()
    desc = bsa._WINDOW.pack(1, 4, 2, 64, n, nk, left, 0, 0, 0, 0.0, 0, 0)
    need = lib.bsa_cache_workspace_bytes(desc, cache._packed)
    assert need > 0
    vq = bsa._view(q, False, q.dtype, 0, "Q")[4]
    O2, L2 = torch.empty_like(O), torch.empty_like(L)
    vo = bsa._view(O2, False, q.dtype, 0, "O")[4]
    ws = torch.full((need + 1024,), 77, dtype=torch.uint8, device="cuda")
    for at, size in ((None, need), (ws.data_ptr(), need - 1), (ws.data_ptr() + 16, need), (ws.data_ptr(), 0)):
        assert lib.bsa_cache_forward(desc, cache._packed, vq, vo, L2.data_ptr(), at, size, None) == 1
    assert lib.bsa_cache_forward(desc, cache._packed, vq, vo, L2.data_ptr(), ws.data_ptr(), need, torch.cuda.current_stream().cuda_stream or None) == 0
    torch.cuda.synchronize()
    assert torch.equal(O, O2) and torch.equal(L, L2) and (ws[need:] == 77).all()


def test_two_calls_at_once():
    """Reads, writes of another cache and attention of all three kinds on four streams at once, again and again."""
    caches = [filled(26 + i, 1, 2, nk, 64, "bf16", "hnd", 64)[0] for i, nk in enumerate((40000, 700, 6000))]
    qs = [queries(12 + i, 1, 4, n, 64, "bf16", "hnd") for i, n in enumerate((1, 300, 300))]
    calls = [lambda i=i: bsa.cache_forward(qs[i], caches[i], left=100 if i == 1 else -1) for i in range(3)]
    want = [c() for c in calls]
    K, V = bsa.cache_read(caches[2], 6000)
    other = bsa.cache_create(1, 2, 6000, 64)

    def copy():
        bsa.cache_write(other, K, V)
        return bsa.cache_read(other, 6000)
    calls.append(copy)
    want.append((K, V))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in calls]
    for _ in range(5):
        got = []
        for s, c in zip(streams, calls):
            with torch.cuda.stream(s):
                got.append(c())
        torch.cuda.synchronize()
        for a, b in zip(got, want):
            assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
    assert bsa.window_status() == 0
