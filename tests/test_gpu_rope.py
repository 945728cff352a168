"""Rotary positions through the C ABI against the formula in 64 bits.

A product's and the sum's fp32 roundings, the fixed-point angle (2^-31 half turns, then 2^-24 of it in fp32: 2e-7 rad) and the sine and
cosine (2 ulp) leave an element off by less than 2^-20 of the absolute values that it is made of; rounding it adds half a step: half a unit of
relative precision, but never less than 2^-25 in half, whose steps stop shrinking at 2^-24 (an element below 2^-14 made of two small ones
shows it: with 2^-11 of the element alone one in some million was 1.2 times the bound)."""
import pytest
import torch

from paper_2609_25869_b200 import bsa
from tests import window_reference as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}
LEAST = {torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}


def make(seed, shape, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return torch.empty(shape, device="cuda", dtype=DT[dtype]).normal_(0, 1, generator=g)


def shape_of(layout, b, h, n, d):
    s = (b, h, n, d) if layout == "hnd" else (b, n, h, d)
    return s if b else s[1:]


def check(got, x, angle, turns, **kw):
    want, made = R.rotate(x, angle, turns, **kw)
    R.assert_within(got, want, R.HALF_STEP[x.dtype] * want.abs() * 1.01 + 2.0 ** -20 * made + LEAST[x.dtype], "rotation")


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("pairs", ["interleaved", "halves"])
@pytest.mark.parametrize("axes,d", [((64,), 64), ((44, 42, 42), 128), ((16, 20, 20), 64), ((8, 12), 32), ((2, 6, 4, 0), 72), ((100,), 256), ((128, 128), 256),
                                    ((6,), 8)])
@pytest.mark.parametrize("inverse", [False, True])
def test_given_positions(dtype, layout, pairs, axes, d, inverse):
    b, h, hk, n = 2, 3, 1, 37
    q, k = make(1, shape_of(layout, b, h, n, d), dtype), make(2, shape_of(layout, b, hk, n, d), dtype)
    pos = torch.randint(-50, 3000, (b, n, len(axes)), dtype=torch.int32, device="cuda")
    shared = len(axes) == 3
    got = bsa.rope(q, k, axes=axes, positions=pos, pairs=pairs, shared_freq=shared, inverse=inverse, layout=layout, theta=500.0)
    a, t = R.angles(n, axes, positions=pos, shared_freq=shared, theta=500.0, device="cuda")
    for y, x in zip(got, (q, k)):
        check(y, x, a, t, pairs=pairs, inverse=inverse, layout=layout)


@pytest.mark.parametrize("n,first,grid,origin", [(24, 0, (2, 3, 4), None), (300, 77, (3, 5, 14), (1000, 0, -7)), (1, 0, (1, 1, 1), (5, 6, 7)), (2, 1, (1, 1, 1), None)])
@pytest.mark.parametrize("batch", [0, 1, 3])
def test_grid(n, first, grid, origin, batch):
    q, k = make(3, shape_of("nhd", batch, 5, n, 128), "bf16"), make(4, shape_of("nhd", batch, 5, n, 128), "bf16")
    got = bsa.rope(q, k, axes=(44, 42, 42), grid=grid, first=first, origin=origin, layout="nhd")
    a, t = R.angles(n, (44, 42, 42), grid=grid, first=first, origin=origin, device="cuda")
    for y, x in zip(got, (q, k)):
        check(y, x, a, t, layout="nhd")
    alone = bsa.rope(q, axes=(44, 42, 42), grid=grid, first=first, origin=origin, layout="nhd")
    assert torch.equal(alone, got[0])


@pytest.mark.parametrize("pairs", ["interleaved", "halves"])
def test_tokens_off_the_grid_and_unrotated_channels_keep_their_bits(pairs):
    x = make(5, (2, 40, 64), "bf16")
    x[0, 3, 5], x[1, 39, 9], x[0, 20, 60] = float("nan"), float("inf"), float("-inf")
    y = bsa.rope(x, axes=(8, 24, 24), grid=(1, 5, 6), first=5, pairs=pairs)
    bits = lambda v: v.contiguous().view(torch.int16)  # noqa: E731
    assert torch.equal(bits(y[:, :5]), bits(x[:, :5])) and torch.equal(bits(y[:, 35:]), bits(x[:, 35:]))
    assert torch.equal(bits(y[:, :, 56:]), bits(x[:, :, 56:]))
    assert not torch.equal(y[:, 6:35, :56], x[:, 6:35, :56])


@pytest.mark.parametrize("far", [10 ** 6, 2 ** 24 + 1, 2 ** 31 - 200, -(2 ** 31) + 3])
def test_far_positions(far):
    q = make(6, (2, 64, 128), "fp16")
    pos = (torch.arange(64, device="cuda") + far).clamp(max=2 ** 31 - 1).to(torch.int32).view(64, 1)
    y = bsa.rope(q, axes=(128,), positions=pos)
    a, t = R.angles(64, (128,), positions=pos, device="cuda")
    # (the reference's own angle: a position below 2^31 times a frequency with 2^-53 of itself wrong, 2.4e-7 rad, and its reduction as much)
    want, made = R.rotate(q, a, t)
    R.assert_within(y, want, 2.0 ** -11 * want.abs() * 1.01 + (2.0 ** -20 + 5e-7) * made + LEAST[q.dtype], "far rotation")


def test_own_frequencies_and_the_way_back():
    x = make(7, (3, 50, 64), "fp16")
    freq = [0.9 ** i * 3.0 for i in range(20)]
    pos = torch.randint(0, 500, (50, 2), dtype=torch.int32, device="cuda")
    y = bsa.rope(x, axes=(24, 16), positions=pos, freq=freq)
    a, t = R.angles(50, (24, 16), positions=pos, freq=freq, device="cuda")
    check(y, x, a, t)
    z = bsa.rope(y, axes=(24, 16), positions=pos, freq=freq, inverse=True)
    # two roundings of values of up to sqrt(2) max(|a|, |b|), turned once
    assert (z.double() - x.double()).abs().max() <= 3 * 2.0 ** -11 * x.double().abs().max()


@pytest.mark.parametrize("pairs,axes", [("interleaved", (44, 42, 42)), ("halves", (64, 64)), ("halves", (10, 10, 10))])
def test_in_place_views_and_caches(pairs, axes):
    qkv = make(8, (2, 33, 3, 4, 128), "bf16")  # a fused projection: [batch, tokens, q/k/v, heads, d]
    q, k, v = qkv.unbind(2)
    pos = torch.randint(0, 200, (33, len(axes)), dtype=torch.int32, device="cuda")
    want_q, want_k = bsa.rope(q.contiguous(), k.contiguous(), axes=axes, positions=pos, pairs=pairs, layout="nhd")
    keep = qkv.clone()
    cache = torch.full((2, 4, 100, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    bsa.rope(q, k, axes=axes, positions=pos, pairs=pairs, layout="nhd", out=(q, cache[:, :, 20:53].transpose(1, 2)))
    assert torch.equal(q, want_q) and torch.equal(cache[:, :, 20:53].transpose(1, 2), want_k)
    assert torch.equal(qkv[:, :, 1:], keep[:, :, 1:])
    assert (cache[:, :, :20] == 7).all() and (cache[:, :, 53:] == 7).all()


def test_beyond_32_bits_of_elements():
    n, h, d = 2 ** 16 + 3, 257, 128  # 2.16e9 elements
    x = torch.zeros((n, h, d), dtype=torch.bfloat16, device="cuda")
    x[-1, -1], x[0, 0] = 1.0, 1.0
    pos = torch.arange(n, dtype=torch.int32, device="cuda").view(n, 1)
    y = bsa.rope(x, axes=(128,), positions=pos, layout="nhd", out=x)
    a, t = R.angles(n, (128,), positions=pos, device="cuda")
    for i in (0, n - 1):
        one = torch.ones(1, 1, 1, 128, dtype=torch.bfloat16, device="cuda")
        check(y[i:i + 1, h - 1 if i else 0].view(1, 1, 1, 128), one, a[:, i:i + 1], t[i:i + 1])
    assert not y[5].any()


def test_streams_graphs_and_refusals():
    x = make(9, (4, 100, 128), "bf16")
    want = bsa.rope(x, axes=(128,), grid=(100,))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = bsa.rope(x, axes=(128,), grid=(100,))
    torch.cuda.current_stream().wait_stream(side)
    b = torch.empty_like(x)
    side.wait_stream(torch.cuda.current_stream())
    bsa.rope(x, axes=(128,), grid=(100,), out=b, stream=side)
    side.synchronize()
    g, y, z = torch.cuda.CUDAGraph(), x.clone(), torch.empty_like(x)
    with torch.cuda.graph(g):
        bsa.rope(y, axes=(128,), grid=(100,), out=z)
    y.copy_(x)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(a, want) and torch.equal(b, want) and torch.equal(z, want)
    with pytest.raises(ValueError):
        bsa.rope(x, axes=(128,))
    with pytest.raises(ValueError):
        bsa.rope(x, axes=(128,), grid=(10, 10))
    with pytest.raises(ValueError):
        bsa.rope(x, axes=(128,), positions=torch.zeros(100, 1, device="cuda"))
    with pytest.raises(ValueError):
        bsa.rope(x, axes=(128,), positions=torch.zeros(99, 1, dtype=torch.int32, device="cuda"))
    with pytest.raises(ValueError):
        bsa.rope(x, x.half(), axes=(128,), grid=(100,))
    with pytest.raises(ValueError):
        bsa.rope(x, x[:, :50], axes=(128,), grid=(100,))
    with pytest.raises(ValueError):
        bsa.rope(x.transpose(1, 2), axes=(100,), grid=(128,))
    with pytest.raises(ValueError):
        bsa.rope(x, axes=(128,), grid=(100,), freq=[1.0])
    with pytest.raises(bsa.BsaError):
        bsa.rope(x, axes=(128,), grid=(101,))
    with pytest.raises(bsa.BsaError):
        bsa.rope(x[:, :, 1:121], axes=(100,), grid=(100,))  # no 16-byte boundary
    with pytest.raises(bsa.BsaError):
        bsa.rope(x[:1].expand(4, 100, 128), axes=(128,), grid=(100,), out=torch.empty_like(x))


def test_a_grid_that_ends_at_the_last_int32_position():
    """Its last token stands on 2^31 - 1 of either axis, as if given; the first axis from the lowest position on."""
    x = torch.randn(2, 30, 64, device="cuda").bfloat16()
    origin, grid = (-(1 << 31), (1 << 31) - 1 - 4), (6, 5)
    where = [(origin[0] + i, origin[1] + j) for i in range(6) for j in range(5)]
    want = bsa.rope(x, axes=(24, 40), positions=torch.tensor(where, dtype=torch.int32, device="cuda"))
    assert torch.equal(bsa.rope(x, axes=(24, 40), grid=grid, origin=origin), want)
