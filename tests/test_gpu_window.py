"""Windowed attention through the C ABI: outputs and gradients against the formulas in 64 bits, element by element within what the
roundings allow (window_reference.py has the bounds)."""
import math

import pytest
import torch

from paper_2609_25869_b200 import bsa
from tests import window_reference as R

pytestmark = pytest.mark.gpu
DT = {"bf16": torch.bfloat16, "fp16": torch.float16}


def tensors(seed, layout, b, h, hk, n, nk, d, dtype):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    out = []
    for heads, rows in ((h, n), (hk, nk), (hk, nk), (h, n)):
        s = (b, heads, rows, d) if layout == "hnd" else (b, rows, heads, d)
        out.append(torch.empty(s if b else s[1:], device="cuda", dtype=DT[dtype]).normal_(0, 1, generator=g))
    return out


def ints(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device="cuda")


def check_forward(q, k, v, **kw):
    O, L = bsa.window_forward(q, k, v, **kw)
    torch.cuda.synchronize()
    assert bsa.window_status() == 0
    wO, wL, tO, tL = R.forward(q, k, v, u=R.HALF_STEP[q.dtype], **kw)
    R.assert_within(L, wL, tL, "LSE")
    R.assert_within(O, wO, tO, "O")
    return O, L


def check_backward(q, k, v, g, O, L, **kw):
    got = bsa.window_backward(q, k, v, O, L, g, **kw)
    torch.cuda.synchronize()
    assert bsa.window_status() == 0
    for x, (want, tol), what in zip(got, R.backward(q, k, v, O, L, g, u=R.HALF_STEP[q.dtype], **kw), ("dQ", "dK", "dV")):
        R.assert_within(x, want, tol, what)
    return got


#       b  h  hk    n    nk   left right sinks  starts           lengths
CASES = [
    (1, 1, 1, 128, 128, -1, -1, 0, None, None),               # one whole tile
    (0, 2, 1, 300, 300, 100, 0, 0, None, None),               # no batch dimension; ragged rows and keys
    (1, 2, 2, 513, 513, 0, 0, 0, None, None),                 # a row sees itself
    (2, 4, 2, 200, 700, -1, 0, 0, None, None),                # the last 200 of 700 positions
    (1, 4, 1, 129, 1000, 127, 128, 5, None, None),
    (3, 2, 2, 257, 900, 300, 100, 150, [0, 500, -60], [400, 757, 300]),  # padded, a chunk, rows in front of the sequence
    (2, 3, 3, 140, 140, 64, 63, 500, [0, 0], [140, 1]),       # sinks beyond the keys, one key
    (2, 2, 1, 150, 150, 30, 0, 3, [0, -200], [0, 150]),       # nothing is seen: no keys; no row at a position
    (1, 2, 2, 640, 640, 1, 1, 129, None, None),               # sinks end inside their second tile
    (1, 8, 1, 100, 2000, 700, -1, 40, [1100], [1300]),        # the future without limit, keys behind the length
    (1, 1, 1, 1000, 1000, 5000, 0, 0, None, None),            # a window longer than the sequence
]


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (64, "fp16"), (128, "bf16"), (128, "fp16")])
@pytest.mark.parametrize("case", CASES, ids=lambda c: "x".join(str(x) for x in c[:8]))
def test_forward_and_backward(case, d, dtype, layout):
    b, h, hk, n, nk, left, right, sinks, starts, lengths = case
    q, k, v, g = tensors(sum(case[1:5]) + d, layout, b, h, hk, n, nk, d, dtype)
    kw = dict(left=left, right=right, sinks=sinks, q_start=ints(starts), kv_len=ints(lengths), layout=layout)
    O, L = check_forward(q, k, v, **kw)
    check_backward(q, k, v, g, O, L, **kw)


#       b  h   hk n  nk     left right sinks starts          lengths
FEW = [
    (1, 1, 1, 1, 1, 0, 0, 0, None, None),
    (0, 8, 2, 1, 333, 100, 0, 4, None, None),
    (3, 4, 4, 1, 2000, 300, 0, 4, [1999, 700, 5], [2000, 701, 3]),     # the last: at no position
    (2, 7, 1, 2, 50, -1, 0, 0, [48, -1], [50, 1]),
    (1, 32, 8, 4, 9000, 3000, 0, 100, None, None),                     # 16 rows
    (2, 8, 1, 4, 5000, -1, -1, 0, [4990, 100], [4994, 103]),           # 32 rows: two blocks, the last row of one padding
    (2, 2, 2, 3, 777, 20, 5, 33, [300, -1], [777, 400]),               # sinks end inside a step, windows inside others
    (1, 16, 16, 1, 20000, -1, 0, 0, None, None),
    (2, 3, 3, 1, 64, 8, 0, 2, [0, 0], [0, 1]),                         # no keys; one key
    (2, 2, 1, 1, 110000, -1, 0, 0, [109998, 70000], [109999, 70001]),  # clusters of sixteen
    (1, 4, 1, 8, 600, 590, 0, 1, None, None),                          # 32 rows of different windows
    (1, 4, 1, 9, 600, 590, 0, 1, None, None),                          # 36: three blocks, the last of four rows
    (1, 2, 1, 32, 900, 130, 40, 20, [780], [800]),                     # 64, the last rows at no position
    (1, 3, 1, 85, 5000, -1, 40, 20, [4700], [4750]),                   # 255 over many keys, the last rows at no position
    (1, 1, 1, 256, 5000, 4500, 0, 0, None, None),                      # 256: the most that this kernel takes
    (2, 75, 75, 17, 300, 100, 0, 3, [283, 100], [300, 116]),           # 150 heads, two blocks each: the kernel for tiles, with few rows
]


@pytest.mark.parametrize("layout", ["hnd", "nhd"])
@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (64, "fp16"), (128, "bf16"), (128, "fp16")])
@pytest.mark.parametrize("case", FEW, ids=lambda c: "x".join(str(x) for x in c[:8]))
def test_few_rows(case, d, dtype, layout):
    b, h, hk, n, nk, left, right, sinks, starts, lengths = case
    q, k, v, g = tensors(sum(case[1:5]) + d, layout, b, h, hk, n, nk, d, dtype)
    kw = dict(left=left, right=right, sinks=sinks, q_start=ints(starts), kv_len=ints(lengths), layout=layout)
    O, L = check_forward(q, k, v, **kw)
    check_backward(q, k, v, g, O, L, **kw)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("n", [1, 3, 200])
def test_keys_that_no_row_sees_may_hold_anything(d, n):
    """Behind the length, in front of the window, between the sinks and the window: NaN and infinities there change no bit."""
    q, k, v, g = tensors(11, "hnd", 2, 4, 2, n, 1000, d, "bf16")
    starts, lengths = [600, 130], [600 + n, 130 + n]
    kw = dict(left=150, right=0, sinks=7, q_start=ints(starts), kv_len=ints(lengths))
    O, L = check_forward(q, k, v, **kw)
    G = check_backward(q, k, v, g, O, L, **kw)
    k2, v2 = k.clone(), v.clone()
    for b in range(2):
        hidden = [slice(lengths[b], None)] + ([slice(7, starts[b] - 150)] if starts[b] - 150 > 7 else [])
        for s in hidden:
            k2[b, :, s], v2[b, :, s] = float("nan"), float("nan")
            k2[b, :, s][:, ::2], v2[b, :, s][:, ::3] = float("inf"), float("-inf")
    O2, L2 = bsa.window_forward(q, k2, v2, **kw)
    G2 = bsa.window_backward(q, k2, v2, O2, L2, g, **kw)
    assert torch.equal(O, O2) and torch.equal(L, L2) and all(torch.equal(a, b) for a, b in zip(G, G2))


@pytest.mark.parametrize("d", [64, 128])
def test_rows_at_no_position_may_hold_anything(d):
    q, k, v, g = tensors(12, "nhd", 2, 2, 1, 300, 300, d, "fp16")
    kw = dict(left=-1, right=10, sinks=0, q_start=ints([0, -40]), kv_len=ints([211, 200]), layout="nhd")
    O, L = check_forward(q, k, v, **kw)
    G = check_backward(q, k, v, g, O, L, **kw)
    q2, g2 = q.clone(), g.clone()
    for t in (q2, g2):
        t[0, 211:], t[1, :40], t[1, 240:] = float("nan"), float("inf"), float("nan")
    O2, L2 = bsa.window_forward(q2, k, v, **kw)
    G2 = bsa.window_backward(q2, k, v, O2, L2, g2, **kw)
    assert torch.equal(O, O2) and torch.equal(L, L2) and all(torch.equal(a, b) for a, b in zip(G, G2))
    assert not O[0, 211:].any() and (L[1, :, :40] == -math.inf).all() and not G[0][0, 211:].any()


@pytest.mark.parametrize("dtype", ["bf16", "fp16"])
@pytest.mark.parametrize("n", [1, 400])
def test_scores_that_grow_along_the_keys(n, dtype):
    """Every tile lies above the reference of the tiles before it by far more than 2^8, up to weights of exactly zero."""
    d, nk = 128, 700
    q, k, v, g = tensors(13, "hnd", 1, 2, 1, n, nk, d, dtype)
    q[:], k[:] = 0, 0
    q[..., 0] = 4.0
    k[..., 0] = torch.arange(nk, device="cuda").to(k.dtype) * 0.5
    kw = dict(left=-1, right=-1, sinks=0, scale=0.25)
    O, L = check_forward(q, k, v, **kw)
    check_backward(q, k, v, g, O, L, **kw)
    k[..., 0] = -k[..., 0]
    check_forward(q, k, v, **kw)


@pytest.mark.parametrize("d,dtype", [(64, "bf16"), (128, "bf16"), (128, "fp16")])
def test_references_that_move_now_and_then(d, dtype):
    """Long lists in which single tiles lie far above all before them, in places that differ from head to head; many items per CTA, windows
    and sinks, so that such tiles come first, second and last in their lists."""
    h, n = 40, 2600
    q, k, v, _ = tensors(21, "hnd", 1, h, h, n, n, d, dtype)
    g = torch.Generator().manual_seed(5)
    q[..., 0], k[..., 0] = 6.0, 0.0
    level = torch.zeros(h, n)
    for i in range(h):
        for j in sorted(torch.randint(0, n, (6,), generator=g).tolist()):
            level[i, j:] += float(torch.randint(2, 9, (1,), generator=g)) * d ** 0.5 / 6.0
        # falls again now and then, so that windows further on see their own rises
        level[i, torch.randint(0, n, (1,), generator=g).item():] *= 0.25
    k[0, :, :, 0] = level.to(k)
    for kw in (dict(left=900, right=0, sinks=3), dict(left=400, right=200, sinks=140), dict(left=-1, right=0)):
        check_forward(q, k, v, **kw)


def test_scale_and_large_scores():
    q, k, v, g = tensors(14, "hnd", 1, 2, 2, 256, 256, 64, "fp16")
    for scale in (1.0, 1e-3):
        kw = dict(left=60, right=0, sinks=1, scale=scale)
        O, L = check_forward(q, k, v, **kw)
        check_backward(q, k, v, g, O, L, **kw)


@pytest.mark.parametrize("sinks,left", [(1, 100), (130, 200), (300, 64)])
@pytest.mark.parametrize("group", [1, 3])
def test_sinks_of_long_sequences(sinks, left, group):
    """The sinks' tiles are cut into shares of their queries."""
    q, k, v, g = tensors(15, "hnd", 1, 2 * group, 2, 3000, 3000, 64, "bf16")
    kw = dict(left=left, right=0, sinks=sinks)
    O, L = check_forward(q, k, v, **kw)
    check_backward(q, k, v, g, O, L, **kw)


@pytest.mark.parametrize("h,hk,n,left", [(1, 1, 1500, -1), (2, 1, 1200, 900), (8, 1, 600, 100), (3, 3, 1100, -1)])
@pytest.mark.parametrize("d", [64, 128])
def test_gradients_of_few_heads(h, hk, n, left, d):
    """So few key tiles that every one is cut into shares."""
    q, k, v, g = tensors(23, "hnd", 1, h, hk, n, n, d, "bf16")
    kw = dict(left=left, right=0, sinks=5, kv_len=ints([n - 70]), q_start=ints([0]))
    O, L = check_forward(q, k, v, **kw)
    G = check_backward(q, k, v, g, O, L, **kw)
    assert all(torch.equal(a, b) for a, b in zip(G, bsa.window_backward(q, k, v, O, L, g, **kw)))


def test_views_of_a_fused_projection_and_of_a_cache():
    b, n, h, d = 2, 200, 4, 128
    qkv = torch.randn(b, n, 3, h, d, device="cuda").bfloat16()
    q, k, v = qkv.unbind(2)
    kw = dict(left=50, right=0, sinks=2, layout="nhd")
    O, L = check_forward(q, k, v, **kw)
    O2, L2 = bsa.window_forward(q.contiguous(), k.contiguous(), v.contiguous(), **kw)
    assert torch.equal(O, O2) and torch.equal(L, L2)
    g = torch.randn_like(O)
    G = check_backward(q, k, v, g, O, L, **kw)
    grads = torch.full_like(qkv, 9.0)  # the gradients into one tensor again
    dq, dk, dv = grads.unbind(2)
    bsa.window_backward(q, k, v, O, L, g, dQ=dq, dK=dk, dV=dv, **kw)
    assert all(torch.equal(a, x) for a, x in zip(G, (dq, dk, dv)))
    cache = torch.randn(2, b, h, 512, d, device="cuda").bfloat16()  # [k/v, batch, heads, capacity, d], 200 rows in use
    cache[0, :, :, :n], cache[1, :, :, :n] = k.transpose(1, 2), v.transpose(1, 2)
    O3, _ = bsa.window_forward(q.transpose(1, 2), cache[0], cache[1], left=50, sinks=2, q_start=ints([0] * b), kv_len=ints([n] * b))
    assert torch.equal(O3.transpose(1, 2), O)
    # rows behind O's own in a larger buffer stay as they are
    buf = torch.full((b, h, n + 100, d), 5.0, dtype=torch.bfloat16, device="cuda")
    bsa.window_forward(q.transpose(1, 2), cache[0, :, :, :n], cache[1, :, :, :n], left=50, sinks=2, O=buf[:, :, :n])
    assert torch.equal(buf[:, :, :n].transpose(1, 2), O) and (buf[:, :, n:] == 5).all()


@pytest.mark.parametrize("n", [1, 130])
def test_a_cache_beyond_32_bits_of_elements(n):
    h, nk, d = 9, 1 << 21, 128  # 2.4e9 elements
    k = torch.zeros((h, nk, d), dtype=torch.bfloat16, device="cuda")
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    k[-1, -600:].normal_(0, 1, generator=g)
    k[-1, :8].normal_(0, 1, generator=g)
    q = torch.empty((h, n, d), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g)
    O, L = bsa.window_forward(q, k, k, left=400, sinks=3)
    near = torch.cat([k[-1:, :3], k[-1:, -600:]], 1)
    wO, wL, tO, tL = R.forward(q[-1:], near, near, left=400, sinks=3, u=2.0 ** -8)
    R.assert_within(L[-1:], wL, tL, "LSE")
    R.assert_within(O[-1:], wO, tO, "O")
    assert not O[0].any()


@pytest.mark.parametrize("d", [64, 128])
def test_bits_do_not_change_from_run_to_run_or_with_the_batch(d):
    q, k, v, g = tensors(16, "hnd", 3, 12, 4, 2000, 2000, d, "bf16")
    kw = dict(left=300, right=20, sinks=70)
    O, L = bsa.window_forward(q, k, v, **kw)
    G = bsa.window_backward(q, k, v, O, L, g, **kw)
    for _ in range(3):
        O2, L2 = bsa.window_forward(q, k, v, **kw)
        assert torch.equal(O, O2) and torch.equal(L, L2)
        assert all(torch.equal(a, b) for a, b in zip(G, bsa.window_backward(q, k, v, O, L, g, **kw)))
    one = [t[1:2, :6].contiguous() if t.shape[1] == 12 else t[1:2, :2].contiguous() for t in (q, k, v)]
    O1, L1 = bsa.window_forward(*one, **kw)
    assert torch.equal(O1, O[1:2, :6]) and torch.equal(L1, L[1:2, :6])
    dQ1 = bsa.window_backward(*one, O1, L1, g[1:2, :6].contiguous(), **kw)[0]
    assert torch.equal(dQ1, G[0][1:2, :6])


def test_many_items_with_edges_on_every_tile():
    """Short windows over many items: the protocol between the warps runs through all of its orders, and ends."""
    q, k, v, g = tensors(22, "nhd", 2, 24, 24, 6000, 6000, 64, "bf16")
    kw = dict(left=200, right=100, sinks=300, layout="nhd")
    O, L = bsa.window_forward(q, k, v, **kw)
    for _ in range(20):
        O2, L2 = bsa.window_forward(q, k, v, **kw)
    assert bsa.window_status() == 0 and torch.equal(O, O2) and torch.equal(L, L2)
    part = dict(left=200, right=100, sinks=300, layout="nhd")
    for h in (0, 23):
        wO, wL, tO, tL = R.forward(q[1:, :, h:h + 1], k[1:, :, h:h + 1], v[1:, :, h:h + 1], u=2.0 ** -8, **part)
        R.assert_within(O[1:, :, h:h + 1], wO, tO, "O")
        R.assert_within(L[1:, h:h + 1], wL, tL, "LSE")


@pytest.mark.parametrize("n", [2, 300])
def test_streams_and_graphs(n):
    q, k, v, g = tensors(17, "hnd", 2, 4, 2, n, 600, 64, "bf16")
    lens = ints([600, 450])
    kw = dict(left=100, sinks=4, kv_len=lens)
    O, L = bsa.window_forward(q, k, v, **kw)
    G = bsa.window_backward(q, k, v, O, L, g, **kw)
    side, other = torch.cuda.Stream(), torch.cuda.Stream()
    results = []
    for s in (side, other):  # two calls at once
        s.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(s):
            o, l = bsa.window_forward(q, k, v, **kw)
            results.append((o, l, *bsa.window_backward(q, k, v, o, l, g, **kw)))
    for s in (side, other):
        torch.cuda.current_stream().wait_stream(s)
    for r in results:
        assert all(torch.equal(a, b) for a, b in zip(r, (O, L, *G)))
    # one graph: forward and backward; the lengths change between replays
    graph, q2, lens2 = torch.cuda.CUDAGraph(), q.clone(), lens.clone()
    kw2 = dict(kw, kv_len=lens2)
    with torch.cuda.graph(graph):
        o, l = bsa.window_forward(q2, k, v, **kw2)
        grads = bsa.window_backward(q2, k, v, o, l, g, **kw2)
    for new in ([600, 450], [333, 2], [600, 450]):
        lens2.copy_(ints(new))
        graph.replay()
        want = bsa.window_forward(q, k, v, **dict(kw, kv_len=ints(new)))
        assert torch.equal(o, want[0]) and torch.equal(l, want[1])
        assert all(torch.equal(a, b) for a, b in zip(grads, bsa.window_backward(q, k, v, *want, g, **dict(kw, kv_len=ints(new)))))
    assert all(torch.equal(a, b) for a, b in zip(grads, G))


def test_a_layer_from_positions_to_gradients():
    """Rotation, attention and the way back as a training step uses them, and the same rotation in front of a block-sparse plan."""
    b, h, hk, n, d, axes, grid = 2, 4, 2, 240, 64, (16, 24, 24), (4, 6, 10)
    q, k, v, g = tensors(18, "nhd", b, h, hk, n, n, d, "fp16")
    kw = dict(left=70, right=30, sinks=10, layout="nhd")
    qr, kr = bsa.rope(q, k, axes=axes, grid=grid, layout="nhd")
    O, L = bsa.window_forward(qr, kr, v, **kw)
    dqr, dkr, dv = bsa.window_backward(qr, kr, v, O, L, g, **kw)
    dq, dk = bsa.rope(dqr, dkr, axes=axes, grid=grid, layout="nhd", inverse=True)
    # the whole chain in 64 bits, differentiated automatically
    angle, turns = R.angles(n, axes, grid=grid, device="cuda")
    leaves = [t.double().requires_grad_() for t in (q, k, v)]

    def turn(x):
        y = x.transpose(1, 2)
        c, s = angle.cos().unsqueeze(1), angle.sin().unsqueeze(1)
        u, w = y[..., 0::2], y[..., 1::2]
        return torch.stack([u * c - w * s, u * s + w * c], -1).flatten(-2)
    Q, K, V = turn(leaves[0]), turn(leaves[1]), leaves[2].transpose(1, 2)
    m = R.sees(n, n, b, 70, 30, 10, None, None, "cuda")[:, None]
    S = (Q @ K.repeat_interleave(2, 1).transpose(-1, -2) * d ** -0.5).masked_fill(~m, -math.inf)
    want = torch.softmax(S, -1) @ V.repeat_interleave(2, 1)
    (want.transpose(1, 2) * g.double()).sum().backward()
    # each of the chain's seven roundings (rotations, P, O, dS, gradients) is half a step of 2^-11 of its values at most; in the
    # 2-norm they add up to less than seven of them
    for got, ref in ((O.double(), want.transpose(1, 2)), (dq.double(), leaves[0].grad), (dk.double(), leaves[1].grad), (dv.double(), leaves[2].grad)):
        assert (got - ref).norm() <= 7 * 2.0 ** -11 * ref.norm()
    mask = torch.ones(b * h, 4, 4, dtype=torch.uint8, device="cuda")
    qh, kh, vh = (x.transpose(1, 2).repeat_interleave(h // x.shape[2], 1).reshape(b * h, n, d).contiguous() for x in (qr, kr, v))
    with bsa.plan_create(mask, 64, 64, n, b * h, d, dtype="fp16") as plan:
        dense, lse = plan.forward(qh, kh, vh)
    O2, L2 = bsa.window_forward(qr, kr, v, left=-1, right=-1, layout="nhd")
    assert (dense.view(b, h, n, d).transpose(1, 2).double() - O2.double()).norm() <= 4 * 2.0 ** -11 * O2.double().norm()
    assert (lse.view(b, h, n) - L2).abs().max() <= 1e-4


def test_streaming_token_by_token_equals_one_pass():
    """A cache that is filled token by token: positions into the cache, then the new token's attention."""
    h, hk, n, d = 4, 2, 40, 64
    q, k, v, _ = tensors(19, "hnd", 1, h, hk, n, n, d, "bf16")
    kw = dict(left=9, sinks=3)
    Q, K = bsa.rope(q, k, axes=(64,), grid=(n,))
    whole, lse = bsa.window_forward(Q, K, v, **kw)
    ck, cv = (torch.full((1, hk, 64, d), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for t in range(n):
        pos = torch.full((1, 1), t, dtype=torch.int32, device="cuda")
        qt = torch.empty_like(q[:, :, t:t + 1])
        bsa.rope(q[:, :, t:t + 1], k[:, :, t:t + 1], axes=(64,), positions=pos, out=(qt, ck[:, :, t:t + 1]))
        cv[:, :, t] = v[:, :, t]
        o, l = bsa.window_forward(qt, ck, cv, q_start=ints([t]), kv_len=ints([t + 1]), **kw)
        # two kernels, each within half a step for P and for O of the formula
        assert (o[:, :, 0].double() - whole[:, :, t].double()).norm() <= 4 * 2.0 ** -8 * whole[:, :, t].double().norm()
        assert (l[:, :, 0] - lse[:, :, t]).abs().max() <= 2e-5


def test_refusals():
    q, k, v, g = tensors(20, "hnd", 2, 4, 2, 100, 200, 64, "bf16")
    O, L = bsa.window_forward(q, k, v, left=5)
    for bad in (dict(q=q.float()), dict(k=k.half()), dict(v=v[:, :1]), dict(k=k[:1]), dict(k=k[0]), dict(q=q.transpose(2, 3)),
                dict(q=q[..., :32], k=k)):
        t = {"q": q, "k": k, "v": v, **bad}
        with pytest.raises(ValueError):
            bsa.window_forward(t["q"], t["k"], t["v"], left=5)
    for bad in (dict(O=O[:1]), dict(LSE=L.double()), dict(LSE=L[:, :2]), dict(q_start=torch.zeros(2, device="cuda")),
                dict(kv_len=torch.zeros(3, dtype=torch.int32, device="cuda")), dict(kv_len=torch.zeros(2, dtype=torch.int32))):
        with pytest.raises(ValueError):
            bsa.window_forward(q, k, v, left=5, **bad)
    for bad in (dict(left=-2), dict(left=5, sinks=-1), dict(left=5, scale=-1.0)):
        with pytest.raises(bsa.BsaError) as e:
            bsa.window_forward(q, k, v, **bad)
        assert e.value.status == 1
    with pytest.raises(bsa.BsaError):  # strides of 4 elements; a key head for every row of a batch
        bsa.window_forward(q, torch.zeros(2, 2, 200, 68, device="cuda").bfloat16()[..., :64], v, left=5)
    with pytest.raises(bsa.BsaError):
        bsa.window_forward(q, k[:, :1].expand(2, 2, 200, 64), v, left=5)
    with pytest.raises(bsa.BsaError) as e:
        x = torch.zeros(2, 100, 256, device="cuda").bfloat16()
        bsa.window_forward(x, x, x, left=5)
    assert e.value.status == 2
    with pytest.raises(ValueError):
        bsa.window_backward(q, k, v, O, L, g[:1], left=5)
    with pytest.raises(ValueError):
        bsa.window_backward(q, k, v, O, L, g, left=5, dK=torch.empty_like(q))
    desc = bsa._WINDOW.pack(2, 4, 2, 64, 100, 200, 5, 0, 0, 0, 0.0, 0, 0)
    need = bsa.lib().bsa_window_workspace_bytes(desc)
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    vs = [bsa._view(t, False, q.dtype, 0, "")[4] for t in (q, k, v, O)]
    gs = [bsa._view(t, False, q.dtype, 0, "")[4] for t in (g, torch.empty_like(q), torch.empty_like(k), torch.empty_like(v))]
    call = lambda p, n: bsa.lib().bsa_window_backward(desc, *vs, L.data_ptr(), *gs, p, n, None)  # noqa: E731
    assert call(ws.data_ptr(), need - 1) == 1 and call(None, need) == 1 and call(ws.data_ptr() + 4, need) == 1
    assert call(ws.data_ptr(), need) == 0
    torch.cuda.synchronize()


def test_first_calls_of_a_process_may_be_captured():
    """Nothing that a first call sets up (attributes, addresses, module loading) is refused while a stream is being captured."""
    import os
    import subprocess
    import sys
    code = """
import torch
from paper_2609_25869_b200 import bsa
x = [torch.randn(1, 2, 200, 64, device='cuda').bfloat16() for _ in range(4)]
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    q, k = bsa.rope(x[0], x[1], axes=(64,), grid=(200,))
    O, L = bsa.window_forward(q, k, x[2], left=20, sinks=2)
    o, _ = bsa.window_forward(q[:, :, -1:], k, x[2], left=20, sinks=2)
    G = bsa.window_backward(q, k, x[2], O, L, x[3], left=20, sinks=2)
g.replay()
torch.cuda.synchronize()
q2, k2 = bsa.rope(x[0], x[1], axes=(64,), grid=(200,))
O2, L2 = bsa.window_forward(q2, k2, x[2], left=20, sinks=2)
assert torch.equal(O, O2) and torch.equal(L, L2)
assert all(torch.equal(a, b) for a, b in zip(G, bsa.window_backward(q2, k2, x[2], O2, L2, x[3], left=20, sinks=2)))
assert bsa.window_status() == 0
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("heads", [9, 16, 36])
def test_one_row_of_several_heads_against_a_long_cache(heads, d):
    """Clusters of sixteen that run at once, of eight, and of sixteen again where not all of eight would run at once; short lengths too."""
    n, nk = 1, 100000
    q, k, v, _ = tensors(24, "hnd", 1, heads, heads, n, nk, d, "bf16")
    for length in (nk, 70001, 300):
        kw = dict(left=-1, sinks=0, kv_len=ints([length]))
        O, L = bsa.window_forward(q, k, v, **kw)
        for h in (0, heads - 1):
            wO, wL, tO, tL = R.forward(q[:, h:h + 1], k[:, h:h + 1, :length], v[:, h:h + 1, :length], left=-1, u=2.0 ** -8)
            R.assert_within(L[:, h:h + 1], wL, tL, "LSE")
            R.assert_within(O[:, h:h + 1], wO, tO, "O")
