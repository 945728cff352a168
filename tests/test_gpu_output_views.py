"""Layouts of outputs: those whose entries keep apart are written as they are, those whose entries overlap are refused."""
import random

import pytest
import torch

from paper_2609_25869_b200 import bsa

pytestmark = pytest.mark.gpu


def overlaps(n, s, d):
    """Every element counted (offsets are multiples of 8)."""
    seen = set()
    for b in range(n[0]):
        for h in range(n[1]):
            for r in range(n[2]):
                at = b * s[0] + h * s[1] + r * s[2]
                for e in range(at, at + d, 8):
                    if e in seen:
                        return True
                    seen.add(e)
    return False


def test_overlap_is_decided_exactly():
    """Small layouts with strides drawn at random, most of them interleaved, against the count of every element."""
    rng = random.Random(7)
    buffer = torch.zeros(4096, dtype=torch.bfloat16, device="cuda")
    apart = 0
    for _ in range(400):
        n = [rng.randint(1, 3), rng.randint(1, 4), rng.randint(1, 5)]
        s = [8 * rng.randint(1, 60) for _ in range(3)]
        d = rng.choice([8, 16, 24])
        x = torch.randn(*n, d, device="cuda").bfloat16()
        out = torch.as_strided(buffer, (*n, d), (*s, 1))
        if overlaps(n, s, d):
            with pytest.raises(bsa.BsaError) as e:
                bsa.rope(x, axes=(d,), grid=(n[2],), out=out)
            assert e.value.status == 1, (n, s, d)
        else:
            bsa.rope(x, axes=(d,), grid=(n[2],), out=out)
            assert torch.equal(out, bsa.rope(x, axes=(d,), grid=(n[2],))), (n, s, d)
            apart += 1
    assert 50 < apart < 350


def test_inputs_may_overlap():
    """Queries and keys as windows of one buffer that step by less than a row."""
    buffer = torch.randn(128 * 300, device="cuda").bfloat16()
    x = torch.as_strided(buffer, (2, 200, 64), (8, 64, 1))
    O, L = bsa.window_forward(x, x, x, left=20)
    O2, L2 = bsa.window_forward(*[x.contiguous()] * 3, left=20)
    assert torch.equal(O, O2) and torch.equal(L, L2)
    with pytest.raises(bsa.BsaError) as e:
        bsa.window_forward(x, x, x, left=20, O=x)
    assert e.value.status == 1


@pytest.mark.parametrize("h,hk,n,nk", [(4, 4, 700, 700), (8, 2, 700, 1500), (2, 1, 3, 900), (40, 20, 900, 900)])
@pytest.mark.parametrize("d", [64, 128])
def test_outputs_in_the_place_of_what_was_read_before(h, hk, n, nk, d):
    """O over Q, dQ over O, dK and dV over K and V, either way round: the bits of outputs of their own."""
    g = torch.Generator(device="cuda")
    g.manual_seed(61)
    q, k, v, dO = [torch.empty(s, device="cuda", dtype=torch.bfloat16).normal_(0, 1, generator=g)
                   for s in ((1, h, n, d), (1, hk, nk, d), (1, hk, nk, d), (1, h, n, d))]
    kw = dict(left=300, right=20, sinks=5)
    O, L = bsa.window_forward(q, k, v, **kw)
    G = bsa.window_backward(q, k, v, O, L, dO, **kw)
    q2 = q.clone()
    O2, L2 = bsa.window_forward(q2, k, v, O=q2, **kw)
    assert O2 is q2 and torch.equal(O2, O) and torch.equal(L2, L)
    for swap in (False, True):
        k2, v2, o2 = k.clone(), v.clone(), O.clone()
        G2 = bsa.window_backward(q, k2, v2, o2, L, dO, dQ=o2, dK=v2 if swap else k2, dV=k2 if swap else v2, **kw)
        assert all(torch.equal(a, b) for a, b in zip(G, G2))
    if hk == h:
        o2 = O.clone()
        G2 = bsa.window_backward(q, k, v, o2, L, dO, dK=o2, **kw)
        assert all(torch.equal(a, b) for a, b in zip(G, G2))
    for name, x in (("dQ", q), ("dQ", dO)):
        with pytest.raises(bsa.BsaError) as e:
            bsa.window_backward(q, k, v, O, L, dO, **{name: x}, **kw)
        assert e.value.status == 1
    for x in (k, v):
        if x.shape == q.shape:
            with pytest.raises(bsa.BsaError):
                bsa.window_forward(q, k, v, O=x, **kw)
