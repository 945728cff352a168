"""The 64-bit formulas that the GPU tests compare with, themselves: against automatic differentiation and against differences."""
import math

import pytest
import torch

from tests import window_reference as R


def _case(seed, b, h, hk, n, nk, d):
    g = torch.Generator().manual_seed(seed)
    return [torch.randn(b, x, y, d, generator=g, dtype=torch.float64) for x, y in ((h, n), (hk, nk), (hk, nk), (h, n))]


@pytest.mark.parametrize("left,right,sinks,start,length", [(3, 0, 2, None, None), (-1, 2, 0, [0, 4], [9, 12]), (0, -1, 5, [-2, 7], [3, 11])])
def test_gradients_are_those_of_the_forward(left, right, sinks, start, length):
    q, k, v, g = _case(1, 2, 4, 2, 7, 12, 8)
    kw = dict(left=left, right=right, sinks=sinks, q_start=None if start is None else torch.tensor(start),
              kv_len=None if length is None else torch.tensor(length), u=0.0)
    O, L, _, _ = R.forward(q, k, v, **kw)
    (dQ, _), (dK, _), (dV, _) = R.backward(q, k, v, O, L, g, **kw)
    h = 1e-5
    for x, dx in ((q, dQ), (k, dK), (v, dV)):
        way = torch.randn(x.shape, generator=torch.Generator().manual_seed(3), dtype=torch.float64)
        f = [float((R.forward(*[t + s * h * way if t is x else t for t in (q, k, v)], **kw)[0] * g).sum()) for s in (1, -1)]
        want = float((dx * way).sum())
        # a symmetric difference is off by h^2 / 6 times a third derivative, a few units here, and by 2^-52 / h of the values
        assert abs((f[0] - f[1]) / (2 * h) - want) < 1e-7 * (1 + abs(want))


def test_rows_at_no_position_see_nothing():
    m = R.sees(4, 6, 2, 1, 0, 1, torch.tensor([-1, 3]), torch.tensor([6, 5]), "cpu")
    assert m[0].int().tolist() == [[0, 0, 0, 0, 0, 0], [1, 0, 0, 0, 0, 0], [1, 1, 0, 0, 0, 0], [1, 1, 1, 0, 0, 0]]
    assert m[1].int().tolist() == [[1, 0, 1, 1, 0, 0], [1, 0, 0, 1, 1, 0], [0] * 6, [0] * 6]


def test_softmax_of_the_definition():
    q, k, v, _ = _case(5, 1, 2, 1, 3, 5, 4)
    O, L, _, _ = R.forward(q, k, v, left=-1, right=-1, scale=0.3, u=0.0)
    S = q[0, 1, 2] @ k[0, 0].T * 0.3
    assert torch.allclose(O[0, 1, 2], torch.softmax(S, 0) @ v[0, 0]) and math.isclose(float(L[0, 1, 2]), float(torch.logsumexp(S, 0)))


@pytest.mark.parametrize("pairs", ["interleaved", "halves"])
def test_rotation_is_orthogonal_and_its_inverse_its_gradient(pairs):
    x = torch.randn(2, 3, 5, 16, dtype=torch.float64, requires_grad=True)
    a, t = R.angles(5, [4, 6, 4], grid=[1, 2, 2], first=1, origin=[3, 0, -2])
    y, _ = R.rotate(x, a, t, pairs=pairs)
    g = torch.randn(2, 3, 5, 16, dtype=torch.float64)
    back, _ = R.rotate(g, a, t, pairs=pairs, inverse=True)
    (y * g).sum().backward()
    assert torch.allclose(x.grad, back) and torch.allclose((y ** 2).sum(-1), (x ** 2).sum(-1))
    assert torch.equal(y[:, :, 0], x[:, :, 0]) and torch.equal(y[..., 14:], x[..., 14:])
