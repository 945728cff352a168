"""The 8-bit cache written from its definition in 64 bits, and how far attention over it may be from the formula.

Writing and reading are exact: each code is the nearest e4m3 number, each scale the smallest power of two that is large enough.

Attention: what the windowed kernels' bounds count (window_reference.forward), over the cache's values; and besides,
  * an element of a row of queries: tiles take it as 8-bit pieces of x / 2^e, the row's largest being above 224 there.  Down to 2^-6 they add up to it; below,
    the first (e4m3, steps of 2^-9) leaves 2^-10 at most and the second (e5m2, three significant bits, or steps of 2^-16) an eighth of that at
    most: 2^-13, which is below 2^-20 of the row's largest.  (Half's third piece is not counted.  Few rows: halves, 2^-38 of it);
  * where codes of V meet the tensor instruction as halves, a block's values far below the largest block's, whose largest is above 224 there, are off by
    2^-25 at most, half of half's smallest step: below 2^-32 of the largest value of V;
  * few rows take a key's weight, 2^15 at most, times its block's scale relative to the largest as a half: for each key 2^-25 of 2^15 in weight at
    most, times 448 in the largest block's units, which is below 2^-38 of the largest value of V.
"""
from __future__ import annotations

import torch

from tests import window_reference as R


def nearest_code(x):
    """Bytes of the nearest e4m3 numbers to finite x with |x| <= 448 (64 bits); NaN where x is not finite."""
    table = torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    a = x.abs().nan_to_num(0.0, 0.0, 0.0)
    i = torch.searchsorted(table, a).clamp(max=126)
    below = (i - 1).clamp(min=0)
    down, up = a - table[below], table[i] - a
    i = torch.where((down < up) | ((down == up) & (below % 2 == 0)), below, i)
    code = torch.where(x < 0, i + 128, i)
    return torch.where(torch.isfinite(x), code, torch.full_like(code, 127)).to(torch.uint8)


def two_to(e):
    return torch.ldexp(torch.ones(e.shape, dtype=torch.float64), e.to(torch.int32))


def values(codes, scales, block):
    """[batch, heads, N, d] in 64 bits from bytes [batch, heads, N, d] and [batch, heads, blocks]."""
    s = scales.to(torch.int32)
    f = torch.where(s == 255, torch.full(s.shape, float("nan"), dtype=torch.float64), two_to(s - 127))
    return codes.view(torch.float8_e4m3fn).double() * f.repeat_interleave(block, 2)[:, :, :codes.shape[2], None]


def write(x, codes, scales, block, starts, counts):
    """The bytes after rows x [batch, heads, N, d] have been written to codes and scales (on the CPU)."""
    codes, scales, x = codes.clone(), scales.clone(), x.double()
    N_kv = codes.shape[2]
    for b in range(x.shape[0]):
        start = 0 if starts is None else int(starts[b])
        n = x.shape[2] if counts is None else min(max(int(counts[b]), 0), x.shape[2])
        p0, p1 = max(start, 0), min(start + n, N_kv)
        for blk in range(p0 // block, -(-p1 // block) if p1 > p0 else 0):
            lo, hi = max(blk * block, p0), min((blk + 1) * block, p1)
            for h in range(x.shape[1]):
                new = x[b, h, lo - start:hi - start]
                a = float(torch.where(torch.isfinite(new), new.abs(), 0.0).max())
                s = 0
                while a > 448.0 * 2.0 ** (s - 127):
                    s += 1
                if blk * block < p0:
                    old = int(scales[b, h, blk])
                    if s > old:
                        held = codes[b, h, blk * block:p0].view(torch.float8_e4m3fn).double() * 2.0 ** (old - s)
                        codes[b, h, blk * block:p0] = nearest_code(held)
                    s = max(s, old)
                scales[b, h, blk] = s
                codes[b, h, lo:hi] = nearest_code(new * (2.0 ** (127 - s) if s < 255 else 0.0))
    return codes, scales


def read(codes, scales, block, N, starts, counts):
    """Rows [batch, heads, N, d] of the cache in 64 bits."""
    v = values(codes, scales, block)
    out = torch.zeros(v.shape[0], v.shape[1], N, v.shape[3], dtype=torch.float64)
    for b in range(v.shape[0]):
        start = 0 if starts is None else int(starts[b])
        n = N if counts is None else min(max(int(counts[b]), 0), N)
        p0, p1 = max(start, 0), min(start + n, v.shape[2])
        if p0 < p1:
            out[b, :, p0 - start:p1 - start] = v[b, :, p0:p1]
    return out


def forward(Q, K, V, **kw):
    """(O, LSE) and their bounds; K and V: the cache's values in 64 bits, laid out as the cache."""
    u = R.HALF_STEP[Q.dtype]
    wO, wL, tO, tL = R.forward(Q, K, V, u=u, **kw)
    fine = lambda x: x.double().abs().nan_to_num(0.0, 0.0, 0.0).amax()  # noqa: E731
    d = Q.shape[-1]
    scale = kw.get("scale") or d ** -0.5
    score = scale * d * fine(Q) * fine(K) * (2.0 ** -20 + 2.0 ** -37)
    keys = V.shape[-2 if kw.get("layout", "hnd") == "hnd" else -3]
    return wO, wL, tO + fine(V) * (2 * score + 2.0 ** -32 + keys * 2.0 ** -38), tL + score
