"""How far attention over the 8-bit cache may be from the formula, row by row and head by head, for each way that a call may go.

Besides what the windowed kernels' bounds count (window_reference.forward: the output's rounding, P's to the element type, sums in 32 bits):
  * scores.  From the codes an element of Q is off by 2^-20 of its row's largest, for few rows by 2^-37 (cache_reference has the derivation); d such
    products with K of the row's head.  Through 16 bits half's smallest step counts for K: 2^-25.  A row's weights take an error of its scores over as a
    relative one, numerator and denominator: twice it, times the sum of P |v|;
  * V.  From the codes its halves count in the largest of the scales of the blocks that rows of the call see, U: 2^-25 U at most for each, and the
    weights add up to one.  Through 16 bits half's smallest step: 2^-25;
  * P as a half.  By the tile it is computed 2^7 times as large in units of a reference that the row's largest score is not below, so the sum is 2^7 at least, and
    each key's weight is off by 2^-25 of it at most where half's steps stop shrinking: 2^-32 of its |v|.  Few rows have 2^15 times the weight times the
    block's scale relative to U: 2^-40 of 448 U for each key, which is below 2^-31 U.
"""
from __future__ import annotations

import torch

from tests import window_reference as R


def largest_scales(scales, seen, block):
    """[batch, heads] in 64 bits: the largest scale (bytes [batch, heads, blocks]) of the blocks with a key in seen [batch, N_kv]; 255 aside."""
    blocks = scales.shape[-1]
    pad = torch.nn.functional.pad(seen, (0, blocks * block - seen.shape[1])).view(seen.shape[0], 1, blocks, block).any(-1)
    s = scales.to(seen.device).long()
    s = torch.where(pad & (s < 255), s, 0).amax(-1)
    return torch.ldexp(torch.ones(s.shape, dtype=torch.float64, device=s.device), (s - 127).to(torch.int32))


def forward(way, Q, K, V, V_scales, block, *, left, right=0, sinks=0, q_start=None, kv_len=None, scale=0.0):
    """(O, LSE) and their bounds; Q, K, V [batch, heads, rows, d], K and V the cache's values in 64 bits."""
    kw = dict(left=left, right=right, sinks=sinks, q_start=q_start, kv_len=kv_len, scale=scale, u=R.HALF_STEP[Q.dtype])
    wO, wL, tO, tL = R.forward(Q, K, V, **kw)
    A = R.forward(Q, K, V.abs(), **kw)[0]
    b, h, n, d = Q.shape
    group = h // K.shape[1]
    half = Q.dtype == torch.float16
    sees = R.sees(n, K.shape[2], b, left, right, sinks, q_start, kv_len, Q.device)
    seen = sees.any(1)
    per_head = lambda x: x.repeat_interleave(group, 1)[:, :, None]  # noqa: E731
    largest = lambda x: per_head(torch.where(seen[:, None, :, None], x.abs(), 0.0).amax((2, 3)))  # noqa: E731
    U, k, v = per_head(largest_scales(V_scales, seen, block)), largest(K), largest(V)
    keys = sees.sum(-1)[:, None]
    q = Q.double().abs().amax(-1)
    off = (scale or d ** -0.5) * d * q * {"tiles": 2.0 ** -20 * k, "rows": 2.0 ** -37 * k, "unpacked": k * 0 + (2.0 ** -25 if half else 0.0)}[way]
    least = {"tiles": 2.0 ** -25 * U + keys * 2.0 ** -32 * v, "rows": keys * 2.0 ** -31 * U,
             "unpacked": (2.0 ** -25 + keys * 2.0 ** -32 * v) if half else keys * 0.0 * v}[way]
    return wO, wL, tO + 2 * off[..., None] * A + least[..., None], tL + off
