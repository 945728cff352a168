"""Rotary positions and windowed attention written from their formulas in 64 bits, and how far a kernel that computes in fp32 and
rounds to 16 bits may be from them.

What bounds an output of the attention kernels, with u = eps / 2 the relative rounding of the element type:
  * the output's own rounding: u |out|;
  * the rounding of P (and of dS) to the element type for its product: u times the same sum of absolute values;
  * scores: d products added up in fp32, |dS| <= d 2^-24 sum |q||k| scale, which a weight takes over as a relative error; the exponential, the
    reciprocal and the other sums add a few 2^-22.  Both are ``slack`` below, relative to the sums of absolute values.
"""
from __future__ import annotations

import math

import torch

# Half's steps stop shrinking at 2^-24, so a value below 2^-14 is off by up to 2^-25 however small it is.  That counts for dS and for
# the outputs; P is computed so much larger in half that 2^-25 of it is lost in ``slack``.  (bf16's smallest step is 2^-133.)
HALF_STEP = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}


def heads_first(x, layout):
    """[batch, heads, rows, d] in 64 bits, whatever the layout and with or without a batch."""
    x = x if x.dim() == 4 else x.unsqueeze(0)
    return (x if layout == "hnd" else x.transpose(1, 2)).double()


def laid_out(x, like, layout):
    x = x if layout == "hnd" else x.transpose(1, 2)
    return x if like.dim() == 4 else x[0]


def sees(N, N_kv, batch, left, right, sinks, q_start, kv_len, device):
    """[batch, N, N_kv]: which keys a row sees."""
    n = torch.full((batch,), N_kv, device=device) if kv_len is None else kv_len.to(device).long().clamp(0, N_kv)
    s = n - N if q_start is None else q_start.to(device).long()
    p = s[:, None, None] + torch.arange(N, device=device)[None, :, None]
    j = torch.arange(N_kv, device=device)[None, None, :]
    m = (p >= 0) & (p < n[:, None, None]) & (j < n[:, None, None])
    if right >= 0:
        m = m & (j <= p + right)
    if left >= 0:
        m = m & ((j >= p - left) | (j < sinks))
    return m


def _scores(Q, K, group, mask, scale):
    Kg = K.repeat_interleave(group, 1)
    S = torch.where(mask[:, None], (Q @ Kg.transpose(-1, -2)) * scale, torch.full((), -math.inf, dtype=Q.dtype, device=Q.device))
    # fp32 sums of d products, relative to the sum of their absolute values; the exponent takes it over
    err = Q.shape[-1] * 2.0 ** -24 * (Q.abs() @ Kg.abs().transpose(-1, -2)) * scale
    return S, err


def forward(Q, K, V, *, left, right=0, sinks=0, q_start=None, kv_len=None, scale=0.0, layout="hnd", u):
    """(O, LSE) and their bounds; keys that no row sees are taken as zero, whatever they hold."""
    q, k, v = (heads_first(x, layout) for x in (Q, K, V))
    b, h, n, d = q.shape
    scale = scale or d ** -0.5
    m = sees(n, k.shape[2], b, left, right, sinks, q_start, kv_len, q.device)
    seen = m.any(1)[:, None, :, None]
    k, v = torch.where(seen, k, 0.0), torch.where(seen, v, 0.0)
    group = h // k.shape[1]
    S, err = _scores(q, k, group, m, scale)
    LSE = torch.logsumexp(S, -1)
    P = torch.where(m[:, None], torch.exp(S - LSE.unsqueeze(-1)), 0.0)
    vg = v.repeat_interleave(group, 1)
    O, A = P @ vg, P @ vg.abs()
    worst = torch.where(m[:, None], err, 0.0).amax(-1)  # of a row's scores
    slack = 2 * worst.unsqueeze(-1) + 2.0 ** -19
    tol_O = u * (O.abs() + A) * 1.01 + slack * A + (2.0 ** -25 if Q.dtype == torch.float16 else 0.0)
    tol_L = worst + 2.0 ** -20 * (1 + torch.where(torch.isfinite(LSE), LSE.abs(), 0.0))
    shape = LSE if Q.dim() == 4 else LSE[0]
    return laid_out(O, Q, layout), shape, laid_out(tol_O, Q, layout), tol_L if Q.dim() == 4 else tol_L[0]


def backward(Q, K, V, O, LSE, dO, *, left, right=0, sinks=0, q_start=None, kv_len=None, scale=0.0, layout="hnd", u):
    """(dQ, dK, dV) from the saved O and LSE, and their bounds."""
    q, k, v, o, g = (heads_first(x, layout) for x in (Q, K, V, O, dO))
    L = (LSE if Q.dim() == 4 else LSE.unsqueeze(0)).double()
    b, h, n, d = q.shape
    hk = k.shape[1]
    scale = scale or d ** -0.5
    m = sees(n, k.shape[2], b, left, right, sinks, q_start, kv_len, q.device)
    row, key = m.any(2)[:, None, :, None], m.any(1)[:, None, :, None]
    q, o, g = (torch.where(row, x, 0.0) for x in (q, o, g))
    k, v = torch.where(key, k, 0.0), torch.where(key, v, 0.0)
    group = h // hk
    S, err = _scores(q, k, group, m, scale)
    P = torch.where(m[:, None], torch.exp(S - torch.where(torch.isfinite(L), L, 0.0).unsqueeze(-1)), 0.0)
    kg, vg = k.repeat_interleave(group, 1), v.repeat_interleave(group, 1)
    D = (g * o).sum(-1, keepdim=True)
    dP = g @ vg.transpose(-1, -2)
    dS = P * (dP - D)
    # what dP - D is made of, in absolute values: its fp32 sums are off by d 2^-24 of this at most
    made = P * (g.abs() @ vg.abs().transpose(-1, -2) + (g * o).abs().sum(-1, keepdim=True))
    rel = torch.where(m[:, None], 2 * err + 2.0 ** -19, 0.0)
    least = 2.0 ** -25 if Q.dtype == torch.float16 else 0.0
    off_dS = u * dS.abs() * 1.01 + rel * dS.abs() + (d * 2.0 ** -24) * made + least * m[:, None]
    off_P = u * P * 1.01 + rel * P

    def shared(x):
        return x.view(b, hk, group, *x.shape[2:]).sum(2)
    t = lambda x: x.transpose(-1, -2)  # noqa: E731
    dQ, dK, dV = dS @ kg * scale, shared(t(dS) @ q) * scale, shared(t(P) @ g)
    tQ, tK, tV = off_dS @ kg.abs() * scale, shared(t(off_dS) @ q.abs()) * scale, shared(t(off_P) @ g.abs())
    aQ, aK, aV = dS.abs() @ kg.abs() * scale, shared(t(dS.abs()) @ q.abs()) * scale, shared(t(P) @ g.abs())
    out = []
    for x, tol, a, like in ((dQ, tQ, aQ, Q), (dK, tK, aK, K), (dV, tV, aV, V)):
        bound = u * x.abs() * 1.01 + tol + 2.0 ** -19 * a + least  # (fp32 sums over the tiles: a few 2^-22 of the absolute sum)
        out.append((laid_out(x, like, layout), laid_out(bound, like, layout)))
    return out


def assert_within(got, want, tol, what):
    got = got.double()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)) and torch.equal(got[~fine], want[~fine]), f"{what}: infinities differ"
    d = torch.where(fine, got - torch.where(fine, want, 0.0), 0.0).abs()
    bad = d > torch.where(fine, tol, 0.0) + 1e-30
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((d / (tol + 1e-30)).max()):.2f} times the bound"


# ------------------------------------------------------------------ rotary positions
def angles(n_tokens, axes, *, positions=None, grid=None, first=0, origin=None, theta=10000.0, freq=None, shared_freq=False, device="cpu"):
    """[batch or 1, N, pairs] in 64 bits, and which tokens turn."""
    R = sum(axes)
    f, a = [], []
    for ax, n in enumerate(axes):
        for i in range(n // 2):
            f.append(theta ** (-2.0 * len(f) / R) if shared_freq else theta ** (-2.0 * i / n))
            a.append(ax)
    f = torch.tensor(f if freq is None else freq, dtype=torch.float64, device=device)
    if positions is None:
        pos = torch.zeros((1, n_tokens, len(axes)), dtype=torch.float64, device=device)
        turns = torch.zeros(n_tokens, dtype=torch.bool, device=device)
        where = torch.cartesian_prod(*(torch.arange(g, device=device).double() for g in grid)).view(-1, len(grid))
        pos[0, first:first + len(where)] = where + torch.tensor(origin or [0] * len(grid), dtype=torch.float64, device=device)
        turns[first:first + len(where)] = True
    else:
        pos = (positions if positions.dim() == 3 else positions.unsqueeze(0)).double().to(device)
        turns = torch.ones(n_tokens, dtype=torch.bool, device=device)
    return pos[:, :, a] * f, turns


def rotate(x, angle, turns, *, pairs="interleaved", inverse=False, layout="hnd"):
    """The rotated tensor in 64 bits and, for every element, the absolute values it is made of."""
    y = heads_first(x, layout).clone()
    made = y.abs().clone()
    c, s = torch.cos(angle).unsqueeze(1), torch.sin(angle).unsqueeze(1) * (-1 if inverse else 1)
    P = angle.shape[-1]
    one, two = (slice(0, 2 * P, 2), slice(1, 2 * P, 2)) if pairs == "interleaved" else (slice(0, P), slice(P, 2 * P))
    u, v = y[..., one].clone(), y[..., two].clone()
    w = turns[None, None, :, None]
    y[..., one], y[..., two] = torch.where(w, u * c - v * s, u), torch.where(w, u * s + v * c, v)
    made[..., one] = made[..., two] = u.abs() + v.abs()
    return laid_out(y, x, layout), laid_out(made, x, layout)
