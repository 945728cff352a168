"""Rotary positions and sliding-window attention of long token sequences: what is measured of them, and their plain forms.

A token sequence (a clip cut into latent tokens, row-major over time, height and width, or text) gets rotary positions
with one or several axes; its queries then attend to a window of keys around their own position and to a few first
tokens ("sinks") that stay visible for the whole sequence.

Fields of a case
    op       "rope"      rotate Q and K                       "rope_grad"  the gradients through that rotation
             "forward"   windowed attention: O and its LSE    "backward"   dQ, dK, dV from the saved O and LSE
    batch, heads, heads_kv, N, N_kv, d, dtype, layout    tensors [batch, heads, N, d] ("hnd") or [batch, N, heads, d] ("nhd")
    left, right, sinks   the query at position p sees the keys j <= p + right with j >= p - left or j < sinks; -1: no limit
    starts, lengths      "a,b,...": position of each sequence's first query, and its number of keys ("": the queries are
                         the last N positions, and all N_kv keys count); a row at no position of its sequence sees nothing
    axes                 channels rotated by each axis, "44,42,42"
    pairs, shared        how channels pair up, and whether the axes share one list of frequencies
    grid                 "TxHxW": positions are the grid's, row-major; "": they are given, one row of them per token
    first                tokens in front of the grid's (text): these, and tokens behind it, stay as they are
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_CHUNK = 1 << 30            # score elements of one step of the plain form
_MAX_FLOPS = 1.0e13         # a drawn attention case stays below the largest listed one
_MAX_ROPE_ELEMENTS = 5.0e8  # and a drawn rotation too


def _rope(name, op, heads, heads_kv, N, d, axes, batch=1, dtype="bf16", layout="hnd", pairs="interleaved", shared=False,
          grid="", first=0):
    c = {"op": op, "batch": batch, "heads": heads, "heads_kv": heads_kv, "N": N, "d": d, "dtype": dtype, "layout": layout,
         "axes": axes, "pairs": pairs, "shared": shared, "grid": grid, "first": first}
    return dict(c, name=name) if name else c


def _window(name, op, heads, heads_kv, N, N_kv, d, left, right=0, sinks=0, batch=1, dtype="bf16", layout="hnd", starts="",
            lengths=""):
    c = {"op": op, "batch": batch, "heads": heads, "heads_kv": heads_kv, "N": N, "N_kv": N_kv, "d": d, "dtype": dtype,
         "layout": layout, "left": left, "right": right, "sinks": sinks, "starts": starts, "lengths": lengths}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the next token of a stream: one row per head, latency is everything
        _rope("rope_token", "rope", 32, 8, 1, 128, "128", layout="nhd", batch=4),
        # one layer of an 81-frame 720p clip as the fused projection leaves Q and K: 21 x 45 x 80 latent tokens
        _rope("rope_clip", "rope", 24, 24, 75600, 128, "44,42,42", layout="nhd", grid="21x45x80"),
        # text and images mixed: positions given per token, channels paired across halves, one list of frequencies
        _rope("rope_given_halves", "rope", 28, 4, 5003, 128, "32,48,48", batch=2, dtype="fp16", pairs="halves", shared=True),
        # the training step's way back through the rotation, part of the channels unrotated, text in front of the grid
        _rope("rope_clip_grad", "rope_grad", 16, 16, 33024, 64, "16,20,20", layout="hnd", grid="8x64x64", first=256),
        # the next token of four short streams: a window and four sinks out of a cache, latency is everything
        _window("token_window", "forward", 32, 8, 1, 8192, 128, 1023, sinks=4, batch=4, starts="8000,1500,300,5",
                lengths="8001,1501,301,6"),
        # the next token over all of a long cache, sequences of very different length
        _window("token_long", "forward", 32, 8, 1, 115200, 128, -1, batch=6, layout="nhd",
                starts="115199,90000,75599,32767,20001,1110", lengths="115200,90001,75600,32768,20002,1111"),
        # the next chunk of a streamed clip: three latent frames of 1560 tokens against the cached frames of the window and
        # the first frame; inside the chunk every token sees every token of its own and earlier frames, and some later ones
        _window("stream_chunk", "forward", 12, 12, 4680, 32760, 128, 18720, right=4679, sinks=1560),
        # an ordinary training or prefill layer: causal window, shared key heads
        _window("prefill_mid", "forward", 16, 4, 16384, 16384, 128, 2047, sinks=16),
        # a padded batch of half tensors, token-major, small heads
        _window("prefill_padded", "forward", 16, 16, 3600, 3600, 64, 511, right=63, sinks=64, batch=3, dtype="fp16",
                layout="nhd", starts="0,0,0", lengths="3600,2111,1025"),
        # the largest: one layer of a 720p clip, 115200 tokens, the first frame and the last frames visible
        _window("prefill_clip", "forward", 24, 24, 115200, 115200, 128, 4095, right=4095, sinks=1024),
        # gradients of the ordinary layer
        _window("backward_mid", "backward", 16, 4, 16384, 16384, 128, 2047, sinks=16),
        # gradients of a ragged padded batch with small heads, half tensors
        _window("backward_padded", "backward", 12, 12, 5001, 5001, 64, 1023, right=255, sinks=100, batch=2, dtype="fp16",
                layout="nhd", starts="0,0", lengths="5001,3333"),
    ]


def _log(rng, lo, hi):
    return int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))


def draw(rng):
    while True:
        op = rng.choice(["rope", "rope_grad", "forward", "forward", "forward", "backward", "backward"])
        d = rng.choice([64, 128])
        heads_kv = rng.choice([1, 2, 4, 8, 12, 16, 24])
        heads = heads_kv * rng.choice([1, 1, 1, 2, 4, 7, 8])
        batch = rng.choice([1, 1, 2, 3, 4])
        dtype = rng.choice(["bf16", "bf16", "fp16"])
        layout = rng.choice(["hnd", "nhd"])
        if heads > 32:
            continue
        if op in ("rope", "rope_grad"):
            axes = rng.choice([[d], [d // 2, d // 2], [d // 4, 3 * d // 8, 3 * d // 8], [d // 8, 7 * d // 16, 7 * d // 16],
                               [d // 4, d // 4, d // 4]])
            grid, first = "", 0
            N = _log(rng, 1, 75600)
            if len(axes) == 3 and rng.random() < 0.6:
                g = [rng.randint(1, 21), rng.randint(5, 60), rng.randint(5, 80)]
                first = rng.choice([0, 77, 256])
                N = g[0] * g[1] * g[2] + first + rng.choice([0, 0, 19])
                grid = "x".join(str(x) for x in g)
            if batch * N * (heads + heads_kv) * d > _MAX_ROPE_ELEMENTS:
                continue
            return _rope("", op, heads, heads_kv, N, d, ",".join(str(a) for a in axes), batch=batch, dtype=dtype,
                         layout=layout, pairs=rng.choice(["interleaved", "halves"]), shared=rng.random() < 0.5, grid=grid,
                         first=first)
        right = rng.choice([0, 0, 0, 63, _log(rng, 1, 4680)])
        left = rng.choice([-1, _log(rng, 1, 8192), _log(rng, 128, 8192), _log(rng, 128, 8192)])
        sinks = rng.choice([0, 1, 4, 16, 100, _log(rng, 1, 1560)])
        starts = lengths = ""
        if op == "forward" and rng.random() < 0.5:  # tokens or a chunk against a cache
            N_kv = _log(rng, 64, 115200)
            N = min(N_kv, rng.choice([1, 1, 1, 2, 5, _log(rng, 1, 4680)]))
            if rng.random() < 0.6:
                n = [max(N, _log(rng, max(1, N_kv // 32), N_kv)) for _ in range(batch)]
                lengths = ",".join(str(x) for x in n)
                starts = ",".join(str(x - N) for x in n)
        else:
            N = N_kv = _log(rng, 100, 65536 if op == "forward" else 24000)
            if batch > 1 and rng.random() < 0.6:
                lengths = ",".join(str(_log(rng, max(1, N // 32), N)) for _ in range(batch))
                starts = ",".join("0" for _ in range(batch))
        c = _window("", op, heads, heads_kv, N, N_kv, d, left, right, sinks, batch=batch, dtype=dtype, layout=layout,
                    starts=starts, lengths=lengths)
        elements = batch * (2 * heads * N + 2 * heads_kv * N_kv) * d
        dense = 4.0 * d * batch * heads * N * min(N_kv, N_kv if left < 0 else left + max(0, right) + sinks + _rows_of(c))
        if dense <= _MAX_FLOPS * (1.0 if op == "forward" else 0.1) and elements <= 2.0e9:
            return c


# ------------------------------------------------------------------ what a case stands for
def _sequences(c):
    """(position of the first query, number of keys) of every sequence."""
    lengths = [int(x) for x in c["lengths"].split(",")] if c["lengths"] else [c["N_kv"]] * c["batch"]
    starts = [int(x) for x in c["starts"].split(",")] if c["starts"] else [n - c["N"] for n in lengths]
    return list(zip(starts, lengths))


def _pairs_of(c):
    """Visible (query, key) pairs of one head, summed over the sequences, and the keys that some query sees."""
    pairs = keys = 0
    for start, n in _sequences(c):
        lo, hi = max(0, start), min(n, start + c["N"])  # the positions that rows stand at
        if lo >= hi:
            continue
        p = torch.arange(lo, hi, dtype=torch.int64)
        last = torch.full_like(p, n - 1) if c["right"] < 0 else (p + c["right"]).clamp(max=n - 1)
        begin = torch.zeros_like(p) if c["left"] < 0 else (p - c["left"]).clamp(min=0)
        sink = (last + 1).clamp(max=min(c["sinks"], n))
        pairs += int((last + 1 - begin).sum() + torch.minimum(sink, begin).sum())
        keys += int(last[-1] + 1 - begin[0]) + min(int(sink[-1]), int(begin[0]))
    return pairs, keys


def _axes(c):
    return [int(x) for x in c["axes"].split(",")]


def _shape(c, heads, N):
    return (c["batch"], heads, N, c["d"]) if c["layout"] == "hnd" else (c["batch"], N, heads, c["d"])


def work(case):
    c = case
    if c["op"] in ("rope", "rope_grad"):
        n = c["batch"] * c["N"] * c["d"] * (c["heads"] + c["heads_kv"])
        given = 0 if c["grid"] else 4 * c["batch"] * c["N"] * len(_axes(c))
        return {"bytes": 2 * 2 * n + given, "flops": 3 * n}
    pairs, keys = _pairs_of(c)
    rows = c["batch"] * c["heads"] * c["N"]
    q, kv = 2 * rows * c["d"], 2 * keys * c["heads_kv"] * c["d"]
    if c["op"] == "forward":
        return {"bytes": 2 * q + 2 * kv + 4 * rows, "flops": 4 * c["d"] * pairs * c["heads"]}
    dkv = 2 * c["batch"] * c["N_kv"] * c["heads_kv"] * c["d"]
    return {"bytes": 4 * q + 4 * rows + 2 * kv + 2 * dkv, "flops": 10 * c["d"] * pairs * c["heads"]}


# ------------------------------------------------------------------ inputs
def _normal(gen, shape, dtype):
    out = torch.empty(shape, device="cuda", dtype=dtype)
    return out.normal_(0.0, 1.0, generator=gen)


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * int(seed) + 12345)
    dt = _DTYPES[c["dtype"]]
    s = {"case": c}
    if c["op"] in ("rope", "rope_grad"):
        s["Q"] = _normal(gen, _shape(c, c["heads"], c["N"]), dt)
        s["K"] = _normal(gen, _shape(c, c["heads_kv"], c["N"]), dt)
        s["positions"] = None
        if not c["grid"]:
            n = len(_axes(c))
            if n == 1:  # a text sequence that has come some way
                at = torch.randint(0, 100000, (c["batch"], 1), device="cuda", generator=gen)
                pos = (at + torch.arange(c["N"], device="cuda")).unsqueeze(-1)
            else:       # frames of a clip and text between them: a slow axis and fast ones
                slow = torch.sort(torch.randint(0, 100000, (c["batch"], c["N"], 1), device="cuda", generator=gen), 1).values
                pos = torch.cat([slow, torch.randint(0, 96, (c["batch"], c["N"], n - 1), device="cuda", generator=gen)], -1)
            s["positions"] = pos.to(torch.int32).contiguous()
        return s
    s["Q"] = _normal(gen, _shape(c, c["heads"], c["N"]), dt)
    s["K"] = _normal(gen, _shape(c, c["heads_kv"], c["N_kv"]), dt)
    s["V"] = _normal(gen, _shape(c, c["heads_kv"], c["N_kv"]), dt)
    s["starts"] = s["lengths"] = None
    if c["lengths"]:
        s["starts"] = torch.tensor([x[0] for x in _sequences(c)], dtype=torch.int32, device="cuda")
        s["lengths"] = torch.tensor([x[1] for x in _sequences(c)], dtype=torch.int32, device="cuda")
    if c["op"] == "backward":
        s["dO"] = _normal(gen, _shape(c, c["heads"], c["N"]), dt)
        s["O"], s["LSE"] = _plain_forward(c, s["Q"], s["K"], s["V"])
    return s


# ------------------------------------------------------------------ plain forms
def _by_head(c, x):
    return x if c["layout"] == "hnd" else x.transpose(1, 2)


def _as_laid_out(c, x, dtype):
    return (x if c["layout"] == "hnd" else x.transpose(1, 2)).to(dtype).contiguous()


def _angles(c, positions):
    """[batch or 1, N, rotated channels / 2] angles in 64 bits (far positions need them), and which tokens are rotated."""
    axes = _axes(c)
    total = sum(axes)
    axis = torch.tensor([a for a, n in enumerate(axes) for _ in range(n // 2)], device="cuda")
    if c["shared"]:
        e = torch.arange(total // 2, dtype=torch.float64, device="cuda") * 2.0 / total
    else:
        e = torch.cat([torch.arange(n // 2, dtype=torch.float64, device="cuda") * 2.0 / n for n in axes])
    freq = 10000.0 ** -e
    if positions is None:
        g = [int(x) for x in c["grid"].split("x")]
        t = torch.arange(c["N"], device="cuda") - c["first"]
        inside = (t >= 0) & (t < g[0] * g[1] * g[2])
        pos = torch.stack([t // (g[1] * g[2]), t // g[2] % g[1], t % g[2]], -1) * inside.unsqueeze(-1)
        positions = pos.unsqueeze(0)
    return positions[..., axis].double() * freq


def _plain_rope(c, x, positions):
    x = _by_head(c, x).float()
    a = _angles(c, positions).unsqueeze(1)
    cos, sin = a.cos().float(), a.sin().float()
    if c["op"] == "rope_grad":
        sin = -sin
    half = a.shape[-1]
    if c["pairs"] == "halves":
        u, v = x[..., :half], x[..., half:2 * half]
        turned = torch.cat([u * cos - v * sin, u * sin + v * cos], -1)
    else:
        u, v = x[..., 0:2 * half:2], x[..., 1:2 * half:2]
        turned = torch.stack([u * cos - v * sin, u * sin + v * cos], -1).flatten(-2)
    return _as_laid_out(c, torch.cat([turned, x[..., 2 * half:]], -1), _DTYPES[c["dtype"]])


def _rows_of(c):
    """Rows of one step of the plain form: as many as the window is long, so that at most half of the scores are hidden."""
    span = c["N_kv"] if c["left"] < 0 or c["right"] < 0 else min(c["N_kv"], max(512, c["left"] + c["right"]))
    return max(1, min(c["N"], span, _CHUNK // (c["batch"] * c["heads"] * min(c["N_kv"], 2 * span + c["sinks"]))))


def _steps(c):
    """(rows, their keys, what of rows x keys is visible): the keys are those that some row of the step may see."""
    seqs = _sequences(c)
    start = torch.tensor([x[0] for x in seqs], device="cuda").view(-1, 1, 1)
    length = torch.tensor([x[1] for x in seqs], device="cuda").view(-1, 1, 1)
    rows = _rows_of(c)
    for r0 in range(0, c["N"], rows):
        r1 = min(c["N"], r0 + rows)
        lo = 0 if c["left"] < 0 else max(0, min(x[0] for x in seqs) + r0 - c["left"])
        hi = c["N_kv"] if c["right"] < 0 else min(c["N_kv"], max(x[0] for x in seqs) + r1 + c["right"])
        lo = min(lo, max(hi, 0))
        sinks = min(c["sinks"], lo)
        keys = torch.cat([torch.arange(0, sinks, device="cuda"), torch.arange(lo, max(lo, hi), device="cuda")])
        p = start + torch.arange(r0, r1, device="cuda").view(1, -1, 1)
        sees = (keys < length) & (p >= 0) & (p < length)
        if c["right"] >= 0:
            sees &= keys <= p + c["right"]
        if c["left"] >= 0:
            sees &= (keys >= p - c["left"]) | (keys < c["sinks"])
        yield slice(r0, r1), keys, sees.view(c["batch"], 1, 1, r1 - r0, -1)


def _grouped(c, x, rows):
    """[batch, key heads, query heads of each, rows, d] in 32 bits."""
    return x[:, :, rows].float().unflatten(1, (c["heads_kv"], -1))


def _plain_forward(c, Q, K, V):
    Q, K, V = (_by_head(c, x) for x in (Q, K, V))
    O = torch.zeros(Q.shape, dtype=torch.float32, device="cuda")
    LSE = torch.full(Q.shape[:3], -math.inf, dtype=torch.float32, device="cuda")
    for rows, keys, sees in _steps(c):
        q, k, v = _grouped(c, Q, rows), K[:, :, keys].float().unsqueeze(2), V[:, :, keys].float().unsqueeze(2)
        s = (q / math.sqrt(c["d"])) @ k.transpose(-1, -2)
        s.masked_fill_(~sees, -math.inf)
        m = s.amax(-1, keepdim=True) if keys.numel() else torch.full_like(q[..., :1], -math.inf)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        e = s.sub_(m).exp_()
        total = e.sum(-1, keepdim=True)
        O[:, :, rows] = ((e @ v) / torch.where(total > 0, total, torch.ones_like(total))).flatten(1, 2)
        LSE[:, :, rows] = (m + total.log()).squeeze(-1).flatten(1, 2)
    return _as_laid_out(c, O, _DTYPES[c["dtype"]]), LSE


def _plain_backward(c, s):
    Q, K, V, O, dO = (_by_head(c, s[n]) for n in ("Q", "K", "V", "O", "dO"))
    dQ = torch.zeros(Q.shape, dtype=torch.float32, device="cuda")
    dK, dV = torch.zeros(K.shape, dtype=torch.float32, device="cuda"), torch.zeros(V.shape, dtype=torch.float32, device="cuda")
    scale = 1.0 / math.sqrt(c["d"])
    for rows, keys, sees in _steps(c):
        q, o, g = (_grouped(c, x, rows) for x in (Q, O, dO))
        k, v = K[:, :, keys].float().unsqueeze(2), V[:, :, keys].float().unsqueeze(2)
        lse = s["LSE"][:, :, rows].unflatten(1, (c["heads_kv"], -1)).unsqueeze(-1)
        p = (q * scale) @ k.transpose(-1, -2)
        p.sub_(lse).exp_().masked_fill_(~sees, 0.0)
        dV.index_add_(2, keys, (p.transpose(-1, -2) @ g).sum(2))
        ds = (g @ v.transpose(-1, -2)).sub_((g * o).sum(-1, keepdim=True)).mul_(p).mul_(scale)
        dQ[:, :, rows] = (ds @ k).flatten(1, 2)
        dK.index_add_(2, keys, (ds.transpose(-1, -2) @ q).sum(2))
    dt = _DTYPES[c["dtype"]]
    return tuple(_as_laid_out(c, x, dt) for x in (dQ, dK, dV))


# ------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    if own:
        from paper_2609_25869_b200 import bsa
        if c["op"] in ("rope", "rope_grad"):
            where = {"positions": s["positions"]} if s["positions"] is not None else {
                "grid": [int(x) for x in c["grid"].split("x")], "first": c["first"]}
            return bsa.rope(s["Q"], s["K"], axes=_axes(c), pairs=c["pairs"], shared_freq=c["shared"], layout=c["layout"],
                            inverse=c["op"] == "rope_grad", **where)
        window = {"left": c["left"], "right": c["right"], "sinks": c["sinks"], "q_start": s["starts"],
                  "kv_len": s["lengths"], "layout": c["layout"]}
        if c["op"] == "forward":
            return bsa.window_forward(s["Q"], s["K"], s["V"], **window)
        return bsa.window_backward(s["Q"], s["K"], s["V"], s["O"], s["LSE"], s["dO"], **window)
    if c["op"] in ("rope", "rope_grad"):
        return _plain_rope(c, s["Q"], s["positions"]), _plain_rope(c, s["K"], s["positions"])
    if c["op"] == "forward":
        return _plain_forward(c, s["Q"], s["K"], s["V"])
    return _plain_backward(c, s)


# ------------------------------------------------------------------ the definitions in 64 bits
def _exact_rope(c, s):
    axes = _axes(c)
    rate, axis = [], []
    for a, n in enumerate(axes):
        for i in range(n // 2):
            rate.append(10000.0 ** (-2.0 * len(rate) / sum(axes)) if c["shared"] else 10000.0 ** (-2.0 * i / n))
            axis.append(a)
    rate = torch.tensor(rate, dtype=torch.float64, device="cuda")
    if s["positions"] is not None:
        at = s["positions"].double()
    else:
        T, H, W = (int(x) for x in c["grid"].split("x"))
        at = torch.zeros((1, c["N"], 3), dtype=torch.float64, device="cuda")
        here = torch.cartesian_prod(*(torch.arange(n, dtype=torch.float64, device="cuda") for n in (T, H, W)))
        at[0, c["first"]:c["first"] + T * H * W] = here
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), at[:, :, axis] * rate)
    if c["op"] == "rope_grad":
        turn = turn.conj()
    turn = turn.unsqueeze(1 if c["layout"] == "hnd" else 2)
    outs = []
    for name in ("Q", "K"):
        x = s[name].double()
        n = 2 * len(axis)
        if c["pairs"] == "halves":
            z = torch.complex(x[..., :n // 2], x[..., n // 2:n]) * turn
            x[..., :n // 2], x[..., n // 2:n] = z.real, z.imag
        else:
            z = torch.view_as_complex(x[..., :n].unflatten(-1, (-1, 2)).contiguous()) * turn
            x[..., :n] = torch.view_as_real(z).flatten(-2)
        outs.append(x)
    return tuple(outs)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"] in ("rope", "rope_grad"):
        return _exact_rope(c, s)
    group, backward = c["heads"] // c["heads_kv"], c["op"] == "backward"
    put = (lambda x: x) if c["layout"] == "hnd" else (lambda x: x.permute(0, 2, 1, 3).contiguous())
    get = (lambda n, b, h: s[n][b, h]) if c["layout"] == "hnd" else (lambda n, b, h: s[n][b, :, h])
    new = lambda h, n: torch.zeros((c["batch"], h, n, c["d"]), dtype=torch.float64, device="cuda")  # noqa: E731
    out, grads = new(c["heads"], c["N"]), (new(c["heads"], c["N"]), new(c["heads_kv"], c["N_kv"]), new(c["heads_kv"], c["N_kv"]))
    lse = torch.full((c["batch"], c["heads"], c["N"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, (start, n) in enumerate(_sequences(c)):
        for r0 in range(0, c["N"], 2048):
            r1 = min(c["N"], r0 + 2048)
            p = torch.arange(start + r0, start + r1, device="cuda")
            p0, p1 = max(0, start + r0), min(n, start + r1)  # positions of the rows that see anything
            if p0 >= p1:
                continue
            first = 0 if c["left"] < 0 else max(0, p0 - c["left"])
            end = n if c["right"] < 0 else min(n, p1 + c["right"])
            j = torch.tensor(sorted(set(range(min(c["sinks"], end))) | set(range(first, end))), device="cuda")
            hidden = ((p < 0) | (p >= n))[:, None].expand(-1, j.numel())
            if c["right"] >= 0:
                hidden = hidden | (j[None] - p[:, None] > c["right"])
            if c["left"] >= 0:
                hidden = hidden | ((p[:, None] - j[None] > c["left"]) & (j >= c["sinks"])[None])
            for h in range(c["heads"]):
                q, k, v = get("Q", b, h)[r0:r1].double(), get("K", b, h // group)[j].double(), get("V", b, h // group)[j].double()
                score = torch.einsum("id,jd->ij", q, k) * c["d"] ** -0.5
                score[hidden] = -math.inf
                if not backward:
                    lse[b, h, r0:r1] = torch.logsumexp(score, 1)
                    out[b, h, r0:r1] = torch.einsum("ij,jd->id", torch.nan_to_num(torch.softmax(score, 1)), v)
                    continue
                o, g = get("O", b, h)[r0:r1].double(), get("dO", b, h)[r0:r1].double()
                weight = torch.exp(score - s["LSE"][b, h, r0:r1, None].double())
                weight[hidden] = 0.0
                grads[2][b, h // group].index_add_(0, j, torch.einsum("ij,id->jd", weight, g))
                slope = weight * (torch.einsum("id,jd->ij", g, v) - torch.einsum("id,id->i", g, o)[:, None]) * c["d"] ** -0.5
                grads[0][b, h, r0:r1] = torch.einsum("ij,jd->id", slope, k)
                grads[1][b, h // group].index_add_(0, j, torch.einsum("ij,id->jd", slope, q))
    return tuple(put(x) for x in grads) if backward else (put(out), lse)
