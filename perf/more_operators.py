"""A key/value cache held in 8 bits, with a scale for each block of tokens and head: what is measured of writing it, reading it back
and attending to it, and the plain forms.

A streamed clip or text keeps the keys and values of its past tokens.  In 16 bits they fill the memory and, for the next token, all of
the time; here an element is an e4m3 number and a block of tokens of one head shares a power of two (e8m0), so that half is kept and read.

Fields of a case
    op       "store"   new tokens are written behind those that the cache holds, and their blocks are read back
             "read"    a stretch of the cache in 16 bits, as another attention takes it
             "attend"  attention of some queries to a window of the cache and its first tokens: O and its LSE
    batch, heads_kv, N_kv, d, block, layout   the cache: [batch, heads_kv, N_kv, d] ("hnd") or [batch, N_kv, heads_kv, d] ("nhd"),
                                              scales [batch, heads_kv, N_kv / block]
    dtype                what is written, read back, asked and answered
    N, starts, counts    rows of the call: new tokens, tokens to read, queries; "a,b,...": position of each sequence's first row,
                         and how many of its N rows count (store, read) or how many keys it has (attend)
    heads, left, right, sinks   the query at position p sees the keys j <= p + right with j >= p - left or j < sinks; -1: no limit;
                                a row at no position of its sequence sees nothing
"""
from __future__ import annotations

import math

import torch

own = False

_DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
_CHUNK = 1 << 29          # score elements of one step of the plain form
_MAX_FLOPS = 6.0e12       # a drawn attention stays below the largest listed one,
_MAX_ELEMENTS = 1.2e8     # and what a drawn call writes or reads below that


def _store(name, heads_kv, N, N_kv, d, starts, counts, batch=1, op="store", block=64, dtype="bf16", layout="hnd"):
    c = {"op": op, "batch": batch, "heads_kv": heads_kv, "N": N, "N_kv": N_kv, "d": d, "block": block, "dtype": dtype,
         "layout": layout, "starts": starts, "counts": counts}
    return dict(c, name=name) if name else c


def _attend(name, heads, heads_kv, N, N_kv, d, left, starts, counts, right=0, sinks=0, batch=1, block=64, dtype="bf16", layout="hnd"):
    c = _store(name, heads_kv, N, N_kv, d, starts, counts, batch, "attend", block, dtype, layout)
    return dict(c, heads=heads, left=left, right=right, sinks=sinks)


def listed():
    return [
        # the next token of four short streams: latency is everything
        _store("store_token", 8, 1, 8192, 128, "8000,1500,300,5", "1,1,1,1", batch=4),
        # the next chunk of a streamed clip, three latent frames of 1560 tokens, token-major as the projection leaves it
        _store("store_chunk", 12, 4680, 32760, 128, "18720", "4680", layout="nhd"),
        # a padded batch of half tensors, small heads, short blocks, each sequence further on than the last
        _store("store_padded", 16, 1111, 3600, 64, "0,333,2050", "1111,700,65", batch=3, block=32, dtype="fp16", layout="nhd"),
        # the last fifteen latent frames in 16 bits, as a block-sparse plan's forward takes them
        _store("read_window", 12, 23400, 32760, 128, "9360", "23400", op="read"),
        # prompts of a padded batch read back
        _store("read_padded", 16, 3600, 8192, 64, "0,1000,77", "3600,2111,1025", batch=3, op="read", block=128, dtype="fp16", layout="nhd"),
        # the next token of four short streams: a window and four sinks out of a cache, latency is everything
        _attend("token_window", 32, 8, 1, 8192, 128, 1023, "8000,1500,300,5", "8001,1501,301,6", sinks=4, batch=4),
        # the next token over all of a long cache, sequences of very different length
        _attend("token_long", 32, 8, 1, 115200, 128, -1, "115199,90000,75599,32767,20001,1110", "115200,90001,75600,32768,20002,1111",
                batch=6, layout="nhd"),
        # five drafted tokens, half tensors, small heads, blocks of 16 tokens
        _attend("tokens_drafted", 16, 2, 5, 40000, 64, -1, "39990,20001,7", "39995,20006,12", batch=3, block=16, dtype="fp16"),
        # a short chunk against a long cache: 300 rows a head
        _attend("rows_long", 8, 8, 300, 65536, 128, -1, "65000", "65300", block=128),
        # the next chunk of a streamed clip against the cached frames of its window and the first frame
        _attend("chunk_window", 12, 12, 4680, 32760, 128, 18720, "28080", "32760", right=4679, sinks=1560),
        # a padded batch of half tensors over a cache just written, token-major, small heads
        _attend("chunk_padded", 16, 4, 3600, 3600, 64, 511, "0,0,0", "3600,2111,1025", right=63, sinks=64, batch=3, block=32, dtype="fp16",
                layout="nhd"),
        # the largest: a chunk against all that a 720p clip has cached
        _attend("chunk_clip", 24, 24, 4680, 115200, 128, -1, "110520", "115200", right=4679, layout="nhd"),
    ]


def _log(rng, lo, hi):
    return int(round(2.0 ** rng.uniform(math.log2(lo), math.log2(hi))))


def draw(rng):
    while True:
        op = rng.choice(["store", "store", "read", "attend", "attend", "attend", "attend"])
        d = rng.choice([64, 128])
        heads_kv = rng.choice([1, 2, 4, 8, 12, 16, 24])
        heads = heads_kv * rng.choice([1, 1, 1, 2, 4, 7, 8])
        batch = rng.choice([1, 1, 2, 3, 4])
        rest = {"batch": batch, "block": rng.choice([16, 32, 64, 64, 128]), "dtype": rng.choice(["bf16", "bf16", "fp16"]),
                "layout": rng.choice(["hnd", "nhd"])}
        if heads > 32:
            continue
        N_kv = _log(rng, 64, 115200)
        if op != "attend":
            N = min(N_kv, rng.choice([1, 1, 5, _log(rng, 1, 4680), _log(rng, 1, 32760)]))
            at = [rng.choice([0, rng.randint(0, N_kv - N), rng.randint(0, N_kv - 1)]) for _ in range(batch)]
            n = [min(N_kv - s, rng.choice([N, N, rng.randint(1, N)])) for s in at]
            if batch * heads_kv * N * d > _MAX_ELEMENTS or batch * heads_kv * N_kv * d > 1.0e9:
                continue
            return _store("", heads_kv, N, N_kv, d, ",".join(map(str, at)), ",".join(map(str, n)), op=op, **rest)
        right = rng.choice([0, 0, 0, 63, _log(rng, 1, 4680)])
        left = rng.choice([-1, -1, _log(rng, 1, 8192), _log(rng, 128, 32760)])
        sinks = rng.choice([0, 1, 4, 16, 100, _log(rng, 1, 1560)])
        N = min(N_kv, rng.choice([1, 1, 1, 2, 5, _log(rng, 1, 600), _log(rng, 1, 4680)]))
        n = [rng.choice([N_kv, max(N, _log(rng, max(1, N_kv // 32), N_kv))]) for _ in range(batch)]
        c = _attend("", heads, heads_kv, N, N_kv, d, left, ",".join(str(x - N) for x in n), ",".join(map(str, n)), right=right, sinks=sinks,
                    **rest)
        if work(c)["flops"] <= _MAX_FLOPS and batch * heads_kv * N_kv * d <= 4.0e8:
            return c


# ------------------------------------------------------------------ what a case stands for
def _rows(c):
    """(position of the first row, its rows that count or its keys) of every sequence."""
    return list(zip((int(x) for x in c["starts"].split(",")), (int(x) for x in c["counts"].split(","))))


def _touched(c):
    """(position of the first token read back, how many) of every sequence of a "store": its blocks up to the last new token."""
    return [(s // c["block"] * c["block"], s + n - s // c["block"] * c["block"]) for s, n in _rows(c)]


def work(case):
    c = case
    row = c["heads_kv"] * c["d"]
    blocks = lambda s, n: (s + n - 1) // c["block"] - s // c["block"] + 1  # noqa: E731
    if c["op"] == "store":
        new = sum(n for _, n in _rows(c))
        back = sum(n for _, n in _touched(c))
        scales = sum(blocks(s, n) for s, n in _rows(c)) * c["heads_kv"]
        return {"bytes": 2 * row * (3 * new + 3 * back) + 4 * scales, "flops": 4 * row * (new + back)}
    if c["op"] == "read":
        n = sum(n for _, n in _rows(c))
        return {"bytes": 2 * row * 3 * n + 2 * c["heads_kv"] * sum(blocks(s, n) for s, n in _rows(c)), "flops": 2 * row * n}
    pairs = keys = rows = 0
    for start, n in _rows(c):
        lo, hi = max(0, start), min(n, start + c["N"])
        rows += c["N"]
        if lo >= hi:
            continue
        p = torch.arange(lo, hi, dtype=torch.int64)
        last = torch.full_like(p, n - 1) if c["right"] < 0 else (p + c["right"]).clamp(max=n - 1)
        begin = torch.zeros_like(p) if c["left"] < 0 else (p - c["left"]).clamp(min=0)
        sink = (last + 1).clamp(max=min(c["sinks"], n))
        pairs += int((last + 1 - begin).sum() + torch.minimum(sink, begin).sum())
        keys += int(last[-1] + 1 - begin[0]) + min(int(sink[-1]), int(begin[0]))
    return {"bytes": rows * c["heads"] * (4 * c["d"] + 4) + 2 * keys * c["heads_kv"] * c["d"] + 2 * keys * c["heads_kv"] // c["block"],
            "flops": 4 * c["d"] * pairs * c["heads"]}


# ------------------------------------------------------------------ inputs
def _shape(c, heads, N):
    return (c["batch"], heads, N, c["d"]) if c["layout"] == "hnd" else (c["batch"], N, heads, c["d"])


def _by_head(c, x):
    return x if c["layout"] == "hnd" else x.transpose(1, 2)


def _tokens(gen, c, N):
    """Keys or values of N tokens: normal, some tokens and heads louder than others."""
    x = torch.empty(_shape(c, c["heads_kv"], N), device="cuda", dtype=_DTYPES[c["dtype"]]).normal_(0.0, 1.0, generator=gen)
    loud = torch.empty((c["batch"], c["heads_kv"], N, 1), device="cuda").normal_(0.0, 0.3, generator=gen).exp_()
    return x.mul_(loud if c["layout"] == "hnd" else loud.transpose(1, 2))


def prepare(case, seed):
    c = case
    gen = torch.Generator(device="cuda")
    gen.manual_seed(1000003 * int(seed) + 54321)
    s = {"case": c, "starts": torch.tensor([x[0] for x in _rows(c)], dtype=torch.int32, device="cuda"),
         "counts": torch.tensor([x[1] for x in _rows(c)], dtype=torch.int32, device="cuda")}
    # the cache: written from its beginning
    blocks = -(-c["N_kv"] // c["block"])
    for name in ("K", "V"):
        s[name + "8"] = torch.zeros(_shape(c, c["heads_kv"], c["N_kv"]), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
        s[name + "_scale"] = torch.zeros((c["batch"], c["heads_kv"], blocks), dtype=torch.uint8, device="cuda").view(torch.float8_e8m0fnu)
        _plain_write(c, _tokens(gen, c, c["N_kv"]), s[name + "8"], s[name + "_scale"], torch.zeros_like(s["starts"]),
                     torch.full_like(s["counts"], c["N_kv"]))
    if c["op"] == "attend":
        s["Q"] = torch.empty(_shape(c, c["heads"], c["N"]), device="cuda", dtype=_DTYPES[c["dtype"]]).normal_(0.0, 1.0, generator=gen)
    if c["op"] == "store":
        s["K"], s["V"] = _tokens(gen, c, c["N"]), _tokens(gen, c, c["N"])
        s["first"] = torch.tensor([x[0] for x in _touched(c)], dtype=torch.int32, device="cuda")
        s["held"] = torch.tensor([x[1] for x in _touched(c)], dtype=torch.int32, device="cuda")
    return s


# ------------------------------------------------------------------ plain forms
def _power(code):
    """2^(code - 127) in 32 bits, NaN for 255."""
    code = code.to(torch.int32)
    bits = torch.where(code > 0, code << 23, torch.full_like(code, 1 << 22))
    return torch.where(code == 255, torch.full_like(bits, 0x7fc00000), bits).view(torch.float32)


def _scale_code(most):
    """The smallest power of two, as its code, that takes `most` (finite, in 32 bits) to at most 448."""
    bits = most.view(torch.int32)
    above = (bits & 0x7fffff) > 0x600000  # 448 = 1.75 * 2^8
    return ((bits >> 23) - 8 + above.to(torch.int32)).clamp(min=0)


def _plain_write(c, x, cache, scales, start, count):
    B, h, d = c["block"], c["heads_kv"], c["d"]
    x, codes, scale = _by_head(c, x).float(), _by_head(c, cache.view(torch.uint8)), scales.view(torch.uint8)
    N = x.shape[2]
    nb = (N + B - 2) // B + 1
    start, count = start.long().view(-1, 1), count.long().view(-1, 1)
    block = start // B + torch.arange(nb, device="cuda")                                # [batch, nb]
    at = (block.unsqueeze(-1) * B + torch.arange(B, device="cuda")).flatten(1)          # [batch, nb * B]
    new = (at >= start) & (at < start + count) & (at < c["N_kv"])
    kept = (at < start) & (at >= 0)
    live = (block * B < start + count) & (block * B < c["N_kv"])                        # blocks that get a token
    who = torch.arange(c["batch"], device="cuda").view(-1, 1)
    value = x.transpose(1, 2)[who, (at - start).clamp(0, N - 1)].transpose(1, 2) * new[:, None, :, None]
    most = value.abs().amax(-1).unflatten(2, (nb, B)).amax(-1)                          # [batch, h, nb]
    code = _scale_code(most)
    old = scale.transpose(1, 2)[who, block.clamp(0, scale.shape[2] - 1)].transpose(1, 2).to(torch.int32)
    code = torch.where(kept.unflatten(1, (nb, B)).any(-1).unsqueeze(1), torch.maximum(old, code), code)
    wide = lambda v: v.repeat_interleave(B, 2).unsqueeze(-1)  # noqa: E731
    value = value * _power(254 - wide(code))
    stored = codes.transpose(1, 2)[who, at.clamp(0, c["N_kv"] - 1)].transpose(1, 2).view(torch.float8_e4m3fn).float()
    value = torch.where(new[:, None, :, None], value, stored * _power((wide(old) - wide(code) + 127).clamp(min=0)))
    value = value.to(torch.float8_e4m3fn).view(torch.uint8)
    touch = (new | (kept & live.repeat_interleave(B, 1))).unsqueeze(1).expand(-1, h, -1)
    b, hh, i = touch.nonzero(as_tuple=True)
    codes[b, hh, at[b, i]] = value[b, hh, i]
    b, hh, i = live.unsqueeze(1).expand(-1, h, -1).nonzero(as_tuple=True)
    scale[b, hh, block[b, i]] = code[b, hh, i].to(torch.uint8)


def _plain_values(c, cache, scales, first, N):
    """[batch, heads, N, d] in 32 bits: the cache's values from each sequence's position `first` on."""
    at = (first.long().view(-1, 1) + torch.arange(N, device="cuda")).clamp(0, c["N_kv"] - 1)
    who = torch.arange(c["batch"], device="cuda").view(-1, 1)
    value = _by_head(c, cache.view(torch.uint8)).transpose(1, 2)[who, at].transpose(1, 2).view(torch.float8_e4m3fn).float()
    return value * _power(scales.view(torch.uint8).transpose(1, 2)[who, at // c["block"]].transpose(1, 2)).unsqueeze(-1)


def _plain_read(c, cache, scales, first, count, N):
    value = _plain_values(c, cache, scales, first, N)
    i = torch.arange(N, device="cuda")
    there = (i < count.view(-1, 1)) & (first.view(-1, 1) + i < c["N_kv"])
    value = torch.where(there[:, None, :, None], value, torch.zeros_like(value))
    return (value if c["layout"] == "hnd" else value.transpose(1, 2)).to(_DTYPES[c["dtype"]]).contiguous()


def _step_rows(c):
    """Rows of one step: as many as the window is long, so that at most half of the scores are hidden."""
    span = c["N_kv"] if c["left"] < 0 or c["right"] < 0 else min(c["N_kv"], max(512, c["left"] + c["right"]))
    return max(1, min(c["N"], span, _CHUNK // (c["batch"] * c["heads"] * min(c["N_kv"], 2 * span + c["sinks"]))))


def _plain_attend(c, s):
    seqs = _rows(c)
    start, length = s["starts"].view(-1, 1, 1), s["counts"].view(-1, 1, 1)
    origin = torch.zeros_like(s["starts"])
    K, V = (_plain_values(c, s[n + "8"], s[n + "_scale"], origin, c["N_kv"]) for n in ("K", "V"))
    Q = _by_head(c, s["Q"])
    O = torch.zeros(Q.shape, dtype=torch.float32, device="cuda")
    LSE = torch.full(Q.shape[:3], -math.inf, dtype=torch.float32, device="cuda")
    rows = _step_rows(c)
    for r0 in range(0, c["N"], rows):
        r1 = min(c["N"], r0 + rows)
        lo = 0 if c["left"] < 0 else max(0, min(x[0] for x in seqs) + r0 - c["left"])
        hi = c["N_kv"] if c["right"] < 0 else min(c["N_kv"], max(x[0] for x in seqs) + r1 + c["right"])
        lo = min(lo, max(hi, 0))
        keys = torch.cat([torch.arange(0, min(c["sinks"], lo), device="cuda"), torch.arange(lo, max(lo, hi), device="cuda")])
        p = start + torch.arange(r0, r1, device="cuda").view(1, -1, 1)
        sees = (keys < length) & (p >= 0) & (p < length)
        if c["right"] >= 0:
            sees &= keys <= p + c["right"]
        if c["left"] >= 0:
            sees &= (keys >= p - c["left"]) | (keys < c["sinks"])
        q = Q[:, :, r0:r1].float().unflatten(1, (c["heads_kv"], -1)) / math.sqrt(c["d"])
        score = q @ K[:, :, keys].unsqueeze(2).transpose(-1, -2)
        score.masked_fill_(~sees.view(c["batch"], 1, 1, r1 - r0, -1), -math.inf)
        m = score.amax(-1, keepdim=True) if keys.numel() else torch.full_like(q[..., :1], -math.inf)
        m = torch.where(m == -math.inf, torch.zeros_like(m), m)
        e = score.sub_(m).exp_()
        total = e.sum(-1, keepdim=True)
        O[:, :, r0:r1] = ((e @ V[:, :, keys].unsqueeze(2)) / torch.where(total > 0, total, torch.ones_like(total))).flatten(1, 2)
        LSE[:, :, r0:r1] = (m + total.log()).squeeze(-1).flatten(1, 2)
    return (O if c["layout"] == "hnd" else O.transpose(1, 2)).to(_DTYPES[c["dtype"]]).contiguous(), LSE


# ------------------------------------------------------------------ one pass
def run(state):
    s, c = state, state["case"]
    back = c["N"] + c["block"] - 1  # rows that hold every block a "store" touches
    if own:
        from paper_2609_25869_b200 import bsa
        if "cache" not in s:  # the handle that a program keeps beside the tensors
            s["cache"] = bsa.Cache(s["K8"], s["V8"], s["K_scale"], s["V_scale"], block=c["block"], layout=c["layout"])
        if c["op"] == "store":
            bsa.cache_write(s["cache"], s["K"], s["V"], start=s["starts"], count=s["counts"])
            return bsa.cache_read(s["cache"], back, start=s["first"], count=s["held"], dtype=_DTYPES[c["dtype"]])
        if c["op"] == "read":
            return bsa.cache_read(s["cache"], c["N"], start=s["starts"], count=s["counts"], dtype=_DTYPES[c["dtype"]])
        return bsa.cache_forward(s["Q"], s["cache"], left=c["left"], right=c["right"], sinks=c["sinks"], q_start=s["starts"],
                                 kv_len=s["counts"])
    if c["op"] == "attend":
        return _plain_attend(c, s)
    if c["op"] == "store":
        for name in ("K", "V"):
            _plain_write(c, s[name], s[name + "8"], s[name + "_scale"], s["starts"], s["counts"])
        return tuple(_plain_read(c, s[n + "8"], s[n + "_scale"], s["first"], s["held"], back) for n in ("K", "V"))
    return tuple(_plain_read(c, s[n + "8"], s[n + "_scale"], s["starts"], s["counts"], c["N"]) for n in ("K", "V"))


# ------------------------------------------------------------------ the definitions in 64 bits
def _two_to(e):
    """2^e of whole numbers in 64 bits, from its bits (a pow() that is off by its last one would turn ties)."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def _numbers(cache, scales, block, head_axis):
    """All that a cache holds, [batch, heads, N_kv, d] in 64 bits."""
    e = scales.view(torch.uint8).long() - 127
    step = _two_to(e)
    x = cache.double()
    x = x if head_axis == 1 else x.permute(0, 2, 1, 3)
    return x * step.repeat_interleave(block, 2)[:, :, :x.shape[2], None]


def _nearest_e4m3(x):
    """The nearest number with four significant bits, exponents from -6 and subnormals of 2^-9; ties to the even one."""
    _, e = torch.frexp(x.abs())
    step = _two_to((e - 4).clamp(min=-9))
    return torch.round(x / step) * step


def exact(case, seed):
    c, s = case, prepare(case, seed)
    axis = 1 if c["layout"] == "hnd" else 2
    held = [_numbers(s[n + "8"], s[n + "_scale"], c["block"], axis) for n in ("K", "V")]
    lay = lambda x: x if axis == 1 else x.permute(0, 2, 1, 3).contiguous()  # noqa: E731
    if c["op"] != "attend":
        out = []
        steps = torch.tensor([448.0 * 2.0 ** e for e in range(-127, 121)], dtype=torch.float64, device="cuda")
        for name, now in zip(("K", "V"), held):
            N = c["N"] if c["op"] == "read" else c["N"] + c["block"] - 1
            y = torch.zeros((c["batch"], c["heads_kv"], N, c["d"]), dtype=torch.float64, device="cuda")
            for b, (start, n) in enumerate(_rows(c)):
                if c["op"] == "read":
                    y[b, :, :n] = now[b, :, start:start + n]
                    continue
                fresh = (s[name][b] if axis == 1 else s[name][b].transpose(0, 1)).double()
                e_old = s[name + "_scale"].view(torch.uint8)[b].long() - 127
                base = start // c["block"] * c["block"]
                for lo in range(base, start + n, c["block"]):
                    hi = min(lo + c["block"], start + n)
                    a = max(lo, start)
                    new = fresh[:, a - start:hi - start]
                    most = new.abs().amax((1, 2))
                    e = torch.searchsorted(steps, most) - 127  # the first that is large enough
                    if a > lo:
                        e = torch.maximum(e, e_old[:, lo // c["block"]])
                    both = torch.cat([now[b, :, lo:a], new], 1)
                    unit = _two_to(e).view(-1, 1, 1)
                    y[b, :, lo - base:hi - base] = _nearest_e4m3(both / unit) * unit
            out.append(lay(y))
        return tuple(out)
    group = c["heads"] // c["heads_kv"]
    O = torch.zeros((c["batch"], c["heads"], c["N"], c["d"]), dtype=torch.float64, device="cuda")
    LSE = torch.full((c["batch"], c["heads"], c["N"]), -math.inf, dtype=torch.float64, device="cuda")
    for b, (start, n) in enumerate(_rows(c)):
        for r0 in range(0, c["N"], 1024):
            r1 = min(c["N"], r0 + 1024)
            p0, p1 = max(0, start + r0), min(n, start + r1)
            if p0 >= p1:
                continue
            p = torch.arange(start + r0, start + r1, device="cuda")
            first = 0 if c["left"] < 0 else max(0, p0 - c["left"])
            end = n if c["right"] < 0 else min(n, p1 + c["right"])
            every = torch.arange(0, end, device="cuda")
            j = every[(every < c["sinks"]) | (every >= first)]
            hidden = ((p < 0) | (p >= n))[:, None].expand(-1, j.numel())
            if c["right"] >= 0:
                hidden = hidden | (j[None] - p[:, None] > c["right"])
            if c["left"] >= 0:
                hidden = hidden | ((p[:, None] - j[None] > c["left"]) & (j >= c["sinks"])[None])
            for h in range(c["heads"]):
                q = (s["Q"][b, h] if axis == 1 else s["Q"][b, :, h])[r0:r1].double()
                score = torch.einsum("id,jd->ij", q, held[0][b, h // group][j]) * c["d"] ** -0.5
                score[hidden] = -math.inf
                LSE[b, h, r0:r1] = torch.logsumexp(score, 1)
                O[b, h, r0:r1] = torch.einsum("ij,jd->id", torch.nan_to_num(torch.softmax(score, 1)), held[1][b, h // group][j])
    return lay(O), LSE
