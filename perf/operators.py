"""Attention over a paged key/value cache, and the cache's quantised write and read-back.

What is measured: the calls that a program makes after (or instead of) a
compression pass - keeping the rows in pages of bf16, 8-bit or 4-bit codes and
attending to them with single tokens (an answer being written) and with chunks
(a question, new frames). `run` makes them through the package where `own` is
true, and in plain torch operations where it is not.
"""
import math

import numpy as np
import torch

own = False

GROUP = 64                       # channels that share a step and a minimum
LEVELS = {"u8": 255, "u4": 15}
LARGEST = 32768.0                # a group with a larger magnitude is marked


# ------------------------------------------------------------------- the cases
def listed():
    """Sizes are this repository's: 4 or 8 KV heads of 128 channels, frames of 196 or 256 tokens, caches cut
    to 6272, 12288 or 24576 rows; 7 or 8 query heads for each KV head."""
    return [
        # The answer's tokens of 8 streams, one each, quantised as they are written, all layers' heads in one call.
        dict(name="write 8 tokens u4", op="write", fmt="u4", seqs=8, rows=1, kv=6273, ragged=1, heads=112, dim=128, page=64),
        # 16 new frames of one layer (1 fps video, one accumulate step).
        dict(name="write 16 frames u8", op="write", fmt="u8", seqs=1, rows=3136, kv=9408, ragged=0, heads=4, dim=128, page=64),
        # A whole compacted cache (28 layers x 4 heads) moved into 4-bit pages.
        dict(name="write compacted u4", op="write", fmt="u4", seqs=1, rows=6272, kv=6272, ragged=0, heads=112, dim=128, page=128),
        # One layer read back for a consumer that wants bf16 rows.
        dict(name="read layer u8", op="read", fmt="u8", seqs=1, rows=6272, kv=6272, ragged=0, heads=4, dim=128, page=64),
        # 8 streams' caches of one layer, ragged, read back.
        dict(name="read 8 streams u4", op="read", fmt="u4", seqs=8, rows=24576, kv=24576, ragged=1, heads=8, dim=128, page=32),
        # One token of one stream over its compacted cache: latency counts.
        dict(name="token bf16 6272", op="attend", fmt="bf16", seqs=1, rows=1, kv=6272, ragged=0, heads=4, share=7, dim=128, page=64,
             window=0, sinks=0, lse=1),
        # 8 streams' tokens over their 24576-row caches.
        dict(name="token bf16 8x24576", op="attend", fmt="bf16", seqs=8, rows=1, kv=24576, ragged=0, heads=8, share=8, dim=128, page=64,
             window=0, sinks=0, lse=0),
        # The same at 4 bits, the streams at different lengths.
        dict(name="token u4 32 ragged", op="attend", fmt="u4", seqs=32, rows=1, kv=24577, ragged=1, heads=8, share=8, dim=128, page=32,
             window=0, sinks=0, lse=0),
        # Questions of up to 61 tokens, 8-bit caches of different lengths.
        dict(name="question u8 8 ragged", op="attend", fmt="u8", seqs=8, rows=61, kv=12349, ragged=1, heads=4, share=7, dim=128, page=64,
             window=0, sinks=0, lse=0),
        # One new frame over the compacted cache.
        dict(name="frame bf16 6468", op="attend", fmt="bf16", seqs=1, rows=196, kv=6468, ragged=0, heads=4, share=7, dim=128, page=64,
             window=0, sinks=0, lse=0),
        # 16 new frames over the compacted cache, up to the cap.
        dict(name="16 frames bf16 9408", op="attend", fmt="bf16", seqs=1, rows=3136, kv=9408, ragged=0, heads=4, share=7, dim=128, page=64,
             window=0, sinks=0, lse=0),
        # A long text prompt under a window with 4 first tokens kept, narrow heads, nothing cached before it.
        dict(name="prompt window 8191", op="attend", fmt="bf16", seqs=1, rows=8191, kv=8191, ragged=0, heads=4, share=4, dim=64, page=16,
             window=2000, sinks=4, lse=0),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    while True:
        op = rng.choice(["write", "read", "attend", "attend", "attend", "attend"])
        fmt = rng.choice(["bf16", "u8", "u4"]) if op == "attend" else rng.choice(["u8", "u4"])
        c = dict(op=op, fmt=fmt, heads=rng.choice([1, 2, 4, 8]), dim=rng.choice([64, 128, 128, 80, 96] if fmt == "bf16" else [64, 128, 128]),
                 page=rng.choice([16, 32, 64, 128, 256]), ragged=rng.randint(0, 1))
        if op != "attend":
            c.update(seqs=_log(rng, 1, 32), rows=_log(rng, 1, 8192), heads=rng.choice([1, 4, 8, 28, 112]))
            c["kv"] = c["rows"] if op == "read" else c["rows"] + _log(rng, 1, 2048)
            if c["seqs"] * c["rows"] * c["heads"] > 6272 * 112:
                continue
        else:
            c["share"] = rng.choice([1, 2, 3, 4, 5, 6, 7, 8])
            c["lse"] = 0
            if rng.random() < 0.5:                       # single tokens
                c.update(seqs=_log(rng, 1, 64), rows=1, kv=_log(rng, 1, 32768))
            else:                                        # chunks
                c.update(seqs=_log(rng, 1, 8), rows=_log(rng, 2, 4096))
                c["kv"] = c["rows"] + _log(rng, 1, 16384)
            masked = rng.random() < 0.3
            c.update(window=_log(rng, 16, 4096) if masked else 0, sinks=rng.randint(0, 32) if masked else 0)
        if c["seqs"] * c["kv"] * c["heads"] > 8 * 24576 * 8:
            continue
        w = work(c)
        if w["bytes"] <= 0.81e9 and w["flops"] <= 3.5e11 and c["seqs"] * c["rows"] * c["kv"] * c["heads"] * c.get("share", 0) <= 1.1e9:
            return c


def _lengths(case):
    """(new rows, cached rows with them) of each sequence: the case's own where it is not ragged, else spread below it,
    the first sequence's the full ones."""
    rows, kv = [], []
    for b in range(case["seqs"]):
        f = 1.0 - 0.85 * ((b * 0.6180339887498949) % 1.0) if case["ragged"] else 1.0
        n = max(1, int(case["rows"] * f))
        rows.append(n)
        kv.append(n if case["rows"] == case["kv"] else max(n, int(case["kv"] * f)))
    return rows, kv


def _row_bytes(case):
    if case["fmt"] == "bf16":
        return 2 * case["dim"]
    return case["dim"] // (1 if case["fmt"] == "u8" else 2) + 4 * (case["dim"] // GROUP)


def work(case):
    rows, kv = _lengths(case)
    d, h = case["dim"], case["heads"]
    if case["op"] != "attend":
        n = sum(rows) * h * 2
        wide, held = n * d * 2, n * _row_bytes(case)
        # written and read back, or read: each value in, its code out, and the other way
        return {"bytes": 2 * (wide + held) if case["op"] == "write" else wide + held, "flops": 4 * n * d}
    pairs = seen = 0
    for n, length in zip(rows, kv):
        p = np.arange(length - n, length, dtype=np.int64)          # positions of the new tokens
        lo = np.maximum(0, p - case["window"] + 1) if case["window"] else np.zeros_like(p)
        pairs += int((p + 1 - lo + np.minimum(lo, case["sinks"])).sum())
        seen += int(length - lo[0] + min(lo[0], case["sinks"]))
    q_heads = h * case["share"]
    return {"bytes": seen * h * 2 * _row_bytes(case) + sum(rows) * q_heads * d * 4, "flops": 4 * d * q_heads * pairs}


# ------------------------------------------------------------- the packed format
def _f16_toward(x, up):
    """x (float32) as float16, rounded up or down; x lies within float16's range."""
    h = x.to(torch.float16)
    off = (h.float() < x) if up else (h.float() > x)
    bits = h.view(torch.int16).to(torch.int32) & 0xFFFF
    negative = bits >= 0x8000
    away = torch.where(negative, -1, 1) if up else torch.where(negative, 1, -1)  # toward +inf / -inf in bit patterns
    moved = bits + away
    zero = (bits & 0x7FFF) == 0
    moved = torch.where(zero, torch.full_like(bits, 0x0001 if up else 0x8001), moved)
    bits = torch.where(off, moved, bits)
    return torch.where(bits >= 0x8000, bits - 0x10000, bits).to(torch.int16).view(torch.float16)


def _quantise(x, fmt):
    """x [..., dim] -> (codes uint8 [..., groups, 64], step and minimum float16 [..., groups, 2])."""
    levels = LEVELS[fmt]
    g = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1), g.amax(-1)
    good = torch.isfinite(g).all(-1) & (torch.maximum(lo.abs(), hi.abs()) <= LARGEST)
    lo, hi = torch.where(good, lo, 0.0), torch.where(good, hi, 0.0)
    low = _f16_toward(lo, False)
    step = _f16_toward((hi - low.float()) / torch.full_like(hi, levels), True)  # by a tensor: a scalar's reciprocal rounds twice
    s, m = step.float()[..., None], low.float()[..., None]
    u = torch.where((s > 0) & good[..., None], torch.round((g - m) / torch.where(s > 0, s, 1.0)), 0.0)
    nan = torch.full_like(step, float("nan"))
    par = torch.stack([torch.where(good, step, nan), torch.where(good, low, nan)], -1)
    return u.nan_to_num(0.0).clamp(0, levels).to(torch.uint8), par


def _pack(u, fmt):
    """Codes [..., groups, 64] -> bytes [..., dim or dim/2]. A group's 4-byte words hold 4 (u8) or 8 (u4, low nibble
    first) neighbouring channels each; word t + 4 w of the group is stored in place t * (words / 4) + w."""
    if fmt == "u4":
        u = u[..., 0::2] | (u[..., 1::2] << 4)
    w = u.unflatten(-1, (-1, 4, 4))                      # [..., w, t, byte]
    return w.transpose(-3, -2).flatten(-4)               # [..., groups * t * w * byte]


def _unpack(b, fmt, dim):
    w = b.unflatten(-1, (dim // GROUP, 4, -1, 4)).transpose(-3, -2).flatten(-3)
    if fmt == "u8":
        return w
    return torch.stack([w & 15, w >> 4], -1).flatten(-2)


# ------------------------------------------------------------------- the inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed & 0x7FFFFFFFFFFF)


def _rows_like_keys(shape, gen, dev):
    """Keys as a decoder's: unit rows with a few wide channels that have an offset."""
    x = torch.randn(shape, generator=gen, device=dev, dtype=torch.bfloat16)
    dim = shape[-1]
    wide = torch.randint(0, dim, (max(1, dim // 32),), generator=gen, device=dev)
    gain = torch.ones(dim, device=dev)
    gain[wide] = 4.0
    shift = torch.zeros(dim, device=dev)
    shift[wide] = torch.randn(wide.shape, generator=gen, device=dev) * 3.0
    return x.mul_(gain.to(x.dtype)).add_(shift.to(x.dtype))


def _rows_like_values(shape, gen, dev):
    """Values: Gaussian directions with lognormal magnitudes."""
    x = torch.randn(shape, generator=gen, device=dev, dtype=torch.bfloat16)
    size = torch.randn(shape[:-1] + (1,), generator=gen, device=dev).mul_(0.5).exp_()
    return x.mul_(size.to(x.dtype))


def prepare(case, seed):
    dev, gen = "cuda", _generator(seed)
    rows, kv = _lengths(case)
    seqs, heads, dim, page, fmt = case["seqs"], case["heads"], case["dim"], case["page"], case["fmt"]
    wide = -(-max(kv) // page)
    need = sum(-(-n // page) for n in kv)
    pages = need + 3
    s = dict(case=case, rows=rows, kv=kv, wide=wide)
    s["max_rows"], s["max_kv"], s["total"] = max(rows), max(kv), sum(rows)
    s["row_start"] = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device=dev)
    s["kv_len"] = torch.tensor(kv, dtype=torch.int32, device=dev)
    order = torch.randperm(pages, generator=gen, device=dev).to(torch.int32)   # pages are handed out in no order
    table = torch.full((seqs, wide), -1, dtype=torch.int32, device=dev)        # entries past a sequence's end are never read
    at = 0
    for b, n in enumerate(kv):
        k = -(-n // page)
        table[b, :k] = order[at:at + k]
        at += k
    s["table"] = table
    shape = (pages, heads, page, dim)
    if case["op"] == "write":
        s["k_new"] = _rows_like_keys((s["total"], heads, dim), gen, dev)
        s["v_new"] = _rows_like_values((s["total"], heads, dim), gen, dev)
    for name, make in (("k", _rows_like_keys), ("v", _rows_like_values)):
        if fmt == "bf16":
            s[name], s[name + "_par"] = make(shape, gen, dev), None
        elif case["op"] == "write":
            s[name] = torch.zeros(shape[:-1] + (dim // (1 if fmt == "u8" else 2),), dtype=torch.uint8, device=dev)
            s[name + "_par"] = torch.zeros(shape[:-1] + (dim // GROUP, 2), dtype=torch.float16, device=dev)
        else:
            codes = torch.empty(shape[:-1] + (dim // (1 if fmt == "u8" else 2),), dtype=torch.uint8, device=dev)
            par = torch.empty(shape[:-1] + (dim // GROUP, 2), dtype=torch.float16, device=dev)
            part = max(1, (1 << 26) // (heads * page * dim))
            for i in range(0, pages, part):
                n = min(part, pages - i)
                u, p = _quantise(make((n,) + shape[1:], gen, dev), fmt)
                codes[i:i + n], par[i:i + n] = _pack(u, fmt), p
            s[name], s[name + "_par"] = codes, par
        if case["op"] != "write":                                              # a pool's unused rows hold anything
            rest = s[name] if fmt == "bf16" else s[name + "_par"]
            rest[order[at:].long()] = float("nan")
            for b, n in enumerate(kv):
                if n % page:
                    rest[table[b, n // page].long(), :, n % page:] = float("nan")
    if case["op"] == "attend":
        q_heads = heads * case["share"]
        s["q"] = torch.randn((s["total"], q_heads, dim), generator=gen, device=dev, dtype=torch.bfloat16) * 1.5
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((s["total"], q_heads), dtype=torch.float32, device=dev) if case["lse"] else None
        s["scale"] = dim ** -0.5
    else:
        s["k_out"] = torch.empty((s["total"], heads, dim), dtype=torch.bfloat16, device=dev)
        s["v_out"] = torch.empty_like(s["k_out"])
    return s


# --------------------------------------------------------------------- the passes
def _run_own(s):
    from paper_2506_15745_gb300.paged import PagedCache, PagedBatch

    case = s["case"]
    if "cache" not in s:  # the handles a program keeps
        s["cache"] = PagedCache.from_tensors(case["fmt"], s["k"], s["v"], s["k_par"], s["v_par"])
        s["batch"] = PagedBatch(s["table"], s["row_start"], s["kv_len"], total_rows=s["total"], max_rows=s["max_rows"],
                                max_kv=s["max_kv"])
    cache, batch = s["cache"], s["batch"]
    if case["op"] == "attend":
        cache.attend(s["q"], batch, out=s["out"], lse=s["lse"], scale=s["scale"], window=case["window"], sinks=case["sinks"])
        return [s["out"]] if s["lse"] is None else [s["out"], s["lse"]]
    if case["op"] == "write":
        cache.write(s["k_new"], s["v_new"], batch)
    cache.read(batch, s["k_out"], s["v_out"])
    return [s["k_out"], s["v_out"]]


def _places(s):
    """(page, row in it) of every new row, packed: int64 [total] each; and each new row's sequence."""
    n = (s["row_start"][1:] - s["row_start"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(len(s["rows"]), device="cuda"), n, output_size=s["total"])
    i = torch.arange(s["total"], device="cuda") - s["row_start"].long()[seq]
    at = s["kv_len"].long()[seq] - n[seq] + i
    page = s["case"]["page"]
    return s["table"].long()[seq, at // page], at % page, seq, i, at


def _values(codes, par, fmt, dim):
    """Codes [..., bytes] and parameters [..., groups, 2] -> float32 [..., dim]."""
    u = _unpack(codes, fmt, dim).float()
    return (u * par[..., 0:1].float() + par[..., 1:2].float()).flatten(-2)


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    fmt, dim, heads, page = case["fmt"], case["dim"], case["heads"], case["page"]
    pid, row, seq, i, at = _places(s)
    if case["op"] != "attend":
        out = []
        for name in ("k", "v"):
            if case["op"] == "write":
                u, par = _quantise(s[name + "_new"], fmt)
                s[name][pid, :, row] = _pack(u, fmt)
                s[name + "_par"][pid, :, row] = par
            out.append(_values(s[name][pid, :, row], s[name + "_par"][pid, :, row], fmt, dim).to(torch.bfloat16))
        return out

    seqs, share, wide = case["seqs"], case["share"], s["wide"]
    length = s["kv_len"].long()
    j = torch.arange(wide * page, device="cuda")
    inside = j < length[:, None]                                               # [seqs, keys]
    table = s["table"].long().clamp(min=0)

    def gather(name):
        x = s[name][table]                                                     # [seqs, wide, heads, page, ...]
        x = _values(x, s[name + "_par"][table], fmt, dim) if fmt != "bf16" else x.float()
        x = x.transpose(1, 2).reshape(seqs, heads, wide * page, dim)
        return torch.where(inside[:, None, :, None], x, 0.0)

    q = torch.zeros((seqs, s["max_rows"], heads * share, dim), device="cuda")  # padded to the longest chunk
    q[seq, i] = s["q"].float()
    pos = torch.full((seqs, s["max_rows"]), -1, dtype=torch.int64, device="cuda")
    pos[seq, i] = at
    q = q.unflatten(2, (heads, share)).permute(0, 2, 3, 1, 4).reshape(seqs, heads, share * s["max_rows"], dim)
    score = (q @ gather("k").transpose(-1, -2)).mul_(s["scale"]).unflatten(2, (share, s["max_rows"]))
    sees = inside[:, None, :] & (j <= pos[..., None])
    if case["window"]:
        sees &= (j > pos[..., None] - case["window"]) | (j < case["sinks"])
    score.masked_fill_(~sees[:, None, None], float("-inf"))
    top = score.amax(-1, keepdim=True)
    top = torch.where(torch.isfinite(top), top, 0.0)
    p = score.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = p.flatten(2, 3) @ gather("v")
    o = o.unflatten(2, (share, s["max_rows"])) / torch.where(total > 0, total, 1.0)
    o = o.permute(0, 3, 1, 2, 4).flatten(2, 3)[seq, i].to(torch.bfloat16)
    if s["lse"] is None:
        return [o]
    lse = (total.log() + top).squeeze(-1).permute(0, 3, 1, 2).flatten(2, 3)[seq, i]
    return [o, lse]


# ------------------------------------------------------------------- 64 bits
def exact(case, seed):
    """From the definition, a sequence and a head at a time, in 64 bits."""
    if work(case)["flops"] > 5e12:
        return None
    s = prepare(case, seed)
    fmt, dim, page = case["fmt"], case["dim"], case["page"]
    start = [0] + list(np.cumsum(s["rows"]))

    def whole(name, b, h, n):
        """Rows 0..n-1 of sequence b, head h."""
        at = np.arange(n)
        pid = s["table"][b][torch.as_tensor(at // page, device="cuda")].long()
        r = torch.as_tensor(at % page, device="cuda")
        x = s[name][pid, h, r]
        if fmt == "bf16":
            return x.double()
        step, low = s[name + "_par"][pid, h, r].double().unbind(-1)            # [n, groups]
        out = torch.empty((n, dim), dtype=torch.float64, device="cuda")
        per = 4 if fmt == "u8" else 8                                          # channels of a word
        words = GROUP // per
        for c in range(dim):
            g, k = divmod(c % GROUP, per)
            place = (g % 4) * (words // 4) + g // 4
            byte = (c // GROUP) * words * 4 + place * 4 + (k if fmt == "u8" else k // 2)
            code = x[:, byte].long()
            if fmt == "u4":
                code = (code >> (4 * (k % 2))) & 15
            out[:, c] = code.double() * step[:, c // GROUP] + low[:, c // GROUP]
        return out

    if case["op"] == "write":  # read back, a written value is its group's nearest level
        out = []
        for name in ("k", "v"):
            x = s[name + "_new"].double()
            done = torch.empty_like(x)
            for c in range(0, dim, GROUP):
                g = x[..., c:c + GROUP]
                low = _f16_exactly(g.min(-1).values, -1)[..., None]
                step = _f16_exactly((g.max(-1).values[..., None] - low).squeeze(-1) / LEVELS[fmt], 1)[..., None]
                level = torch.where(step > 0, ((g - low) / step).round().clamp(0, LEVELS[fmt]), 0.0)
                done[..., c:c + GROUP] = level * step + low
            out.append(done)
        return out
    if case["op"] == "read":
        return [torch.cat([torch.stack([whole(name, b, h, length)[length - n:] for h in range(case["heads"])], 1)
                           for b, (n, length) in enumerate(zip(s["rows"], s["kv"]))]) for name in ("k", "v")]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    for b, (n, length) in enumerate(zip(s["rows"], s["kv"])):
        key = torch.arange(length, device="cuda")
        for h in range(case["heads"]):
            k, v = whole("k", b, h, length), whole("v", b, h, length)
            for first in range(0, n, 1024):
                last = min(n, first + 1024)
                pos = torch.arange(length - n + first, length - n + last, device="cuda")[:, None]
                hidden = key > pos
                if case["window"]:
                    hidden |= (key <= pos - case["window"]) & (key >= case["sinks"])
                for head in range(h * case["share"], (h + 1) * case["share"]):
                    at = slice(start[b] + first, start[b] + last)
                    z = (s["q"][at, head].double() @ k.T * s["scale"]).masked_fill(hidden, -math.inf)
                    lse[at, head] = torch.logsumexp(z, -1)
                    o[at, head] = torch.softmax(z, -1) @ v
    return [o] if not case["lse"] else [o, lse]


def _f16_exactly(x, way):
    """x (float64) rounded to float16's values, down (-1) or up (1), by the spacing at its magnitude."""
    spacing = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -14))).clamp(min=-14) - 10)
    return (torch.floor(x / spacing) if way < 0 else torch.ceil(x / spacing)) * spacing
