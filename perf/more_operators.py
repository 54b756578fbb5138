"""A decoder's step over a long paged cache: rotated queries and keys, pages chosen by
their bounds, attention over the chosen pages, and pages copied and compacted.

What is measured: the calls that a program makes for each layer while it writes
an answer from a cache of many pages. New rows' queries and keys are normalised
and rotated on their way into pages; the bounds of the pages' keys are brought
up to date; each new row chooses pages by them and attends to those alone; a
session is forked or cut to its kept rows by moving pages. `run` makes the
calls through the package where `own` is true, and in plain torch operations
where it is not.
"""
import math

import numpy as np
import torch

own = False

GROUP = 64                       # channels that share a step and a minimum
LEVELS = {"u8": 255, "u4": 15}
LARGEST = 32768.0                # a group with a larger magnitude is marked
POSITIONS = 32768                # rows of the rotation's table
LEAST = -40                      # exponent of the smallest step of bounds and of 8-bit queries


# ------------------------------------------------------------------- the cases
def listed():
    """Sizes are this repository's: 4 or 8 KV heads of 128 channels with 7 or 8 query heads each, 112 heads where all layers
    go at once, frames of 196 tokens, caches of 6272 to 9408 rows, and of 24576 and more where pages are chosen."""
    return [
        # One token of one stream, positions of three axes (time, height, width): latency counts.
        dict(name="rotate token", op="rotate", fmt="bf16", seqs=1, rows=1, kv=6273, ragged=0, heads=4, share=7, dim=128, page=64,
             rot=128, axes=3, pairs=0, norm=0),
        # 16 new frames of one layer, with norms of queries and keys.
        dict(name="rotate 16 frames", op="rotate", fmt="bf16", seqs=1, rows=3136, kv=9408, ragged=0, heads=4, share=7, dim=128, page=64,
             rot=128, axes=3, pairs=0, norm=1),
        # After the tokens of 8 streams were written: the pages that hold them.
        dict(name="bounds 8 tokens", op="bounds", fmt="bf16", seqs=8, rows=1, kv=24577, ragged=1, heads=8, dim=128, page=64),
        # A whole compacted cache, all layers' heads.
        dict(name="bounds compacted", op="bounds", fmt="bf16", seqs=1, rows=6272, kv=6272, ragged=0, heads=112, dim=128, page=64),
        # One token of one stream: 32 of 98 pages; latency counts.
        dict(name="choose token", op="choose", seqs=1, rows=1, kv=6272, ragged=0, heads=4, share=7, dim=128, page=64, chosen=32,
             first=1, recent=2),
        # 32 streams' tokens: 64 of up to 769 pages.
        dict(name="choose 32 ragged", op="choose", seqs=32, rows=1, kv=24577, ragged=1, heads=8, share=8, dim=128, page=32, chosen=64,
             first=1, recent=2),
        # One token over 32 chosen pages of a long stream: latency counts.
        dict(name="token bf16 32 pages", op="attend", fmt="bf16", seqs=1, rows=1, kv=98304, ragged=0, heads=4, share=7, dim=128, page=64,
             chosen=32, lse=1),
        # 32 streams' tokens over 4-bit pages, 64 of up to 769.
        dict(name="token u4 32 ragged", op="attend", fmt="u4", seqs=32, rows=1, kv=24577, ragged=1, heads=8, share=8, dim=128, page=32,
             chosen=64, lse=0),
        # Questions of up to 61 tokens, each token with pages of its own.
        dict(name="question bf16 8 ragged", op="attend", fmt="bf16", seqs=8, rows=61, kv=12349, ragged=1, heads=4, share=7, dim=128, page=64,
             chosen=24, lse=0),
        # 8 sessions forked: their last pages, partly filled, become pages of their own.
        dict(name="copy 8 pages", op="copy", fmt="bf16", pairs_of=8, pages=512, heads=4, dim=128, page=64),
        # A cache cut to the rows that a compression pass keeps, all layers' heads, each with rows of its own.
        dict(name="compact 112 heads", op="gather", fmt="bf16", seqs=1, rows=6272, kv=9408, ragged=0, heads=112, dim=128, page=64),
        # 8 streams' 4-bit pages of one layer cut to two thirds.
        dict(name="compact 8 streams u4", op="gather", fmt="u4", seqs=8, rows=16384, kv=24576, ragged=1, heads=8, dim=128, page=32),
    ]


def _log(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))))


def draw(rng):
    while True:
        op = rng.choice(["rotate", "bounds", "choose", "attend", "attend", "copy", "gather"])
        fmt = rng.choice(["bf16", "bf16", "u8", "u4"])
        c = dict(op=op, heads=rng.choice([1, 2, 4, 8]), dim=rng.choice([64, 128, 128, 80, 96] if fmt == "bf16" else [64, 128, 128]),
                 page=rng.choice([16, 32, 64, 64, 128]), ragged=rng.randint(0, 1))
        if op != "choose":
            c["fmt"] = fmt
        share = rng.choice([1, 2, 3, 4, 5, 6, 7, 8])
        if op == "rotate":
            if fmt == "u4":  # what bf16 leaves open moves a 4-bit code by a whole step
                c["fmt"] = "u8"
            c.update(share=share, seqs=_log(rng, 1, 32), rows=_log(rng, 1, 4096), axes=rng.choice([1, 3]) if c["dim"] != 80 else 1,
                     pairs=rng.randint(0, 1), norm=rng.randint(0, 1))
            c["rot"] = rng.choice([c["dim"], c["dim"], 64])
            c["kv"] = c["rows"] + _log(rng, 1, 2048)
        elif op == "bounds":
            c.update(heads=rng.choice([1, 4, 8, 28, 112]), seqs=_log(rng, 1, 32), rows=_log(rng, 1, 8192))
            c["kv"] = c["rows"] + _log(rng, 1, 8192)
        elif op in ("choose", "attend"):
            c.update(share=share, seqs=_log(rng, 1, 48), rows=1 if rng.random() < 0.6 else _log(rng, 2, 64))
            c["kv"] = c["rows"] + _log(rng, 1, 65536)
            c["chosen"] = _log(rng, 4, 96)
            if op == "choose":
                if c["kv"] <= c["chosen"] * c["page"]:  # nothing to choose
                    continue
                c.update(first=rng.randint(0, 2), recent=rng.randint(1, 2))
            else:
                c["lse"] = rng.randint(0, 1)
        elif op == "copy":
            c.update(pairs_of=_log(rng, 1, 1024), pages=2048)
            del c["ragged"]
            if c["pages"] * c["heads"] * c["page"] * c["dim"] > 1.4e8:
                continue
        else:
            c.update(heads=rng.choice([1, 4, 8, 28, 112]), seqs=_log(rng, 1, 16), kv=_log(rng, 2, 24576))
            c["rows"] = max(1, int(c["kv"] * rng.uniform(0.3, 0.9)))
        if op != "copy":
            if c["seqs"] * c["kv"] * c["heads"] * c["dim"] > 1.3e8:
                continue
            if op in ("choose", "attend") and c["seqs"] * c["rows"] * c["heads"] * (
                    c["chosen"] * c["page"] * c["dim"] / 1.2e8 if op == "attend" else -(-c["kv"] // c["page"]) * c["share"] / 1e8) > 1:
                continue
            if op == "rotate" and c["seqs"] * c["rows"] * c["heads"] * (c["share"] + 2) * c["dim"] > 1.4e7:
                continue
        return c


def _lengths(case):
    """(new rows, rows held with them) of each sequence: the case's own where it is not ragged, else spread below it, the
    first sequence's the full ones."""
    rows, kv = [], []
    for b in range(case["seqs"]):
        f = 1.0 - 0.85 * ((b * 0.6180339887498949) % 1.0) if case["ragged"] else 1.0
        n = max(1, int(case["rows"] * f))
        rows.append(n)
        kv.append(max(n, int(case["kv"] * f)))
    return rows, kv


def _padded(dim):
    return 64 if dim <= 64 else 128


def _row_bytes(case):
    if case["fmt"] == "bf16":
        return 2 * case["dim"]
    return case["dim"] // (1 if case["fmt"] == "u8" else 2) + 4 * (case["dim"] // GROUP)


def work(case):
    d, h, page = case["dim"], case["heads"], case["page"]
    if case["op"] == "copy":
        return {"bytes": case["pairs_of"] * h * page * 2 * 2 * _row_bytes(case) + 8 * case["pairs_of"] +
                (case["pairs_of"] * h * page * 2 * 2 * d if case["fmt"] != "bf16" else 0), "flops": 0}
    rows, kv = _lengths(case)
    if case["op"] == "rotate":
        n = sum(rows)
        out = 2 * d if case["fmt"] == "bf16" else _row_bytes(case) + 2 * d          # codes are read back
        return {"bytes": n * h * ((case["share"] + 2) * 2 * d + case["share"] * 2 * d + 2 * out) + n * (4 * case["rot"] + 4 * case["axes"]),
                "flops": n * h * (case["share"] + 1) * (3 * case["rot"] + 4 * d * case["norm"])}
    if case["op"] == "gather":
        moved = sum(rows) * h * 2
        return {"bytes": moved * (2 * _row_bytes(case) + 2) + (moved * 2 * d if case["fmt"] != "bf16" else 0), "flops": 0}
    if case["op"] == "bounds":
        first = [(length - n) // page * page for n, length in zip(rows, kv)]
        seen = sum(length - f for length, f in zip(kv, first))
        held = sum(-(-length // page) - f // page for length, f in zip(kv, first))
        return {"bytes": h * (seen * _row_bytes(case) + held * (2 * _padded(d) + 4)), "flops": 2 * h * seen * d}
    pages = [-(-length // page) for length in kv]
    if case["op"] == "choose":
        q = sum(rows) * h * case["share"] * d * 2
        return {"bytes": q + h * sum(pages) * (2 * _padded(d) + 4) + 4 * sum(rows) * h * case["chosen"],
                "flops": 4 * d * h * case["share"] * sum(n * p for n, p in zip(rows, pages))}
    # Pages of one sequence that some of its rows chose, as often as independent choices give.
    some = sum(p * (1 - (1 - min(1.0, case["chosen"] / p)) ** n) for n, p in zip(rows, pages))
    each = sum(n * min(p * page, length, case["chosen"] * page) for n, p, length in zip(rows, pages, kv))
    return {"bytes": int(min(some * page, sum(kv))) * h * 2 * _row_bytes(case) + sum(rows) * h * (case["share"] * d * 4 + 4 * case["chosen"]),
            "flops": 4 * d * h * case["share"] * each}


def _exponent(top):
    """The smallest e >= LEAST with top <= 127 * 2^e, by top's own exponent."""
    m, e = torch.frexp(top.double())
    return torch.where(m * 128.0 <= 127.0, e - 7, e - 6).clamp(min=LEAST).double()


# ------------------------------------------------------------- the packed format
def _f16_toward(x, up):
    """x (float32) as float16, rounded up or down; x lies within float16's range."""
    h = x.to(torch.float16)
    off = (h.float() < x) if up else (h.float() > x)
    bits = h.view(torch.int16).to(torch.int32) & 0xFFFF
    negative = bits >= 0x8000
    away = torch.where(negative, -1, 1) if up else torch.where(negative, 1, -1)
    moved = torch.where((bits & 0x7FFF) == 0, torch.full_like(bits, 0x0001 if up else 0x8001), bits + away)
    bits = torch.where(off, moved, bits)
    return torch.where(bits >= 0x8000, bits - 0x10000, bits).to(torch.int16).view(torch.float16)


def _quantise(x, fmt):
    """x [..., dim] -> (codes uint8 [..., groups, 64], step and minimum float16 [..., groups, 2])."""
    g = x.float().unflatten(-1, (-1, GROUP))
    lo, hi = g.amin(-1), g.amax(-1)
    good = torch.isfinite(g).all(-1) & (torch.maximum(lo.abs(), hi.abs()) <= LARGEST)
    lo, hi = torch.where(good, lo, 0.0), torch.where(good, hi, 0.0)
    low = _f16_toward(lo, False)
    step = _f16_toward((hi - low.float()) / torch.full_like(hi, LEVELS[fmt]), True)
    s, m = step.float()[..., None], low.float()[..., None]
    u = torch.where((s > 0) & good[..., None], torch.round((g - m) / torch.where(s > 0, s, 1.0)), 0.0)
    nan = torch.full_like(step, float("nan"))
    par = torch.stack([torch.where(good, step, nan), torch.where(good, low, nan)], -1)
    return u.nan_to_num(0.0).clamp(0, LEVELS[fmt]).to(torch.uint8), par


def _pack(u, fmt):
    """Codes [..., groups, 64] -> bytes [..., dim or dim/2]: the word of channels 4(t + 4w).. or 8(t + 4w).. of a group in
    place t * (words / 4) + w."""
    if fmt == "u4":
        u = u[..., 0::2] | (u[..., 1::2] << 4)
    return u.unflatten(-1, (-1, 4, 4)).transpose(-3, -2).flatten(-4)


def _values(codes, par, fmt, dim):
    """Bytes [..., dim or dim/2] and parameters [..., groups, 2] -> float32 [..., dim]."""
    w = codes.unflatten(-1, (dim // GROUP, 4, -1, 4)).transpose(-3, -2).flatten(-3)
    if fmt == "u4":
        w = torch.stack([w & 15, w >> 4], -1).flatten(-2)
    return (w.float() * par[..., 0:1].float() + par[..., 1:2].float()).flatten(-2)


# ------------------------------------------------------------------- the inputs
def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(seed & 0x7FFFFFFFFFFF)


def _keys(shape, gen):
    """Keys of a stream's pages as a decoder's: rows of a page have a direction in common, a few wide channels an offset."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    if len(shape) == 4:
        x += torch.randn(shape[:2] + (1, shape[3]), generator=gen, device="cuda", dtype=torch.bfloat16)
    wide = torch.randint(0, shape[-1], (max(1, shape[-1] // 32),), generator=gen, device="cuda")
    gain, shift = torch.ones(shape[-1], device="cuda"), torch.zeros(shape[-1], device="cuda")
    gain[wide] = 4.0
    shift[wide] = torch.randn(wide.shape, generator=gen, device="cuda") * 3.0
    return x.mul_(gain.to(x.dtype)).add_(shift.to(x.dtype))


def _normal_values(shape, gen):
    """Values: Gaussian directions with lognormal magnitudes."""
    x = torch.randn(shape, generator=gen, device="cuda", dtype=torch.bfloat16)
    return x.mul_(torch.randn(shape[:-1] + (1,), generator=gen, device="cuda").mul_(0.5).exp_().to(x.dtype))


def _pool(s, gen, pages, filled, name=""):
    """Tensors of a pool: k, v and, for codes, k_par, v_par, under these names + `name`."""
    case = s["case"]
    heads, dim, page, fmt = case["heads"], case["dim"], case["page"], case["fmt"]
    shape = (pages, heads, page, dim)
    for x, make in (("k", _keys), ("v", _normal_values)):
        if fmt == "bf16":
            s[x + name] = make(shape, gen) if filled else torch.zeros(shape, dtype=torch.bfloat16, device="cuda")
            s[x + name + "_par"] = None
            continue
        codes = torch.zeros(shape[:-1] + (dim // (1 if fmt == "u8" else 2),), dtype=torch.uint8, device="cuda")
        par = torch.zeros(shape[:-1] + (dim // GROUP, 2), dtype=torch.float16, device="cuda")
        part = max(1, (1 << 25) // (heads * page * dim))
        for i in range(0, pages if filled else 0, part):
            n = min(part, pages - i)
            u, p = _quantise(make((n,) + shape[1:], gen), fmt)
            codes[i:i + n], par[i:i + n] = _pack(u, fmt), p
        s[x + name], s[x + name + "_par"] = codes, par


def _tables(s, gen, kv, page, name=""):
    """Page tables of sequences of kv rows over a pool whose pages are handed out in no order; the number of its pages."""
    held = [-(-n // page) for n in kv]
    pages = sum(held) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    table = torch.full((len(kv), max(held)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, k in enumerate(held):
        table[b, :k] = order[at:at + k]
        at += k
    s["table" + name] = table
    s["kv_len" + name] = torch.tensor(kv, dtype=torch.int32, device="cuda")
    s["max_kv" + name] = max(kv)
    return pages


def prepare(case, seed):
    gen = _generator(seed)
    s = dict(case=case)
    page, heads, dim, op = case["page"], case["heads"], case["dim"], case["op"]
    if op == "copy":
        n, pages = case["pairs_of"], case["pages"]
        _pool(s, gen, pages, True)
        order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
        s["source"], s["target"] = order[:n].contiguous(), order[n:2 * n].contiguous()
        s["table"] = s["target"][None]
        s["row_start"] = torch.tensor([0, n * page], dtype=torch.int32, device="cuda")
        s["kv_len"] = torch.tensor([n * page], dtype=torch.int32, device="cuda")
        s["total"] = s["max_rows"] = s["max_kv"] = n * page
        return s
    rows, kv = _lengths(case)
    total = sum(rows)
    s["row_start"] = torch.tensor([0] + list(np.cumsum(rows)), dtype=torch.int32, device="cuda")
    s["total"], s["max_rows"] = total, max(rows)
    if op == "gather":  # rows kept of each head, ascending: the latest eighth, and others
        pages = _tables(s, gen, kv, page, "_from")
        _pool(s, gen, pages, True, "_from")
        _pool(s, gen, _tables(s, gen, rows, page), False)
        kept = torch.zeros((case["seqs"], heads, max(rows)), dtype=torch.int32, device="cuda")
        for b, (n, length) in enumerate(zip(rows, kv)):
            x = torch.rand((heads, length), generator=gen, device="cuda")
            x[:, length - max(1, n // 8):] += 1.0
            kept[b, :, :n] = x.topk(n, -1).indices.sort(-1).values.to(torch.int32)
        s["kept"] = kept
        return s
    pages = _tables(s, gen, kv, page)
    if op == "rotate":
        share, rot = case["share"], case["rot"]
        _pool(s, gen, pages, False)
        s["q"] = torch.randn((total, heads * share, dim), generator=gen, device="cuda", dtype=torch.bfloat16) * 1.5
        s["q_out"] = torch.empty_like(s["q"])
        s["k_new"], s["v_new"] = _keys((total, heads, dim), gen), _normal_values((total, heads, dim), gen)
        angle = torch.arange(POSITIONS, dtype=torch.float64, device="cuda")[:, None] * (
            1e6 ** (-2.0 * torch.arange(rot // 2, dtype=torch.float64, device="cuda") / rot))
        s["turns"] = torch.cat([angle.cos(), angle.sin()], 1).float()
        s["positions"] = torch.randint(0, POSITIONS, (case["axes"], total), generator=gen, device="cuda", dtype=torch.int32)
        third = rot // 2 // 3 // 8 * 8
        s["sections"] = [rot // 2 - 2 * third, third, third][:case["axes"]] if case["axes"] > 1 else [rot // 2]
        for x in ("q", "k"):
            w = 1.0 + 0.2 * torch.randn(dim, generator=gen, device="cuda")
            s[x + "_weight"] = w.to(torch.bfloat16) if case["norm"] else None
        return s
    if op == "bounds":
        _pool(s, gen, pages, True)
        s["codes"] = torch.zeros((pages, heads, 2, _padded(dim)), dtype=torch.int8, device="cuda")
        s["steps"] = torch.zeros((pages, heads), device="cuda")
        return s
    if op == "choose":  # bounds of pages whose keys lie 2 or 3 deviations around a direction of the page's own
        mid = torch.randn((pages, heads, dim), generator=gen, device="cuda")
        wide = 1.5 + torch.rand((pages, heads, dim), generator=gen, device="cuda")
        top = (mid.abs() + wide).amax(-1)
        step = torch.exp2(_exponent(top)).float()
        s["codes"] = torch.zeros((pages, heads, 2, _padded(dim)), dtype=torch.int8, device="cuda")
        for i, (x, rounded) in enumerate(((mid - wide, torch.floor), (mid + wide, torch.ceil))):
            s["codes"][:, :, i, :dim] = rounded(x / step[..., None]).to(torch.int8)
        s["steps"] = step
        s["q"] = torch.randn((total, heads * case["share"], dim), generator=gen, device="cuda", dtype=torch.bfloat16) * 1.5
        s["chosen"] = torch.full((total, heads, case["chosen"]), -1, dtype=torch.int32, device="cuda")
        return s
    _pool(s, gen, pages, True)
    s["q"] = torch.randn((total, heads * case["share"], dim), generator=gen, device="cuda", dtype=torch.bfloat16) * 1.5
    s["out"] = torch.empty_like(s["q"])
    s["lse"] = torch.empty((total, heads * case["share"]), device="cuda") if case["lse"] else None
    s["scale"] = dim ** -0.5
    # Lists as choosing makes them: ascending, a row's own page among them, all pages where there are no more.
    n = case["chosen"]
    chosen = torch.full((total, heads, n), -1, dtype=torch.int32, device="cuda")
    at = 0
    for rows_b, length in zip(rows, kv):
        own_page = torch.arange(length - rows_b, length, device="cuda") // page
        held = -(-length // page)
        x = torch.rand((rows_b, heads, held), generator=gen, device="cuda")
        j = torch.arange(held, device="cuda")
        x = torch.where(j > own_page[:, None, None], -1.0, x)
        x = torch.where((j == own_page[:, None, None]) | (j == 0), 2.0, x)
        best = x.topk(min(n, held), -1)
        some = torch.where(best.values < 0, 1 << 30, best.indices).sort(-1).values
        chosen[at:at + rows_b, :, :some.shape[-1]] = torch.where(some == 1 << 30, -1, some).to(torch.int32)
        at += rows_b
    s["chosen"] = chosen
    return s


# --------------------------------------------------------------------- the passes
def _run_own(s):
    from paper_2506_15745_gb300.paged import PageBounds, PagedBatch, PagedCache, Rotary

    case = s["case"]
    op = case["op"]
    if "batch" not in s:  # the handles a program keeps
        s["batch"] = PagedBatch(s["table"], s["row_start"], s["kv_len"], total_rows=s["total"], max_rows=s["max_rows"], max_kv=s["max_kv"])
        if op != "choose":
            s["cache"] = PagedCache.from_tensors(case["fmt"], s["k"], s["v"], s["k_par"], s["v_par"])
        if op in ("bounds", "choose"):
            s["bounds"] = PageBounds.from_tensors(s["codes"], s["steps"], case["page"], case["dim"])
        if op == "rotate":
            s["rotary"] = Rotary(s["turns"], s["sections"], interleaved=bool(case["pairs"]))
        if op == "gather":
            s["cache_from"] = PagedCache.from_tensors(case["fmt"], *(s[x + "_from" + p] for p in ("", "_par") for x in ("k", "v")))
            # of the source only the lengths matter: no rows of its own are new
            s["batch_from"] = PagedBatch(s["table_from"], torch.zeros_like(s["row_start"]), s["kv_len_from"], total_rows=0, max_rows=0,
                                         max_kv=s["max_kv_from"])
        if case.get("fmt") in LEVELS and op != "bounds" and op != "attend":
            s["k_out"] = torch.empty((s["total"], case["heads"], case["dim"]), dtype=torch.bfloat16, device="cuda")
            s["v_out"] = torch.empty_like(s["k_out"])
    batch = s["batch"]
    if op == "choose":
        s["bounds"].choose(s["q"], batch, case["chosen"], first=case["first"], recent=case["recent"], out=s["chosen"])
        return [s["chosen"]]
    cache = s["cache"]
    if op == "bounds":
        s["bounds"].update(cache, batch)
        return [s["codes"], s["steps"]]
    if op == "attend":
        cache.attend_chosen(s["q"], batch, s["chosen"], out=s["out"], lse=s["lse"], scale=s["scale"])
        return [s["out"]] if s["lse"] is None else [s["out"], s["lse"]]
    out = []
    if op == "rotate":
        out.append(cache.write_rotated(s["q"], s["k_new"], s["v_new"], batch, s["rotary"], s["positions"], q_weight=s["q_weight"],
                                       k_weight=s["k_weight"], q_out=s["q_out"]))
    elif op == "copy":
        cache.copy_pages(s["source"], s["target"])
    else:
        cache.gather(s["cache_from"], s["batch_from"], batch, s["kept"])
    if case["fmt"] == "bf16":
        return out + [s["k"], s["v"]]
    cache.read(batch, s["k_out"], s["v_out"])
    return out + [s["k_out"], s["v_out"]]


def _places(s):
    """(page, row in it) of every new row, packed: int64 [total] each; and each new row's sequence, number in it and position."""
    n = (s["row_start"][1:] - s["row_start"][:-1]).long()
    seq = torch.repeat_interleave(torch.arange(len(n), device="cuda"), n, output_size=s["total"])
    i = torch.arange(s["total"], device="cuda") - s["row_start"].long()[seq]
    at = s["kv_len"].long()[seq] - n[seq] + i
    page = s["case"]["page"]
    return s["table"].long()[seq, at // page], at % page, seq, i, at


def _rotated(s, x, weight):
    """Normalised and rotated rows, float32."""
    case = s["case"]
    rot, half = case["rot"], case["rot"] // 2
    x = x.float()
    if weight is not None:
        x = x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6) * weight.float()
    axis = torch.repeat_interleave(torch.arange(case["axes"], device="cuda"), torch.tensor(s["sections"], device="cuda"), output_size=half)
    place = s["positions"].long()[axis].T                                     # [rows, half]
    f = torch.arange(half, device="cuda")
    c, d = s["turns"][place, f][:, None], s["turns"][place, f + half][:, None]
    a, b = (x[..., 0:rot:2], x[..., 1:rot:2]) if case["pairs"] else (x[..., :half], x[..., half:rot])
    turned = (a * c - b * d, b * c + a * d)
    turned = torch.stack(turned, -1).flatten(-2) if case["pairs"] else torch.cat(turned, -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _scores(s):
    """Each new row's scores of its sequence's pages, [rows, heads, pages], float32: products of integers, exact."""
    case = s["case"]
    seqs, heads, share, dim, wide = case["seqs"], case["heads"], case["share"], case["dim"], s["table"].shape[1]
    _, _, seq, i, at = _places(s)
    q = s["q"].float().unflatten(1, (heads, share))
    e = _exponent(q.abs().amax(-1))
    code = torch.round(q / torch.exp2(e)[..., None].float())
    parts = torch.cat([code.clamp(max=0), code.clamp(min=0)], -1)              # with the lower bounds, with the upper ones
    rows = torch.zeros((seqs, s["max_rows"], heads, share, 2 * dim), device="cuda")
    rows[seq, i] = parts
    table = s["table"].long().clamp(min=0)
    codes = s["codes"][table][..., :dim].float().flatten(-2)                   # [seqs, pages, heads, 2 dim]
    rows = rows.permute(0, 2, 1, 3, 4).reshape(seqs, heads, s["max_rows"] * share, 2 * dim)
    dots = rows @ codes.permute(0, 2, 3, 1)                                    # whole numbers below 2^24
    dots = dots.unflatten(2, (s["max_rows"], share)).permute(0, 2, 1, 3, 4)[seq, i].double()
    dots = dots * torch.exp2(e)[..., None] * s["steps"][table].double().transpose(1, 2)[seq][:, :, None, :]
    return dots.amax(2).float(), at


def run(s):
    if own:
        return _run_own(s)
    case = s["case"]
    op, dim, heads, page, fmt = case["op"], case["dim"], case["heads"], case["page"], case.get("fmt")

    def held(name, at):
        """Rows of a pool, float32."""
        x = s[name][at]
        return x.float() if fmt == "bf16" else _values(x, s[name + "_par"][at], fmt, dim)

    if op == "copy":
        source, target = s["source"].long(), s["target"].long()
        for x in ("k", "v") if fmt == "bf16" else ("k", "v", "k_par", "v_par"):
            s[x][target] = s[x][source]
        if fmt == "bf16":
            return [s["k"], s["v"]]
        return [held(x, target).transpose(1, 2).flatten(0, 1).to(torch.bfloat16) for x in ("k", "v")]
    pid, row, seq, i, at = _places(s)
    if op == "rotate":
        new = {"k": _rotated(s, s["k_new"], s["k_weight"]).to(torch.bfloat16), "v": s["v_new"]}
        out = [_rotated(s, s["q"], s["q_weight"]).to(torch.bfloat16)]
        for x in ("k", "v"):
            if fmt == "bf16":
                s[x][pid, :, row] = new[x]
                out.append(s[x])
            else:
                u, par = _quantise(new[x], fmt)
                s[x][pid, :, row], s[x + "_par"][pid, :, row] = _pack(u, fmt), par
                out.append(held(x, (pid, slice(None), row)).to(torch.bfloat16))
        return out
    if op == "gather":
        h = torch.arange(heads, device="cuda")[None]
        j = s["kept"].long()[seq, :, i]                                        # [rows, heads]
        source = s["table_from"].long()[seq[:, None], j // page]
        for x in ("k", "v") if fmt == "bf16" else ("k", "v", "k_par", "v_par"):
            name = x[0] + "_from" + x[1:]
            s[x][pid, :, row] = s[name][source, h, j % page]
        if fmt == "bf16":
            return [s["k"], s["v"]]
        return [held(x, (pid, slice(None), row)).to(torch.bfloat16) for x in ("k", "v")]
    if op == "bounds":
        wide = s["table"].shape[1]
        new = torch.zeros((case["seqs"], wide), dtype=torch.bool, device="cuda")
        new[seq, at // page] = True
        b, p = new.nonzero(as_tuple=True)
        g = s["table"].long()[b, p]
        inside = torch.arange(page, device="cuda") < (s["kv_len"].long()[b] - p * page)[:, None]
        k = held("k", g).to(torch.bfloat16).float()                            # [pages, heads, page, dim]
        low = torch.where(inside[:, None, :, None], k, math.inf).amin(2)
        high = torch.where(inside[:, None, :, None], k, -math.inf).amax(2)
        top = torch.maximum(low.abs(), high.abs()).amax(-1)
        step = torch.exp2(_exponent(top))
        s["codes"][g, :, 0, :dim] = torch.floor(low / step[..., None]).to(torch.int8)
        s["codes"][g, :, 1, :dim] = torch.ceil(high / step[..., None]).to(torch.int8)
        s["steps"][g] = step.float()
        return [s["codes"], s["steps"]]
    if op == "choose":
        score, at = _scores(s)
        n, last = case["chosen"], (at // page)[:, None, None]
        j = torch.arange(score.shape[-1], device="cuda")
        score = torch.where((j < case["first"]) | (j > last - case["recent"]), math.inf, score)
        score = torch.where(j > last, -math.inf, score)
        best = score.argsort(dim=-1, descending=True, stable=True)[..., :n]    # ties go to the lower page
        best = torch.where(best > last, 1 << 30, best).sort(-1).values
        s["chosen"].fill_(-1)
        s["chosen"][..., :best.shape[-1]] = torch.where(best == 1 << 30, -1, best).to(torch.int32)
        return [s["chosen"]]

    share, n = case["share"], case["chosen"]
    chosen = s["chosen"].long()                                                # [rows, heads, n]
    g = s["table"].long()[seq[:, None, None], chosen.clamp(min=0)]
    h = torch.arange(heads, device="cuda")[None, :, None]
    place = chosen[..., None] * page + torch.arange(page, device="cuda")
    sees = ((chosen[..., None] >= 0) & (place <= at[:, None, None, None])).flatten(2)          # [rows, heads, keys]
    q = s["q"].float().unflatten(1, (heads, share))
    k = torch.where(sees[..., None], held("k", (g, h)).flatten(2, 3), 0.0)
    score = (q @ k.transpose(-1, -2)) * s["scale"]
    del k
    score = score.masked_fill_(~sees[:, :, None], -math.inf)
    top = score.amax(-1, keepdim=True)
    p = score.sub_(torch.where(torch.isfinite(top), top, 0.0)).exp_()
    total = p.sum(-1, keepdim=True)
    v = torch.where(sees[..., None], held("v", (g, h)).flatten(2, 3), 0.0)
    o = ((p @ v) / torch.where(total > 0, total, 1.0)).flatten(1, 2).to(torch.bfloat16)
    if s["lse"] is None:
        return [o]
    return [o, (total.log() + top).squeeze(-1).flatten(1, 2)]


# ------------------------------------------------------------------- 64 bits
def _whole(case, x, par, pid, h, r):
    """Values of rows r of pages pid, head h, in 64 bits, channel by channel where they are codes."""
    fmt, dim = case["fmt"], case["dim"]
    x = x[pid, h, r]
    if fmt == "bf16":
        return x.double()
    step, low = par[pid, h, r].double().unbind(-1)
    out = torch.empty(x.shape[:-1] + (dim,), dtype=torch.float64, device="cuda")
    per = 4 if fmt == "u8" else 8
    words = GROUP // per
    for c in range(dim):
        g, k = divmod(c % GROUP, per)
        code = x[..., (c // GROUP) * words * 4 + ((g % 4) * (words // 4) + g // 4) * 4 + (k if fmt == "u8" else k // 2)].long()
        if fmt == "u4":
            code = (code >> (4 * (k % 2))) & 15
        out[..., c] = code.double() * step[..., c // GROUP] + low[..., c // GROUP]
    return out


def _f16_exactly(x, way):
    """x (float64) rounded to float16's values, down (-1) or up (1), by the spacing at its magnitude."""
    spacing = torch.exp2((torch.frexp(x.abs().clamp(min=2.0 ** -14)).exponent - 11).double())
    return (torch.floor(x / spacing) if way < 0 else torch.ceil(x / spacing)) * spacing


def exact(case, seed):
    """From the definitions, a sequence at a time, in 64 bits."""
    s = prepare(case, seed)
    op, dim, heads, page, fmt = case["op"], case["dim"], case["heads"], case["page"], case.get("fmt")
    if op in ("copy", "gather") and fmt == "bf16":
        pools = [s["k"].double(), s["v"].double()]
    if op == "copy":
        a, b = s["source"].tolist(), s["target"].tolist()
        if fmt == "bf16":
            for x in pools:
                x[b] = x[a]
            return pools
        r = torch.arange(page, device="cuda")
        return [torch.cat([torch.stack([_whole(case, s[x], s[x + "_par"], p, h, r) for h in range(heads)], 1) for p in a]) for x in ("k", "v")] \
            if len(a) <= 64 else None
    rows, kv = _lengths(case)
    start = [0] + list(np.cumsum(rows))
    if op == "gather":
        out = [[], []]
        for b, n in enumerate(rows):
            at = torch.arange(n, device="cuda")
            pid, r = s["table"][b].long()[at // page], at % page
            for h in range(heads):
                j = s["kept"][b, h, :n].long()
                source = s["table_from"][b].long()[j // page]
                for i, x in enumerate(("k", "v")):
                    y = _whole(case, s[x + "_from"], s[x + "_from_par"], source, h, j % page)
                    if fmt == "bf16":
                        pools[i][pid, h, r] = y
                    else:
                        out[i].append(y)
        if fmt == "bf16":
            return pools
        return [torch.cat([torch.stack(x[b * heads:(b + 1) * heads], 1) for b in range(len(rows))]) for x in out]
    if op == "rotate":
        rot, half = case["rot"], case["rot"] // 2
        axis = sum([[a] * n for a, n in enumerate(s["sections"])], [])
        made = {}
        for x, w in (("q", s["q_weight"]), ("k_new", s["k_weight"])):
            y = s[x].double()
            if w is not None:
                y = y / (y.pow(2).sum(-1, keepdim=True) / dim + 1e-6).sqrt() * w.double()
            z = y.clone()
            for f in range(half):
                turn = s["turns"][s["positions"][axis[f]].long()].double()
                c, d = turn[:, f, None], turn[:, half + f, None]
                i, j = (2 * f, 2 * f + 1) if case["pairs"] else (f, f + half)
                z[..., i] = y[..., i] * c - y[..., j] * d
                z[..., j] = y[..., i] * d + y[..., j] * c
            made[x] = z
        out = [made["q"]]
        for x, y in (("k", made["k_new"]), ("v", s["v_new"].double())):
            if fmt != "bf16":  # keys are bf16 before they are codes
                y = y.to(torch.bfloat16).double()
                done = torch.empty_like(y)
                for c in range(0, dim, GROUP):
                    g = y[..., c:c + GROUP]
                    low = _f16_exactly(g.min(-1).values, -1)[..., None]
                    step = _f16_exactly((g.max(-1).values[..., None] - low).squeeze(-1) / LEVELS[fmt], 1)[..., None]
                    done[..., c:c + GROUP] = torch.where(step > 0, ((g - low) / step).round().clamp(0, LEVELS[fmt]), 0.0) * step + low
                out.append(done)
                continue
            pool = s[x].double()
            for b, (n, length) in enumerate(zip(rows, kv)):
                at = torch.arange(length - n, length, device="cuda")
                pool[s["table"][b].long()[at // page], :, at % page] = y[start[b]:start[b + 1]]
            out.append(pool)
        return out
    if op == "bounds":
        codes, steps = s["codes"].clone(), s["steps"].double()
        for b, (n, length) in enumerate(zip(rows, kv)):
            if (length - (length - n) // page * page) * heads > 1e6:
                return None
            for p in range((length - n) // page, -(-length // page)):
                g = int(s["table"][b, p])
                r = torch.arange(min(page, length - p * page), device="cuda")
                k = torch.stack([_whole(case, s["k"], s["k_par"], g, h, r) for h in range(heads)]).to(torch.bfloat16).double()
                low, high = k.min(1).values, k.max(1).values
                e = torch.full((heads,), float(LEAST), dtype=torch.float64, device="cuda")
                top = k.abs().amax((1, 2))
                while bool((top > 127 * torch.exp2(e)).any()):
                    e += (top > 127 * torch.exp2(e)).double()
                codes[g, :, 0, :dim] = torch.floor(low / torch.exp2(e)[:, None]).to(torch.int8)
                codes[g, :, 1, :dim] = torch.ceil(high / torch.exp2(e)[:, None]).to(torch.int8)
                steps[g] = torch.exp2(e)
        return [codes, steps]
    if op == "choose":
        out = torch.full(s["chosen"].shape, -1, dtype=torch.int32, device="cuda")
        if sum(rows) * heads > 600:
            return None
        for b, (n, length) in enumerate(zip(rows, kv)):
            for i in range(n):
                last = (length - n + i) // page
                if last < case["chosen"]:
                    out[start[b] + i, :, :last + 1] = torch.arange(last + 1, device="cuda", dtype=torch.int32)
                    continue
                g = s["table"][b, :last + 1].long()
                for h in range(heads):
                    q = s["q"][start[b] + i, h * case["share"]:(h + 1) * case["share"]].double()
                    e = LEAST + sum((q.abs().amax(-1, keepdim=True) > 127 * 2.0 ** x).double() for x in range(LEAST, 60))
                    q = (q / torch.exp2(e)).round()[:, None]
                    low, high = s["codes"][g, h, 0, :dim].double(), s["codes"][g, h, 1, :dim].double()
                    score = (torch.maximum(q * low, q * high).sum(-1) * torch.exp2(e) * s["steps"][g, h].double()).max(0).values.cpu().numpy()
                    middle = np.arange(case["first"], last + 1 - case["recent"])
                    best = middle[np.lexsort((middle, -score[middle]))][:case["chosen"] - case["first"] - case["recent"]]
                    ends = np.r_[np.arange(case["first"]), np.arange(last + 1 - case["recent"], last + 1)]
                    out[start[b] + i, h] = torch.as_tensor(np.sort(np.r_[ends, best]).astype(np.int32), device="cuda")
        return [out]
    o = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.full(s["q"].shape[:2], -math.inf, dtype=torch.float64, device="cuda")
    share = case["share"]
    if sum(rows) * heads > 3000:
        return None
    for b, (n, length) in enumerate(zip(rows, kv)):
        for i in range(n):
            for h in range(heads):
                c = s["chosen"][start[b] + i, h].long()
                j = (c[c >= 0][:, None] * page + torch.arange(page, device="cuda")).flatten()
                j = j[j <= length - n + i]
                g = s["table"][b].long()[j // page]
                k, v = (_whole(case, s[x], s[x + "_par"], g, h, j % page) for x in ("k", "v"))
                at = slice(h * share, (h + 1) * share)
                z = s["q"][start[b] + i, at].double() @ k.T * s["scale"]
                lse[start[b] + i, at] = torch.logsumexp(z, -1)
                o[start[b] + i, at] = torch.softmax(z, -1) @ v
    return [o] if not case["lse"] else [o, lse]
