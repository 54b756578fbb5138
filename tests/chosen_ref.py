"""Plain float64 definitions of the operators beside the paged cache's attention: rotated rows, bounds of pages, pages
chosen by them, attention over chosen pages. For their tests.

Written from include/ipv.h's text; shares no code with the library or its binding. Everything works on CPU tensors.
"""
import math

import torch


def turned(x, weight, eps, table, positions, sections, interleaved):
    """x [rows, heads, dim] float64, table [n_positions, rot], positions [axes, rows]: the rows normalised (weight not None) and rotated,
    and per output the two products' magnitudes, which bound the rounding errors."""
    x, table = x.double(), table.double()
    rot = table.shape[1]
    if weight is not None:
        x = x * weight.double() / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    out, size = x.clone(), x.abs()
    f = 0
    for axis, count in enumerate(sections):
        for _ in range(count):
            i, j = (2 * f, 2 * f + 1) if interleaved else (f, f + rot // 2)
            for r in range(x.shape[0]):
                p = int(positions[axis, r])
                c, s = table[p, [f, f + rot // 2]] if 0 <= p < table.shape[0] else (math.nan, math.nan)
                a, b = x[r, :, i], x[r, :, j]
                out[r, :, i], out[r, :, j] = a * c - b * s, b * c + a * s
                size[r, :, i] = (a * c).abs() + (b * s).abs()
                size[r, :, j] = (b * c).abs() + (a * s).abs()
            f += 1
    return out, size


def exponent(top):
    """The smallest integer e >= -40 with top <= 127 * 2^e."""
    e = -40
    while top > 127.0 * 2.0 ** e:
        e += 1
    return e


def bounds(k):
    """Keys [rows, dim] of a page and head -> (lower, upper) int [dim] each, step."""
    if not torch.isfinite(k).all():
        return None, None, math.nan
    step = 2.0 ** exponent(float(k.abs().max()))
    return (k.amin(0).double() / step).floor().long(), (k.amax(0).double() / step).ceil().long(), step


def scores(q, lo, hi, step):
    """q [share, dim] of one row and KV head; lo, hi [pages, dim], step [pages] -> [pages], NaN: no score. The sums are of
    integers, so any order gives the same."""
    best = torch.full((lo.shape[0],), -math.inf, dtype=torch.float64)
    some = False
    for row in q.double():
        if not torch.isfinite(row).all():
            continue
        some = True
        up = 2.0 ** exponent(float(row.abs().max()))
        c = (row / up).round()
        best = torch.maximum(best, torch.maximum(c * lo, c * hi).sum(-1) * up * step)
    return torch.where(torch.isnan(step) | torch.tensor(not some), math.nan, best)


def choose(score, n, first, recent):
    """The pages chosen of those with these scores, [n], -1 behind the last."""
    pages = score.shape[0]
    if pages <= n:
        return list(range(pages)) + [-1] * (n - pages)
    middle = range(first, pages - recent)
    rank = sorted(middle, key=lambda p: (math.isnan(score[p]), 0.0 if math.isnan(score[p]) else -float(score[p]), p))
    return sorted(list(range(first)) + rank[:n - first - recent] + list(range(pages - recent, pages)))


def attend(q, k, v, chosen, page, scale, sizes=None):
    """One sequence: q [n, q_heads, dim], k, v [length, kv_heads, dim] float64, chosen [n, kv_heads, list]. Returns what
    paged_ref.attend does: out, lse, sums of p |v| (of p sizes, like v), largest scale * sum |q k|."""
    sizes = v.abs() if sizes is None else sizes
    n, hq, dim = q.shape
    length, hk = k.shape[:2]
    share = hq // hk
    out, lse = torch.zeros(n, hq, dim, dtype=torch.float64), torch.full((n, hq), -math.inf, dtype=torch.float64)
    weight, size = torch.zeros_like(out), torch.zeros_like(lse)
    for i in range(n):
        p = length - n + i
        held = p // page + 1 if p >= 0 else 0
        for h in range(hk):
            keys = []
            for c in chosen[i, h, :held].tolist():
                if 0 <= c < held:
                    keys += range(c * page, min((c + 1) * page, p + 1))
            if not keys:
                continue
            kk, vv = k[keys, h], v[keys, h]
            for g in range(h * share, (h + 1) * share):
                s = kk @ q[i, g] * scale
                lse[i, g] = torch.logsumexp(s, 0)
                w = torch.exp(s - lse[i, g])
                out[i, g], weight[i, g] = w @ vv, w @ sizes[keys, h]
                size[i, g] = (kk.abs() @ q[i, g].abs() * abs(scale)).max()
    return out, lse, weight, size
