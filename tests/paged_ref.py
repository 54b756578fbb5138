"""Plain float64 definitions of the paged cache's operators, for its tests.

Written from include/ipv.h's text; shares no code with the library or its
binding. Everything works on CPU tensors.
"""
import math

import torch

GROUP = 64
LEVELS = {"u8": 255, "u4": 15}


def f16_round(x, up):
    """float64 -> the float16 value (as float64) not below (up) or not above x."""
    h = x.to(torch.float16)
    bits = h.view(torch.int16).to(torch.int32) & 0xFFFF
    key = torch.where(bits >= 0x8000, -(bits & 0x7FFF), bits)      # ordered; both zeros are 0
    key = key + torch.where(h.double() < x, 1, 0) if up else key - torch.where(h.double() > x, 1, 0)
    bits = torch.where(key < 0, (-key) | 0x8000, key)
    bits = torch.where(bits >= 0x8000, bits - 0x10000, bits)
    return bits.to(torch.int16).view(torch.float16)


def quantise(x, fmt):
    """bf16 [..., dim] -> codes int64 [..., dim], step, minimum float16 [..., groups]."""
    g = x.double().unflatten(-1, (-1, GROUP))
    good = (g.abs() <= 32768.0).all(-1)
    safe = torch.where(good[..., None], g, 0.0)
    lo, hi = safe.amin(-1), safe.amax(-1)
    m = f16_round(lo, False)
    s = f16_round((hi - m.double()) / LEVELS[fmt], True)
    sd = s.double()[..., None]
    u = torch.where(sd > 0, ((safe - m.double()[..., None]) / torch.where(sd > 0, sd, 1.0)).round(), 0.0)
    u = torch.where(good[..., None], u.clamp(0, LEVELS[fmt]), 0.0).long()
    nan = torch.full_like(s, float("nan"))
    return u.flatten(-2), torch.where(good, s, nan), torch.where(good, m, nan)


def pack(u, fmt):
    """Codes [..., dim] -> stored bytes: each word of a group at the place the header gives it."""
    per = 4 if fmt == "u8" else 8
    words = GROUP // per
    out = torch.zeros(u.shape[:-1] + (u.shape[-1] // (1 if fmt == "u8" else 2),), dtype=torch.uint8)
    for c in range(u.shape[-1]):
        g, k = divmod(c % GROUP, per)
        place = (words // 4) * (g % 4) + g // 4
        byte = (c // GROUP) * words * 4 + place * 4 + (k if fmt == "u8" else k // 2)
        out[..., byte] |= (u[..., c] << (0 if fmt == "u8" else 4 * (k % 2))).to(torch.uint8)
    return out


def values(u, s, m):
    """What codes stand for, float64."""
    g = u.double().unflatten(-1, (-1, GROUP))
    return (g * s.double()[..., None] + m.double()[..., None]).flatten(-2)


def sees(length, n, causal, window, sinks):
    """bool [n, length]: which rows each of the last n positions sees."""
    p = torch.arange(length - n, length)[:, None]
    j = torch.arange(length)[None, :]
    if not causal:
        return torch.ones((n, length), dtype=torch.bool)
    ok = j <= p
    if window:
        ok = ok & ((j > p - window) | (j < sinks))
    return ok


def attend(q, k, v, scale, causal=True, window=0, sinks=0):
    """One sequence: q [n, q_heads, dim], k, v [length, kv_heads, dim], float64.
    Returns out, lse, and the two sums that error bounds are made of: sum of
    p |v| per output, and the largest scale * sum |q k| over visible rows per query."""
    n, hq, dim = q.shape
    length, hk = k.shape[:2]
    share = hq // hk
    ok = sees(length, n, causal, window, sinks)
    out, lse = torch.zeros(n, hq, dim, dtype=torch.float64), torch.full((n, hq), -math.inf, dtype=torch.float64)
    weight, size = torch.zeros_like(out), torch.zeros_like(lse)
    if length == 0 or n == 0:
        return out, lse, weight, size
    some = ok.any(-1)
    for h in range(hq):
        kk, vv = k[:, h // share], v[:, h // share]
        s = (q[:, h] @ kk.T * scale).masked_fill(~ok, -math.inf)
        lse[:, h] = torch.logsumexp(s, -1)
        p = torch.exp(s - torch.where(some, lse[:, h], 0.0)[:, None])
        # a row that nobody of a query sees does not matter, whatever it holds
        out[:, h] = torch.where(some[:, None], p @ vv, 0.0)
        weight[:, h] = p @ vv.abs()
        size[:, h] = (q[:, h].abs() @ kk.abs().T * abs(scale)).masked_fill(~ok, 0.0).amax(-1)
    return out, lse, weight, size
