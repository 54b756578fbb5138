"""Rotated writes, bounds of pages, chosen pages, attention over them, copies and gathers on the GPU against plain
float64 definitions.

Bounds, choices and moves are whole numbers and copies: equal to the bit. Attention keeps to test_gpu_paged.py's
bounds, and over codes 2^-11 sum p (v - m) more: there it is p times the group's step s that is rounded to fp16, off by
up to 2^-11 p s, and it stands before the code u, with v = s u + m; p m is summed in fp32. So an output is off by
2^-11 sum p s u = 2^-11 sum p (v - m), which is no multiple of sum p |v|: a v near 0 in a group that reaches down to m
has s u = -m. (One of 8 heads over 9 rows, v between -3 and 3, was off by 1.16 times the bound without this term; p s
rounded to 11 bits by hand, the rest in float64, gives the same 1.159307468788775.) A rotated value is rounded once to bf16, 2^-8 of it; before that fp32: a sum of up to 128 squares is off by
128 * 2^-24 of itself, its square root by half of that, and the few products and the reciprocal square root (2 ulp)
by 2^-21 together: 2^-16 of the two products' magnitudes covers them."""
import math

import pytest

torch = pytest.importorskip("torch")

import chosen_ref as cref  # noqa: E402
import paged_ref as ref  # noqa: E402
from paper_2506_15745_gb300 import ipv  # noqa: E402
from paper_2506_15745_gb300.cache import PingPongCache  # noqa: E402
from paper_2506_15745_gb300.paged import PageBounds, PagedBatch, PagedCache, Rotary  # noqa: E402
from paper_2506_15745_gb300.sequences import Sequences  # noqa: E402
from test_gpu_paged import Setup, bounds, make_rows  # noqa: E402

pytestmark = pytest.mark.gpu


def ints(*x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def same_bits(a, b):
    return torch.equal(a.cpu().contiguous().view(torch.uint8), b.cpu().contiguous().view(torch.uint8))


def parts(cache):
    return [t for t in (cache.k, cache.v, cache.k_par, cache.v_par) if t is not None]


# ------------------------------------------------------------------- bounds of pages
def held_keys(cache, page, head, rows):
    """Keys of a page as `read` gives them, bf16."""
    if cache.fmt == "bf16":
        return cache.k[page, head, :rows].cpu()
    per = 4 if cache.fmt == "u8" else 8
    b, par = cache.k[page, head, :rows].cpu(), cache.k_par[page, head, :rows].cpu()
    u = torch.zeros((rows, cache.head_dim), dtype=torch.long)
    words = 64 // per
    for c in range(cache.head_dim):
        g, k = divmod(c % 64, per)
        byte = (c // 64) * words * 4 + ((words // 4) * (g % 4) + g // 4) * 4 + (k if per == 4 else k // 2)
        u[:, c] = b[:, byte].long() if per == 4 else (b[:, byte].long() >> (4 * (k % 2))) & 15
    return ref.values(u, par[..., 0], par[..., 1]).float().bfloat16()


def check_bounds(made, cache, pages):
    """pages: (page, rows held) that are up to date; all others are as they were, filled with 77."""
    codes, steps = made.codes.cpu(), made.steps.cpu()
    want_codes, want_steps = torch.full_like(codes, 77), torch.full_like(steps, 77.0)
    for page, rows in pages:
        for h in range(cache.n_kv_heads):
            lo, hi, step = cref.bounds(held_keys(cache, page, h, rows))
            want_codes[page, h] = 0
            want_steps[page, h] = step
            if not math.isnan(step):
                want_codes[page, h, 0, :cache.head_dim], want_codes[page, h, 1, :cache.head_dim] = lo, hi
    assert torch.equal(steps.nan_to_num(-1.0), want_steps.nan_to_num(-1.0))
    assert torch.equal(codes, want_codes)


def new_bounds(cache):
    made = PageBounds(cache)
    made.codes.fill_(77), made.steps.fill_(77.0)
    return made


BOUNDS = [  # fmt, dim, heads, page, [(rows, kv)]
    ("bf16", 128, 2, 16, [(1, 1), (0, 5), (17, 40), (33, 33), (1, 16), (1, 17), (16, 32)]),
    ("bf16", 8, 3, 32, [(1, 70), (64, 64)]),
    ("bf16", 64, 1, 128, [(1, 1), (300, 1000)]),
    ("bf16", 72, 1, 256, [(200, 700)]),
    ("bf16", 120, 5, 16, [(3, 3)] * 9),
    ("u8", 128, 2, 64, [(1, 65), (130, 200), (0, 0)]),
    ("u8", 64, 3, 16, [(40, 40), (1, 7)]),
    ("u4", 128, 1, 32, [(1, 31), (64, 129)]),
    ("u4", 64, 2, 128, [(129, 129)]),
]


@pytest.mark.parametrize("fmt,dim,heads,page,seqs", BOUNDS)
def test_bounds(fmt, dim, heads, page, seqs):
    gen = torch.Generator().manual_seed(dim + page)
    s = Setup(gen, fmt, heads, dim, page, [n for _, n in seqs], [r for r, _ in seqs])  # NaN behind the last rows
    made = new_bounds(s.cache)
    made.update(s.cache, s.batch)
    pages = []
    for b, (n, length) in enumerate(seqs):
        if n:
            pages += [(int(s.table[b, i]), min(page, length - i * page)) for i in range((length - n) // page, (length - 1) // page + 1)]
    check_bounds(made, s.cache, pages)


def test_bounds_of_special_keys():
    """Zeros of both signs, tiny and huge magnitudes, ends of the 8-bit range, NaN and infinities."""
    cache = PagedCache(12, 16, 1, 64)
    x = torch.zeros(12, 16, 64)
    x[1] = -0.0
    x[2] = torch.randn(16, 64, generator=torch.Generator().manual_seed(1)) * 2.0 ** -45   # below the smallest step
    x[3, :, 0] = 2.0 ** -126
    x[4, 3, 5] = -(2.0 ** -133)                                                       # a bf16 subnormal
    x[5] = torch.randn(16, 64, generator=torch.Generator().manual_seed(2)) * 1e30
    x[6, 0, 0], x[6, 0, 1] = 127.0, -127.0
    x[7, 0, 0], x[7, 0, 1] = 127.5, -1e-20
    x[8, 5, 9] = float("nan")
    x[9, 15, 63] = float("inf")
    x[10, 0, 0] = -float("inf")
    x[11, 2, 2] = torch.finfo(torch.bfloat16).max
    cache.k[:, 0] = x.bfloat16().cuda()
    made = new_bounds(cache)
    made.update(cache, PagedBatch(torch.arange(12, dtype=torch.int32, device="cuda")[None], ints(0, 192), ints(192), total_rows=192,
                                  max_rows=192, max_kv=192))
    check_bounds(made, cache, [(p, 16) for p in range(12)])
    steps = made.steps.cpu()[:, 0]
    assert torch.isnan(steps[8:11]).all() and torch.isfinite(steps[[0, 1, 2, 3, 4, 5, 6, 7, 11]]).all()
    k, lo, hi = x.bfloat16().double(), *made.codes.cpu()[:, 0].double().unbind(1)
    for p in (0, 1, 2, 3, 4, 5, 6, 7, 11):  # what they are for
        assert (k[p] >= lo[p] * steps[p].double()).all() and (k[p] <= hi[p] * steps[p].double()).all(), p


def test_bounds_where_the_batch_is_unusual():
    """Pages outside the pool, more new rows than rows."""
    gen = torch.Generator().manual_seed(8)
    cache = PagedCache(4, 16, 2, 64)
    cache.k.copy_(make_rows(gen, 4, 2, 16, 64).cuda())
    made = new_bounds(cache)
    batch = PagedBatch(ints(3, 99, -1, 1, 2, 0).view(3, 2), ints(0, 20, 30, 60), ints(32, 20, 5), total_rows=60, max_rows=30, max_kv=32)
    made.update(cache, batch)
    check_bounds(made, cache, [(3, 16), (1, 4), (2, 5)])


def test_bounds_of_one_page_per_sequence():
    """Without a table, of a strided pool."""
    gen = torch.Generator().manual_seed(9)
    wide = make_rows(gen, 3, 300, 2, 128).cuda()
    k = wide.permute(0, 2, 1, 3)
    cache = PagedCache.from_tensors("bf16", k, k.clone(memory_format=torch.preserve_format))
    made = new_bounds(cache)
    made.update(cache, PagedBatch(None, ints(0, 1, 1, 71), ints(300, 200, 99), total_rows=71, max_rows=70, max_kv=300))
    check_bounds(made, cache, [(0, 300), (2, 99)])


# ------------------------------------------------------------------- the choice
class Choice:
    """Sequences of (rows, kv), bounds of random pages, queries."""

    def __init__(self, seed, seqs, heads, share, dim, page, levels=60, special=True):
        gen = self.gen = torch.Generator().manual_seed(seed)
        self.seqs, self.heads, self.share, self.dim, self.page = seqs, heads, share, dim, page
        padded = 64 if dim <= 64 else 128
        held = [-(-n // page) for _, n in seqs]
        n_pages = sum(held) + 2
        order, at = torch.randperm(n_pages, generator=gen).to(torch.int32), 0
        self.table = torch.full((len(seqs), max(1, max(held))), -1, dtype=torch.int32)
        for b, n in enumerate(held):
            self.table[b, :n] = order[at:at + n]
            at += n
        x = torch.randint(-levels, levels + 1, (2, n_pages, heads, dim), generator=gen)
        self.codes = torch.zeros((n_pages, heads, 2, padded), dtype=torch.int8)
        self.codes[:, :, 0, :dim], self.codes[:, :, 1, :dim] = x.amin(0).to(torch.int8), x.amax(0).to(torch.int8)
        self.steps = 2.0 ** torch.randint(-9, -5, (n_pages, heads), generator=gen).float()
        self.q = (torch.randn((sum(r for r, _ in seqs), heads * share, dim), generator=gen) * 1.5).bfloat16()
        if special and n_pages > 8:
            self.steps[int(order[3]), 0] = math.nan
            self.steps[int(order[5])] = 0.0
            self.table[0, 1] = n_pages + 5  # no page of the pool

    def run(self, n, first, recent, out=None, **kw):
        heads, page = self.heads, self.page
        rows = [r for r, _ in self.seqs]
        self.start = [0]
        for r in rows:
            self.start.append(self.start[-1] + r)
        self.made = PageBounds.from_tensors(self.codes.cuda(), self.steps.cuda(), page, self.dim)
        self.batch = PagedBatch(self.table.cuda(), ints(*self.start), ints(*[k for _, k in self.seqs]), total_rows=self.start[-1],
                                max_rows=max(rows), max_kv=max(k for _, k in self.seqs))
        got = self.made.choose(self.q.cuda(), self.batch, n, first=first, recent=recent, out=out, **kw)
        assert got.shape == (self.start[-1], heads, n)
        return got

    def want(self, n, first, recent, rows=None):
        """[total_rows, heads, n]; of every sequence the new rows `rows` (all if None), others -2."""
        out = torch.full((self.start[-1], self.heads, n), -2, dtype=torch.int32)
        for b, (r, length) in enumerate(self.seqs):
            for i in range(r) if rows is None else [j for j in rows if j < r]:
                p = length - r + i
                pages = p // self.page + 1 if p >= 0 else 0
                g = self.table[b, :pages].long()
                ok = (g >= 0) & (g < self.codes.shape[0])
                safe = torch.where(ok, g, 0)
                for h in range(self.heads):
                    step = torch.where(ok, self.steps[safe, h].double(), math.nan)
                    lo, hi = self.codes[safe, h, :, :self.dim].long().unbind(1)
                    s = cref.scores(self.q[self.start[b] + i, h * self.share:(h + 1) * self.share], lo, hi, step) if pages > n else torch.zeros(pages)
                    out[self.start[b] + i, h] = torch.tensor(cref.choose(s, n, first, recent), dtype=torch.int32)
        return out


CHOICES = [  # sequences, heads, share, dim, page, n, first, recent
    ([(1, 300)], 2, 7, 128, 16, 8, 1, 2),
    ([(1, 16 * n) for n in (1, 2, 7, 8, 9, 10, 30)] + [(1, 129), (1, 145), (1, 0), (0, 200)], 2, 4, 64, 16, 8, 1, 1),
    ([(1, 5000), (3, 4100), (20, 2300)], 1, 1, 128, 16, 24, 0, 1),
    ([(1, 20000)], 1, 8, 128, 16, 64, 3, 2),                  # a cluster of 8 blocks
    ([(1, 9000), (1, 33)], 3, 3, 64, 16, 33, 1, 1),
    ([(5, 5), (40, 50), (9, 200)], 2, 16, 80, 16, 4, 2, 2),   # nothing scored is chosen
    ([(2, 1000)], 1, 64, 128, 16, 10, 1, 3),                  # 8 head tiles
    ([(3, 700)], 4, 5, 8, 32, 1, 0, 1),                       # the row's own page alone
    ([(2, 4000)], 1, 2, 72, 256, 3, 1, 1),
    ([(4, 3000)], 1, 9, 96, 16, 150, 1, 2),
    ([(1, 16 * 1024)], 1, 3, 128, 16, 700, 1, 2),             # more chosen than threads
]


@pytest.mark.parametrize("case", range(len(CHOICES)))
@pytest.mark.parametrize("levels", [60, 1])                   # 1: many equal scores
def test_choices(case, levels):
    seqs, heads, share, dim, page, n, first, recent = CHOICES[case]
    c = Choice(100 + case, seqs, heads, share, dim, page, levels)
    got = c.run(n, first, recent).cpu()
    assert torch.equal(got, c.want(n, first, recent))


@pytest.mark.parametrize("equal", ["all", "two values", "no scores"])
@pytest.mark.parametrize("pages", [40, 256, 258, 259, 600, 3000])
def test_equal_scores_go_to_the_lower_page(equal, pages):
    c = Choice(7, [(1, 16 * pages)], 1, 2, 64, 16, special=False)
    c.codes[:] = c.codes[:1]
    c.steps.fill_(1.0 if equal != "no scores" else math.nan)
    if equal == "two values":
        c.steps[c.table[0, 1::3].long()] = 2.0
    for n, first, recent in ((5, 1, 1), (30, 0, 2), (39, 2, 1)):
        assert torch.equal(c.run(n, first, recent).cpu(), c.want(n, first, recent)), n


def test_the_most_pages():
    """32768 pages of 16 rows; scores of one row, a cluster of 8 blocks."""
    c = Choice(17, [(1, 16 * 32768)], 1, 4, 64, 16)
    for n in (5, 96, 2000):
        assert torch.equal(c.run(n, 1, 1).cpu(), c.want(n, 1, 1)), n


def test_query_heads_that_do_not_count():
    """A query head with a NaN or an infinity is left out; with all of them out no page has a score; zeros, tiny, large ones."""
    c = Choice(23, [(4, 1000)], 2, 3, 128, 16)
    c.q[0, 0, 5] = math.nan
    c.q[0, 4, 100] = -math.inf
    c.q[1, :3, 0] = math.inf
    c.q[2, 0] = 0
    c.q[2, 1] *= 2.0 ** -60
    c.q[2, 2] *= 2.0 ** 40
    c.q[3, 3:] = -0.0
    assert torch.equal(c.run(9, 1, 2).cpu(), c.want(9, 1, 2))


def test_choices_leave_others_rows_alone():
    """Packed rows of no sequence, lists inside a wider tensor, rows before position 0."""
    c = Choice(29, [(3, 500), (30, 20)], 2, 2, 64, 16, special=False)
    wide = torch.full((2, 40, 9), -5, dtype=torch.int32, device="cuda")
    got = c.run(7, 1, 1)
    starts = c.batch
    c.q = torch.cat([c.q, c.q[:7]])
    batch = PagedBatch(starts.table, starts.row_start, starts.kv_len, total_rows=40, max_rows=30, max_kv=500)
    out = wide.transpose(0, 1)[..., 1:8]
    c.made.choose(c.q.cuda(), batch, 7, first=1, recent=1, out=out)
    assert torch.equal(out[:33], got) and (out[33:] == -5).all() and (wide[..., 0] == -5).all() and (wide[..., 8] == -5).all()
    assert torch.equal(got.cpu(), c.want(7, 1, 1)) and (got[3:13] == -1).all()
    again = c.made.choose(c.q.cuda(), batch, 7, first=1, recent=1)
    assert (again[33:] == -1).all()


def test_a_choice_promises_no_less_than_any_product():
    """Over keys that were really there: the score of a page is at least the largest q . k of it but for q's rounding,
    half a step of 8 bits in each channel."""
    gen = torch.Generator().manual_seed(37)
    s = Setup(gen, "bf16", 1, 128, 16, [640], [640])
    made = PageBounds(s.cache)
    made.update(s.cache, s.batch)
    q = make_rows(gen, 1, 4, 128)
    g = s.table[0].long()
    lo, hi = made.codes.cpu()[g, 0].long().unbind(1)
    score = cref.scores(q[0], lo, hi, made.steps.cpu()[g, 0].double())
    k = s.k[0][:, 0].view(40, 16, 128)
    best = torch.einsum("prd,hd->prh", k, q[0].double()).amax((1, 2))
    up = max(2.0 ** cref.exponent(float(x.abs().max())) for x in q[0])
    assert (score >= best - 0.5 * up * k.abs().sum(-1).amax(1)).all()


# ------------------------------------------------------------------- attention over chosen pages
def random_lists(gen, s, n, junk=False):
    out = torch.full((s.total, s.heads, n), -1, dtype=torch.int32)
    for b, (r, length) in enumerate(zip(s.rows, s.lens)):
        for i in range(r):
            p = length - r + i
            held = p // s.page + 1 if p >= 0 else 0
            for h in range(s.heads):
                x = torch.randperm(held, generator=gen)[:n].sort().values.to(torch.int32)
                out[int(s.start[b]) + i, h, :len(x)] = x
    if junk:  # no pages, in any places; and pages twice
        bad = torch.rand(out.shape, generator=gen)
        out[bad < 0.15] = -1
        out[(bad > 0.15) & (bad < 0.25)] = 1 << 30
        out[(bad > 0.25) & (bad < 0.3)] = -(1 << 31)
        out[(bad > 0.3) & (bad < 0.4)] = 0
    return out


def above_minimum(cache, v, pages):
    """v - m of a sequence's rows v [length, heads, dim] in these pages: its codes times their steps. 0 over bf16."""
    if cache.fmt == "bf16":
        return torch.zeros_like(v)
    j = torch.arange(v.shape[0])
    m = cache.v_par.cpu()[pages[j // cache.page_size].long(), :, j % cache.page_size, :, 1].double()
    return v - m.repeat_interleave(64, -1)


def check_chosen(s, q, chosen, got, lse, scale):
    got, lse = got.double().cpu(), lse.double().cpu()
    for b, (n, length) in enumerate(zip(s.rows, s.lens)):
        at = slice(int(s.start[b]), int(s.start[b + 1]))
        o, l, weight, size = cref.attend(q[at].double(), s.k[b], s.v[b], chosen[at], s.page, scale)
        vmax = float(s.v[b].abs().max()) if length else 0.0
        tol = bounds(s.fmt, weight, size, o, min(length, chosen.shape[2] * s.page), vmax)
        if s.fmt != "bf16":
            tol = tol + 2.0 ** -11 * cref.attend(q[at].double(), s.k[b], s.v[b], chosen[at], s.page, scale,
                                                 above_minimum(s.cache, s.v[b], s.table[b]))[2]
        off = (got[at] - o).abs()
        assert torch.isfinite(got[at]).all(), (b, n, length)
        assert (off <= tol).all(), (b, n, length, float((off / tol.clamp(min=1e-30)).max()))
        empty = torch.isinf(l)
        assert torch.equal(lse[at][empty], l[empty]) and (got[at][empty] == 0).all()
        ltol = (size * (2.0 ** -16 if s.fmt == "bf16" else 2.0 ** -11 + 2.0 ** -16) + 2.0 ** -20 * (1 + l.abs()))[~empty]
        assert ((lse[at] - l)[~empty].abs() <= ltol).all(), (b, n, length)


def run_chosen(s, share, chosen, seed, **kw):
    gen = torch.Generator().manual_seed(seed)
    q = (torch.randn((s.total, s.heads * share, s.dim), generator=gen) * 1.5).bfloat16()
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    s.cache.attend_chosen(q.cuda(), s.batch, chosen.cuda(), out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    return q, out, lse


CHOSEN = [  # fmt, dim, heads, share, page, [(rows, kv)], n
    ("bf16", 128, 2, 7, 16, [(1, 1), (1, 15), (1, 16), (1, 17), (1, 33), (1, 0), (0, 9), (1, 700)], 5),
    ("bf16", 128, 1, 8, 64, [(1, 6000)], 32),                      # one list over a cluster
    ("bf16", 128, 2, 8, 64, [(9, 3000), (2, 70), (20, 20)], 12),
    ("bf16", 128, 4, 4, 16, [(40, 900)] * 6, 7),                   # tiles taken whole, in turn
    ("bf16", 128, 8, 1, 128, [(1, 2000)] * 20, 3),
    ("bf16", 128, 1, 16, 32, [(3, 500)], 9),                       # two tiles of query heads, or one of 16
    ("bf16", 128, 1, 19, 32, [(3, 500), (1, 2)], 9),
    ("bf16", 64, 2, 3, 16, [(5, 400), (1, 16)], 40),               # longer than any row's pages
    ("bf16", 80, 2, 5, 32, [(3, 300)], 4),
    ("bf16", 8, 1, 2, 16, [(2, 100)], 3),
    ("bf16", 120, 3, 4, 256, [(2, 2000)], 2),
    ("u8", 128, 2, 7, 64, [(1, 2500), (1, 10), (3, 700)], 9),
    ("u8", 64, 4, 2, 16, [(1, 300), (1, 77), (7, 9)], 6),
    ("u8", 128, 1, 8, 32, [(30, 800)] * 3, 11),
    ("u4", 128, 2, 8, 32, [(1, 2500), (1, 10), (2, 700)], 20),
    ("u4", 64, 1, 4, 16, [(60, 600)] * 5, 8),
    ("u4", 128, 3, 5, 128, [(1, 4000)] * 9, 6),
    ("bf16", 128, 1, 1, 16, [(1, 30000)], 1500),                   # a list of 24000 keys
    ("u4", 64, 1, 2, 16, [(1, 30000), (1, 300)], 1500),
    ("bf16", 128, 1, 2, 16, [(1, 50 + (b * 37) % 300) for b in range(300)], 4),
    # Longer than a block takes whole, in numbers that go to clusters of 4, of 2, to blocks one by one, to all in shares, to blocks in turn.
    ("bf16", 128, 2, 7, 16, [(3, 900), (2, 700), (3, 20)], 40),
    ("bf16", 128, 4, 7, 16, [(4, 900), (1, 700), (2, 30)], 40),
    ("bf16", 128, 4, 2, 16, [(3, 900), (2, 700), (0, 100), (3, 2), (3, 1000), (3, 640), (3, 641), (3, 639)], 40),
    ("bf16", 128, 4, 4, 16, [(5, 900 - 80 * b) for b in range(10)], 40),
    ("bf16", 128, 4, 4, 16, [(20, 700)] * 6 + [(0, 5), (1, 3), (0, 0), (20, 900)], 40),
    ("u4", 128, 2, 8, 32, [(9, 2000 - 600 * b) for b in range(4)], 30),
    ("u4", 128, 4, 3, 32, [(9, 2000 - 600 * b) for b in range(4)], 30),
    ("u8", 128, 4, 3, 32, [(9, 2000 - 300 * b) for b in range(6)], 20),
    ("u4", 64, 1, 3, 16, [(1, 600 + (b * 29) % 300) for b in range(500)], 40),
    ("bf16", 64, 1, 2, 16, [(1, 600 + (b * 31) % 300) for b in range(600)], 36),
    ("bf16", 128, 1, 2, 16, [((b % 5) // 4 + (b % 7 > 0), 600 + (b * 31) % 300) for b in range(800)], 36),
]


@pytest.mark.parametrize("junk", [False, True])
@pytest.mark.parametrize("case", range(len(CHOSEN)))
def test_attend_chosen(case, junk):
    fmt, dim, heads, share, page, seqs, n = CHOSEN[case]
    gen = torch.Generator().manual_seed(500 + case)
    s = Setup(gen, fmt, heads, dim, page, [k for _, k in seqs], [r for r, _ in seqs])  # NaN in rows that nobody holds
    chosen = random_lists(gen, s, n, junk)
    q, out, lse = run_chosen(s, share, chosen, 600 + case)
    check_chosen(s, q, chosen, out, lse, dim ** -0.5)


@pytest.mark.parametrize("fmt", ["bf16", "u8", "u4"])
def test_all_pages_chosen_is_attention(fmt):
    """Lists of all pages: what attend gives within both bounds, and more new rows than cached ones."""
    gen = torch.Generator().manual_seed(43)
    s = Setup(gen, fmt, 2, 128, 16, [300, 5, 40], [3, 9, 0])
    chosen = torch.arange(20, dtype=torch.int32).expand(s.total, 2, 20)
    q, out, lse = run_chosen(s, 4, chosen, 44)
    check_chosen(s, q, chosen, out, lse, 128 ** -0.5)
    assert (lse[3:7] == -math.inf).all() and (out[3:7] == 0).all()


@pytest.mark.parametrize("scale", [0.0, -0.1, 2.0 ** -40])
def test_scales(scale):
    gen = torch.Generator().manual_seed(47)
    for fmt in ("bf16", "u4"):
        s = Setup(gen, fmt, 2, 128, 16, [200, 90], [1, 6])
        chosen = random_lists(gen, s, 4)
        q, out, lse = run_chosen(s, 4, chosen, 48, scale=scale)
        check_chosen(s, q, chosen, out, lse, scale)


def test_lists_by_strides_and_one_for_all_heads():
    gen = torch.Generator().manual_seed(53)
    s = Setup(gen, "bf16", 2, 128, 16, [400, 60], [2, 3])
    lists = random_lists(gen, s, 5)
    wide = torch.full((2, s.total, 9), 3, dtype=torch.int32)
    wide[..., 2:7] = lists.transpose(0, 1)
    q, out, lse = run_chosen(s, 4, wide.transpose(0, 1)[..., 2:7], 54)
    check_chosen(s, q, lists, out, lse, 128 ** -0.5)
    one = lists[:, :1].cuda().expand(s.total, 2, 5)
    q, out, lse = run_chosen(s, 4, one, 54)
    check_chosen(s, q, one.cpu(), out, lse, 128 ** -0.5)


@pytest.mark.parametrize("rows", [1, 90])  # a cluster or a block for each list; blocks in turn
def test_rows_of_no_sequence_are_left_alone(rows):
    gen = torch.Generator().manual_seed(55)
    s = Setup(gen, "bf16", 4, 128, 16, [700, 60, 800], [rows, 0, rows])
    chosen = random_lists(gen, s, 40)
    more = torch.cat([chosen, chosen[:1].expand(9, 4, 40)]).cuda()
    q = make_rows(gen, s.total + 9, 8, 128)
    batch = PagedBatch(s.batch.table, s.batch.row_start, s.batch.kv_len, total_rows=s.total + 9, max_rows=rows, max_kv=800)
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    s.cache.attend_chosen(q.cuda(), batch, more, out=out, lse=lse)
    assert (out[s.total:] == 7.0).all() and (lse[s.total:] == 7.0).all()
    check_chosen(s, q[:s.total], chosen, out[:s.total], lse[:s.total], 128 ** -0.5)


def test_one_page_per_sequence():
    gen = torch.Generator().manual_seed(57)
    k, v = make_rows(gen, 3, 2, 300, 128), make_rows(gen, 3, 2, 300, 128)
    cache = PagedCache.from_tensors("bf16", k.cuda(), v.cuda())
    batch = PagedBatch(None, ints(0, 1, 3, 4), ints(300, 77, 1), total_rows=4, max_rows=2, max_kv=300)
    q = make_rows(gen, 4, 8, 128)
    chosen = torch.tensor([[[0, -1]]], dtype=torch.int32).expand(4, 2, 2)
    lse = torch.zeros(4, 8, device="cuda")
    out = cache.attend_chosen(q.cuda(), batch, chosen.contiguous().cuda(), lse=lse).double().cpu()
    for b, (a, e, n) in enumerate(((0, 1, 300), (1, 3, 77), (3, 4, 1))):
        o, l, weight, size = ref.attend(q[a:e].double(), k[b, :, :n].transpose(0, 1).double(), v[b, :, :n].transpose(0, 1).double(), 128 ** -0.5)
        assert ((out[a:e] - o).abs() <= bounds("bf16", weight, size, o, n, 0.0)).all()


def test_a_visible_nan_shows_and_an_unchosen_one_does_not():
    gen = torch.Generator().manual_seed(59)
    s = Setup(gen, "bf16", 1, 128, 16, [100], [1])
    s.cache.k[int(s.table[0, 2])] = math.nan
    s.cache.v[int(s.table[0, 4])] = math.inf
    chosen = torch.tensor([[[0, 1, 3, 6]]], dtype=torch.int32)
    q, out, lse = run_chosen(s, 4, chosen, 60)
    check_chosen(s, q, chosen, out, lse, 128 ** -0.5)
    for page in (2, 4):
        _, out, lse = run_chosen(s, 4, torch.tensor([[[0, page, 6, -1]]], dtype=torch.int32), 60)
        assert not torch.isfinite(out).any()


def test_pages_of_the_pool_past_32_bits():
    """As in the dense attention's test: pages more than 4 GiB apart."""
    page, dim = 64, 128
    gen = torch.Generator().manual_seed(61)
    base = torch.zeros((3, 1 << 30), dtype=torch.bfloat16, device="cuda")
    shape, strides = (3, 1, page, dim), (1 << 30, page * dim, dim, 1)
    cache = PagedCache.from_tensors("bf16", base.as_strided(shape, strides), base.as_strided(shape, strides, 1 << 29))
    n = 180
    batch = PagedBatch(ints(2, 0, 1)[None], ints(0, n), ints(n), total_rows=n, max_rows=n, max_kv=192)
    k, v, q = (make_rows(gen, n, h, dim) for h in (1, 1, 4))
    rotary = Rotary(torch.cat([torch.ones(4, 64), torch.zeros(4, 64)], 1).cuda())  # no turn at all
    assert same_bits(cache.write_rotated(q.cuda(), k.cuda(), v.cuda(), batch, rotary, ints(*[i % 4 for i in range(n)])), q)
    assert torch.equal(cache.k[2, 0].cpu(), k[:64, 0]) and torch.equal(cache.v[1, 0, :52].cpu(), v[128:, 0])
    made = PageBounds(cache)
    made.update(cache, batch)
    for at, rows in ((2, 64), (0, 64), (1, 52)):
        lo, hi, step = cref.bounds(cache.k[at, 0, :rows].cpu())
        assert torch.equal(made.codes[at, 0].cpu(), torch.stack([lo, hi]).to(torch.int8)) and float(made.steps[at, 0]) == step
    chosen = torch.tensor([[[0, 2]]], dtype=torch.int32).expand(n, 1, 2)
    lse = torch.zeros((n, 4), device="cuda")
    out = cache.attend_chosen(q.cuda(), batch, chosen.cuda(), lse=lse).double().cpu()
    o, l, weight, size = cref.attend(q.double(), k.double(), v.double(), chosen, page, dim ** -0.5)
    assert ((out - o).abs() <= bounds("bf16", weight, size, o, 128, 0.0)).all()
    cache.copy_pages(ints(2), ints(1))
    assert torch.equal(cache.k[1], cache.k[2]) and torch.equal(cache.v[1], cache.v[2])
    del out, base


# ------------------------------------------------------------------- rotated writes
ROTATED = [  # fmt, dim, heads, share, page, [(rows, kv)], rot, sections, interleaved, norms (q, k)
    ("bf16", 128, 4, 7, 64, [(1, 1), (0, 5), (17, 40), (33, 33)], 128, [32, 16, 16], False, "qk"),
    ("bf16", 128, 2, 1, 16, [(5, 70)], 128, [64], False, ""),
    ("bf16", 128, 1, 3, 16, [(5, 70)], 64, [8, 8, 8, 8], False, "q"),
    ("bf16", 128, 3, 2, 16, [(5, 70)], 128, [24, 40], True, "k"),
    ("bf16", 80, 2, 5, 32, [(9, 9), (1, 100)], 80, [40], False, "qk"),
    ("bf16", 96, 1, 2, 32, [(9, 9), (1, 100)], 48, [8, 16], True, "qk"),
    ("bf16", 64, 5, 1, 16, [(20, 20)], 64, [32], False, "k"),
    ("bf16", 16, 1, 1, 16, [(3, 5)], 16, [8], False, "qk"),
    ("bf16", 128, 8, 16, 128, [(2, 500)], 32, [16], False, ""),
    ("bf16", 64, 1, 2, 16, [(1, 1 + b) for b in range(70)] + [(0, 4), (0, 4), (3, 3)], 64, [32], True, ""),  # more sequences than lanes
    ("u8", 128, 4, 7, 64, [(1, 65), (30, 200)], 128, [32, 16, 16], False, "qk"),
    ("u8", 64, 3, 2, 16, [(7, 7)], 32, [16], True, "k"),
    ("u4", 128, 1, 4, 16, [(7, 40), (1, 1)], 128, [64], False, ""),
    ("u4", 64, 2, 3, 32, [(60, 60)], 64, [16, 16], False, "q"),
    ("u4", 128, 3, 3, 32, [(11, 60)], 96, [48], True, "qk"),
]


def turns(gen, n, rot):
    a = torch.rand((n, rot // 2), generator=gen, dtype=torch.float64) * 2 * math.pi
    return torch.cat([a.cos(), a.sin()], 1).float()


@pytest.mark.parametrize("case", range(len(ROTATED)))
def test_write_rotated(case):
    fmt, dim, heads, share, page, seqs, rot, sections, interleaved, norms = ROTATED[case]
    gen = torch.Generator().manual_seed(700 + case)
    rows, lens = [r for r, _ in seqs], [n for _, n in seqs]
    s = Setup(gen, fmt, heads, dim, page, lens, rows, garbage=False)
    q, k, v = make_rows(gen, s.total, heads * share, dim), make_rows(gen, s.total, heads, dim), make_rows(gen, s.total, heads, dim)
    w = {x: (1 + 0.3 * torch.randn(dim, generator=gen)).bfloat16() if x in norms else None for x in "qk"}
    table, at = turns(gen, 50, rot), torch.randint(0, 50, (len(sections), s.total), generator=gen, dtype=torch.int32)
    on = lambda t: None if t is None else t.cuda()  # noqa: E731
    rotary = Rotary(table.cuda(), sections, interleaved)
    before = [t.clone() for t in parts(s.cache)]
    got = s.cache.write_rotated(q.cuda(), k.cuda(), v.cuda(), s.batch, rotary, at.cuda(), q_weight=on(w["q"]), k_weight=on(w["k"]), eps=1e-3)
    made = {}
    for name, x in (("q", q), ("k", k)):
        want, size = cref.turned(x, w[name], 1e-3, table, at, sections, interleaved)
        tol = 2.0 ** -8 * want.abs() + 2.0 ** -16 * size + 1e-38
        made[name] = want, tol
    assert ((got.double().cpu() - made["q"][0]).abs() <= made["q"][1]).all()
    # The same rows through a bf16 pool: its keys are within bounds, and what codes hold is `write` of exactly these.
    plain = PagedCache(s.cache.n_pages, page, heads, dim)
    plain.write_rotated(q.cuda(), k.cuda(), v.cuda(), s.batch, rotary, at.cuda(), q_weight=on(w["q"]), k_weight=on(w["k"]), eps=1e-3)
    k_back, v_back = plain.read(s.batch)
    assert ((k_back.double().cpu() - made["k"][0]).abs() <= made["k"][1]).all() and same_bits(v_back, v)
    after = [t.clone() for t in parts(s.cache)]
    for t, old in zip(parts(s.cache), before):
        t.copy_(old)
    s.cache.write(k_back, v_back, s.batch)
    assert all(same_bits(a, t) for a, t in zip(after, parts(s.cache)))  # the whole pool: nothing else was touched


def test_rotated_in_place_and_by_strides():
    """Queries, keys and values as slices of one projection's rows; q rotated where it is."""
    gen = torch.Generator().manual_seed(67)
    s = Setup(gen, "bf16", 2, 128, 16, [50, 9], [4, 9])
    wide = make_rows(gen, s.total, 12, 128)
    table, at = turns(gen, 30, 128), torch.randint(0, 30, (s.total,), generator=gen, dtype=torch.int32)
    x = wide.cuda()
    out = s.cache.write_rotated(x[:, :8], x[:, 8:10], x[:, 10:], s.batch, Rotary(table.cuda()), at.cuda(), q_out=x[:, :8])
    assert out.data_ptr() == x.data_ptr()
    for a, e in ((0, 8), (8, 10)):
        want, size = cref.turned(wide[:, a:e], None, 0.0, table, at[None], [64], False)
        made = x[:, :8] if a == 0 else s.cache.read(s.batch)[0]
        assert ((made.double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16 * size).all()
    assert same_bits(x[:, 8:], wide[:, 8:]) and same_bits(s.cache.read(s.batch)[1], wide[:, 10:])


def test_rotated_writes_drop_what_does_not_fit():
    """As write: rows before position 0, pages outside the pool; packed rows of no sequence are left alone, queries too;
    a position outside the table makes the channels that it turns NaN."""
    gen = torch.Generator().manual_seed(71)
    q, k, v = make_rows(gen, 60, 4, 64), make_rows(gen, 60, 2, 64), make_rows(gen, 60, 2, 64)
    table = turns(gen, 20, 32)
    at = torch.randint(0, 20, (2, 60), generator=gen, dtype=torch.int32)
    at[1, 41], at[0, 42], at[1, 43] = 20, -1, -(1 << 31)
    batch = PagedBatch(ints(0, 99, -1, 1, 2, 2, 2, 2).view(4, 2), ints(0, 20, 40, 45, 90), ints(20, 20, 3, 16), total_rows=60, max_rows=20, max_kv=32)
    rotary = Rotary(table.cuda(), [8, 8])
    cache, same = PagedCache(3, 16, 2, 64), PagedCache(3, 16, 2, 64)
    for c in (cache, same):
        c.k.fill_(9.0), c.v.fill_(9.0)
    out = torch.full((60, 4, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    cache.write_rotated(q.cuda(), k.cuda(), v.cuda(), batch, rotary, at.cuda(), q_out=out)
    want, size = cref.turned(q, None, 0.0, table, at, [8, 8], False)
    got = out.double().cpu()
    assert (got[45:] == 5.0).all()
    assert torch.equal(torch.isnan(got[:45]), torch.isnan(want[:45]))
    assert ((got - want).abs()[:45].nan_to_num(0.0) <= (2.0 ** -8 * want.abs() + 2.0 ** -16 * size)[:45].nan_to_num(0.0)).all()
    assert torch.isnan(want[41:44]).any((1, 2)).all()
    want, size = cref.turned(k, None, 0.0, table, at, [8, 8], False)
    same.write(want.float().bfloat16().cuda(), v.cuda(), batch)
    assert same_bits(cache.v, same.v)
    a, b = cache.k.double().cpu(), same.k.double().cpu()
    assert torch.equal(torch.isnan(a), torch.isnan(b)) and torch.equal(a == 9.0, b == 9.0)
    # each side is rounded once, from values 2^-16 of the products apart
    assert ((a - b).abs().nan_to_num(0.0) <= (2.0 ** -7 * b.abs()).nan_to_num(0.0) + 2.0 ** -15 * float(size.nan_to_num(0.0).max())).all()


def test_norms_of_zero_and_large_rows():
    gen = torch.Generator().manual_seed(73)
    s = Setup(gen, "bf16", 1, 128, 16, [8], [8])
    q, k, v = (make_rows(gen, 8, 1, 128) for _ in range(3))
    q[0], k[1] = 0, 0
    q[2] *= 2.0 ** 50
    k[3] *= 2.0 ** -50
    q[4, 0, 7] = math.inf
    k[5, 0, 9] = math.nan
    w = make_rows(gen, 128, spread=False)
    table, at = turns(gen, 9, 128), torch.arange(8, dtype=torch.int32)[None]
    out = s.cache.write_rotated(q.cuda(), k.cuda(), v.cuda(), s.batch, Rotary(table.cuda()), at.cuda(), q_weight=w.cuda(), k_weight=w.cuda())
    for x, made in ((q, out), (k, s.cache.read(s.batch)[0])):
        want, size = cref.turned(x, w, 1e-6, table, at, [64], False)
        made = made.double().cpu()
        fine = torch.isfinite(x.double()).all(-1)[:, 0]
        assert ((made - want).abs()[fine] <= (2.0 ** -8 * want.abs() + 2.0 ** -16 * size + 1e-38)[fine]).all()
        assert torch.isnan(made[~fine]).any()


def test_a_table_of_angles():
    r = Rotary.of_base(10000.0, 500, 64)
    a = 499.0 * 10000.0 ** (-2.0 * 3 / 64)
    assert abs(float(r.table[499, 3]) - math.cos(a)) <= 2.0 ** -24 and abs(float(r.table[499, 35]) - math.sin(a)) <= 2.0 ** -24
    assert r.sections == [32] and not r.interleaved


# ------------------------------------------------------------------- copies and gathers
@pytest.mark.parametrize("fmt,dim,heads,page", [("bf16", 128, 4, 64), ("bf16", 8, 1, 16), ("bf16", 72, 3, 48), ("bf16", 120, 112, 16), ("u8", 128, 2, 16),
                                                ("u8", 64, 5, 128), ("u4", 128, 3, 32), ("u4", 64, 1, 16), ("bf16", 128, 1, 9408)])
@pytest.mark.parametrize("rows_first", [False, True])
def test_copies(fmt, dim, heads, page, rows_first):
    gen = torch.Generator().manual_seed(dim + heads)
    cache = PagedCache(9, page, heads, dim, fmt)
    if rows_first:  # a pool laid out [page][row][head]
        cache = PagedCache.from_tensors(fmt, *(None if t is None else t.transpose(1, 2).contiguous().transpose(1, 2)
                                               for t in (cache.k, cache.v, cache.k_par, cache.v_par)))
    for t in parts(cache):
        t.copy_(torch.randint(-120, 120, t.shape, generator=gen).to(t.dtype).cuda())
    want = [t.clone() for t in parts(cache)]
    source, target = [3, 3, 8, 99, 1, -1], [0, 7, 5, 4, 9, 6]
    for t in want:
        for a, b in zip(source[:3], target[:3]):
            t[b] = t[a]
    cache.copy_pages(ints(*source), ints(*target))
    assert all(same_bits(a, b) for a, b in zip(parts(cache), want))
    cache.copy_pages(ints(), ints())
    cache.copy_pages(ints(2), ints(2))  # onto itself
    assert all(same_bits(a, b) for a, b in zip(parts(cache), want))


def gathered(s, to_table, to_rows, to_lens, to_page, kept, target):
    """What the target's tensors hold after the gather, moved row by row."""
    want = [t.cpu().clone() for t in parts(target)]
    for t, old in zip(want, parts(s.cache)):
        old = old.cpu()
        for b, (r, length) in enumerate(zip(to_rows, to_lens)):
            for i in range(r):
                j = length - r + i
                if j < 0:
                    continue
                for h in range(s.heads):
                    x = i if kept is None else int(kept[b, h, i])
                    at = int(to_table[b, j // to_page]), h, j % to_page
                    if not 0 <= at[0] < t.shape[0]:
                        continue
                    t[at] = old[int(s.table[b, x // s.page]), h, x % s.page] if 0 <= x < s.lens[b] else 0
    return want


GATHERS = [  # fmt, dim, heads, page from, to, source lengths, [(rows, kv)]
    ("bf16", 128, 4, 64, 64, [300, 40], [(200, 200), (9, 20)]),
    ("bf16", 128, 2, 16, 128, [300, 0, 7], [(40, 200), (5, 5), (0, 9)]),
    ("bf16", 64, 3, 128, 16, [500], [(129, 129)]),
    ("bf16", 8, 2, 16, 32, [50], [(33, 33)]),
    ("bf16", 80, 1, 32, 32, [100, 100], [(64, 64), (1, 1)]),
    ("u8", 128, 2, 32, 16, [90], [(60, 70)]),
    ("u8", 64, 5, 16, 16, [90, 3], [(65, 65), (2, 2)]),
    ("u4", 128, 3, 32, 32, [400], [(300, 300)]),
    ("u4", 64, 1, 16, 64, [70], [(257, 257)]),
]


@pytest.mark.parametrize("listed", [True, False])
@pytest.mark.parametrize("case", range(len(GATHERS)))
def test_gathers(case, listed):
    fmt, dim, heads, page, to_page, lens, seqs = GATHERS[case]
    gen = torch.Generator().manual_seed(800 + case)
    s = Setup(gen, fmt, heads, dim, page, lens, [0] * len(lens), garbage=False)
    rows, to_lens = [r for r, _ in seqs], [n for _, n in seqs]
    t = Setup(gen, fmt, heads, dim, to_page, to_lens, rows, garbage=False)
    kept = None
    if listed:
        kept = torch.zeros((len(lens), heads, max(rows) + 3), dtype=torch.int32)
        for b, n in enumerate(lens):
            kept[b] = torch.randint(0, max(1, n), kept.shape[1:], generator=gen)  # the same row several times, in any order
        kept[0, 0, :3] = torch.tensor([-1, lens[0], 1 << 30])
    want = gathered(s, t.table, rows, to_lens, to_page, kept, t.cache)
    t.cache.gather(s.cache, s.batch, t.batch, None if kept is None else kept.cuda())
    assert all(same_bits(a, b) for a, b in zip(parts(t.cache), want))


def test_gather_to_unusual_places():
    """Into other pages of the same pool, before position 0, pages outside the pool, one list for all heads, a source without a table."""
    gen = torch.Generator().manual_seed(83)
    cache = PagedCache(6, 16, 2, 64)
    cache.k.copy_(make_rows(gen, 6, 2, 16, 64).cuda()), cache.v.copy_(make_rows(gen, 6, 2, 16, 64).cuda())
    k, v = cache.k.cpu().clone(), cache.v.cpu().clone()
    source = PagedBatch(ints(4, 2)[None], ints(0, 0), ints(30), total_rows=0, max_rows=0, max_kv=32)
    kept = torch.randint(0, 30, (20,), generator=gen, dtype=torch.int32)
    to = PagedBatch(ints(5, 77)[None], ints(0, 20), ints(18), total_rows=20, max_rows=20, max_kv=32)
    cache.gather(cache, source, to, kept.cuda()[None, None].expand(1, 2, 20))
    for i in range(2, 18):
        x = int(kept[i])
        k[5, :, i - 2], v[5, :, i - 2] = k[[4, 2][x // 16], :, x % 16], v[[4, 2][x // 16], :, x % 16]
    assert same_bits(cache.k, k) and same_bits(cache.v, v)
    pp = PingPongCache(6, 40, 64, "bf16", patch_ids=False)
    pp.k[0], pp.v[0] = make_rows(gen, 6, 40, 64).cuda(), make_rows(gen, 6, 40, 64).cuda()
    layer = PagedCache.of_layer(pp, 2, 3, 2)
    cache.gather(layer, PagedBatch(None, ints(0, 0), ints(40), total_rows=0, max_rows=0, max_kv=40),
                 PagedBatch(ints(0, 1)[None], ints(0, 25), ints(25), total_rows=25, max_rows=25, max_kv=32))
    assert same_bits(cache.k[0], pp.k[0, 4:6, :16]) and same_bits(cache.v[1, :, :9], pp.v[0, 4:6, 16:25])


# ------------------------------------------------------------------- together
class Session:
    """One layer of a decoder over a pool: rows in by write_rotated, pages chosen, attention over them; what it must give, from the rows
    that the pool itself holds."""

    def __init__(self, fmt, heads, share, dim, page, n_pages, seed):
        self.gen = torch.Generator().manual_seed(seed)
        self.heads, self.share, self.dim, self.page = heads, share, dim, page
        self.cache, self.books = PagedCache(n_pages, page, heads, dim, fmt), Sequences(n_pages, page)
        self.bounds = PageBounds(self.cache)
        self.rotary = Rotary.of_base(10000.0, 4000, dim)
        self.w = make_rows(self.gen, dim, spread=False).abs().cuda()
        self.seen = {}

    def step(self, seqs, n, chosen):
        """n new rows of each of the sequences."""
        copies = sum((self.books.extend(s, n) for s in seqs), [])
        if copies:
            self.cache.copy_pages(ints(*[a for a, _ in copies]), ints(*[b for _, b in copies]))
        batch = self.books.batch(seqs, [n] * len(seqs))
        at = []
        for s in seqs:
            self.seen[s] = self.seen.get(s, 0) + n
            at += range(self.seen[s] - n, self.seen[s])
        total = n * len(seqs)
        q, k, v = (make_rows(self.gen, total, h, self.dim).cuda() for h in (self.heads * self.share, self.heads, self.heads))
        q = self.cache.write_rotated(q, k, v, batch, self.rotary, ints(*at), q_weight=self.w, k_weight=self.w)
        self.bounds.update(self.cache, batch)
        lists = self.bounds.choose(q, batch, chosen, first=1, recent=2)
        lse = torch.empty(total, self.heads * self.share, device="cuda")
        return batch, q, lists, self.cache.attend_chosen(q, batch, lists, lse=lse), lse

    def held(self, seq):
        """k, v [rows, heads, dim] as read gives them; codes' values, once rounded more."""
        n = self.books.rows(seq)
        k, v = self.cache.read(self.books.batch([seq], [n]))
        return k.double().cpu(), v.double().cpu()

    def check(self, seqs, n, chosen, batch, q, lists, out, lse):
        codes, steps, q, out, lists = self.bounds.codes.cpu().long(), self.bounds.steps.cpu().double(), q.cpu(), out.double().cpu(), lists.cpu()
        for b, s in enumerate(seqs):
            at = slice(b * n, (b + 1) * n)
            k, v = self.held(s)
            pages, length = torch.tensor(self.books.pages(s)), self.books.rows(s)
            for i in range(n):
                held = (length - n + i) // self.page + 1
                for h in range(self.heads):
                    lo, hi = codes[pages[:held], h, :, :self.dim].unbind(1)
                    score = cref.scores(q[b * n + i, h * self.share:(h + 1) * self.share], lo, hi, steps[pages[:held], h])
                    assert lists[b * n + i, h].tolist() == cref.choose(score, chosen, 1, 2)
            for i, p in enumerate(pages.tolist()):  # every page's bounds hold its keys
                rows = k[i * self.page:(i + 1) * self.page]
                for h in range(self.heads):
                    lo, hi, step = cref.bounds(rows[:, h])
                    assert float(steps[p, h]) == step and torch.equal(codes[p, h, :, :self.dim], torch.stack([lo, hi])), (s, i)
            o, l, weight, size = cref.attend(q[at].double(), k, v, lists[at], self.page, self.dim ** -0.5)
            tol = bounds(self.cache.fmt, weight, size, o, length, float(v.abs().max()))
            if self.cache.fmt != "bf16":  # `read` rounds the codes' values to bf16: scores by 2^-8 of their products, values by 2^-8
                # and m's distance from the rounded v is p (v - m) up to 2^-8 p |v|, which 2^-11 makes nothing of
                tol = tol + (2.0 ** -8 + torch.expm1(2.0 * 2.0 ** -8 * size[..., None])) * weight * 1.01
                tol = tol + 2.0 ** -11 * cref.attend(q[at].double(), k, v, lists[at], self.page, self.dim ** -0.5,
                                                     above_minimum(self.cache, v, pages))[2].abs()
            assert ((out[at] - o).abs() <= tol).all(), s


@pytest.mark.parametrize("fmt", ["bf16", "u8", "u4"])
def test_a_session(fmt):
    """Two streams are filled, answer, one is forked and both answer, one is cut to kept rows and goes on."""
    s = Session(fmt, 2, 4, 128, 16, 120, 91)
    a, b = s.books.add(), s.books.add()
    s.check([a, b], 200, 6, *s.step([a, b], 200, 6))
    for _ in range(3):
        s.check([b, a], 1, 6, *s.step([b, a], 1, 6))
    c = s.books.fork(a)
    s.seen[c] = s.seen[a]
    s.check([c, a, b], 1, 6, *s.step([c, a, b], 1, 6))  # c writes into a copy of the last page
    k_a, k_c = s.held(a)[0], s.held(c)[0]
    assert torch.equal(k_a[:203], k_c[:203]) and not torch.equal(k_a[203], k_c[203])
    # a is cut to 90 of its 204 rows, each head's own
    kept = torch.stack([torch.randperm(204, generator=s.gen)[:90].sort().values for _ in range(2)]).to(torch.int32)
    old_k, old_v = s.held(a)
    source = s.books.batch([a], [0])
    old = s.books.replace(a, 90)
    whole = s.books.batch([a], [90])
    s.cache.gather(s.cache, source, whole, kept[None].cuda())
    s.bounds.update(s.cache, whole)
    s.books.release(old)
    new_k, new_v = s.held(a)
    for h in range(2):
        assert torch.equal(new_k[:, h], old_k[kept[h].long(), h]) and torch.equal(new_v[:, h], old_v[kept[h].long(), h])
    s.check([a, c], 3, 4, *s.step([a, c], 3, 4))
    s.books.remove(c)
    s.check([a, b], 20, 4, *s.step([a, b], 20, 4))


def test_a_step_in_a_graph():
    """The four calls captured once and replayed for tokens whose rows, positions and lengths change on the device; another stream,
    a workspace of the graph's own, eager calls in between."""
    s = Session("bf16", 2, 4, 128, 16, 64, 97)
    seq = s.books.add()
    s.step([seq], 150, 6)
    s.books.extend(seq, 60)  # room; the lengths below say what is held
    pages = s.books.pages(seq)
    kv_len, at = ints(150), ints(150)
    batch = PagedBatch(s.books.table([seq]).cuda(), ints(0, 1), kv_len, total_rows=1, max_rows=1, max_kv=16 * len(pages))
    q, k, v = (make_rows(s.gen, 1, h, 128).cuda() for h in (8, 2, 2))
    turned, lists, out, lse = torch.empty_like(q), torch.empty((1, 2, 6), dtype=torch.int32, device="cuda"), torch.empty_like(q), torch.empty(1, 8, device="cuda")

    def step():
        kv_len.add_(1)
        s.cache.write_rotated(q, k, v, batch, s.rotary, at, q_weight=s.w, k_weight=s.w, q_out=turned)
        s.bounds.update(s.cache, batch)
        s.bounds.choose(turned, batch, 6, first=1, recent=2, out=lists)
        s.cache.attend_chosen(turned, batch, lists, out=out, lse=lse)
        at.add_(1)

    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        step()
        kv_len.fill_(150), at.fill_(150)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    seen = []
    for i in range(40):
        q.copy_(make_rows(s.gen, 1, 8, 128)), k.copy_(make_rows(s.gen, 1, 2, 128)), v.copy_(make_rows(s.gen, 1, 2, 128))
        graph.replay()
        seen.append((turned.cpu(), lists.cpu(), out.double().cpu()))
        if i == 20:  # an eager call of the same sizes between two replays
            again = s.cache.attend_chosen(turned, batch, lists)
            assert same_bits(again, out)
    torch.cuda.synchronize()
    assert int(kv_len) == 190
    read = PagedBatch(batch.table, ints(0, 190), ints(190), total_rows=190, max_rows=190, max_kv=16 * len(pages))
    k_all, v_all = (t.double().cpu() for t in s.cache.read(read))
    for i in (0, 1, 9, 10, 25, 39):
        n = 151 + i
        o, l, weight, size = cref.attend(seen[i][0].double(), k_all[:n], v_all[:n], seen[i][1], 16, 128 ** -0.5)
        assert seen[i][1][0, 0, 0] == 0 and (seen[i][1][0, :, -1] == (n - 1) // 16).all()
        assert ((seen[i][2] - o).abs() <= bounds("bf16", weight, size, o, n, 0.0)).all(), i


def test_bits_do_not_change_between_runs_streams_and_workspaces():
    gen = torch.Generator().manual_seed(101)
    for fmt, rows, kv, n in (("u8", 1, 3000, 150), ("bf16", 1, 3000, 20), ("bf16", 40, 1500, 12)):
        s = Setup(gen, fmt, 2, 128, 16, [kv, 1700], [rows, rows])
        chosen = random_lists(gen, s, n).cuda()
        q = make_rows(gen, s.total, 14, 128).cuda()
        want = s.cache.attend_chosen(q, s.batch, chosen)
        torch.cuda.synchronize()
        side, ws = torch.cuda.Stream(), torch.empty(64 << 20, dtype=torch.uint8, device="cuda").fill_(255)
        torch.cuda.synchronize()
        for _ in range(3):
            out = s.cache.attend_chosen(q, s.batch, chosen, workspace=ws, stream=side)
            side.synchronize()
            assert same_bits(out, want)


def test_calls_on_a_named_stream():
    """Each call on a stream that is not the current one, its results made there."""
    s = Session("bf16", 2, 4, 64, 16, 40, 103)
    seq = s.books.add(100)
    batch = s.books.batch([seq], [100])
    q, k, v = (make_rows(s.gen, 100, h, 64).cuda() for h in (8, 2, 2))
    at, ws = torch.arange(100, dtype=torch.int32, device="cuda"), torch.empty(32 << 20, dtype=torch.uint8, device="cuda")
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    turned = s.cache.write_rotated(q, k, v, batch, s.rotary, at, stream=side)
    s.bounds.update(s.cache, batch, stream=side)
    lists = s.bounds.choose(turned, batch, 4, stream=side)
    out = s.cache.attend_chosen(turned, batch, lists, workspace=ws, stream=side)
    side.synchronize()
    here = PagedCache(40, 16, 2, 64)
    made = PageBounds(here)
    want = here.write_rotated(q, k, v, batch, s.rotary, at)
    made.update(here, batch)
    again = made.choose(want, batch, 4)
    assert same_bits(turned, want) and same_bits(lists, again) and same_bits(out, here.attend_chosen(want, batch, again))


def test_refusals_on_the_gpu():
    gen = torch.Generator().manual_seed(107)
    s = Setup(gen, "bf16", 1, 128, 16, [20000], [1])
    q, chosen = make_rows(gen, 1, 8, 128).cuda(), torch.arange(1200, dtype=torch.int32, device="cuda")[None, None]
    with pytest.raises(ipv.IpvError, match="workspace"):
        s.cache.attend_chosen(q, s.batch, chosen, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    none = PagedBatch(None, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                      total_rows=0, max_rows=0, max_kv=0)
    assert s.cache.attend_chosen(q[:0], none, chosen[:0]).shape == (0, 8, 128)
    made = PageBounds(s.cache)
    assert made.choose(q[:0], none, 4).shape == (0, 1, 4)
    made.update(s.cache, none)
    s.cache.write_rotated(q[:0], q[:0, :1], q[:0, :1], none, Rotary.of_base(1e4, 10, 128), torch.zeros(0, dtype=torch.int32, device="cuda"))
    s.cache.gather(s.cache, none, none)
    with pytest.raises(ipv.IpvError, match="shape"):
        PageBounds(PagedCache(3, 16, 1, 128)).update(s.cache, s.batch)
