"""The paged cache on the GPU against plain float64 definitions: what is written
is right to the bit, what is read back is rounded once, attention is within
bounds that follow from the roundings it makes.

Bounds. bf16 has unit roundoff 2^-8, fp16 2^-11, fp32 2^-24. An output is
rounded once to bf16: 2^-8 |o|. A softmax weight is rounded to bf16 (bf16
pages) or fp16 (codes, and V's values as well): 2^-8 or 2 * 2^-11 times
sum p |v|; a weight that is subnormal in fp16 is off by at most 2^-25, so n of
them by n 2^-25 max |v|. A score that is off by d moves weights by factors in
e^(+-2d): 2 d sum p |v| to first order. Scores are sums of `dim` fp32 terms,
which a matrix instruction may truncate: 2^-16 sum |q k| covers 128 of them at
2^-23 each; with codes, keys may be rounded to fp16 first, 2^-11 sum |q k|.
exp2's approximation (2^-22) is far below all of these."""
import math

import numpy as np
import pytest

torch = pytest.importorskip("torch")

import paged_ref as ref  # noqa: E402
from paper_2506_15745_gb300 import ipv  # noqa: E402
from paper_2506_15745_gb300.cache import PingPongCache  # noqa: E402
from paper_2506_15745_gb300.paged import PagedBatch, PagedCache  # noqa: E402

pytestmark = pytest.mark.gpu


def make_rows(gen, *shape, spread=True):
    """bf16 rows with a few wide, shifted channels, as decoders' keys have."""
    x = torch.randn(shape, generator=gen)
    if spread:
        c = torch.randint(0, shape[-1], (2,), generator=gen)
        x[..., c] = x[..., c] * 4 + 3
    return x.bfloat16()


class Setup:
    """Sequences in a pool, and what they hold, as float64."""

    def __init__(self, gen, fmt, heads, dim, page, lens, rows, garbage=True, extra_pages=2, max_rows=None, max_kv=None):
        self.fmt, self.heads, self.dim, self.page, self.lens, self.rows = fmt, heads, dim, page, lens, rows
        wide = max(1, max(-(-n // page) for n in lens))
        n_pages = sum(-(-n // page) for n in lens) + extra_pages
        order = torch.randperm(n_pages, generator=gen)
        table = torch.full((len(lens), wide), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(lens):
            c = -(-n // page)
            table[b, :c] = order[at:at + c].to(torch.int32)
            at += c
        self.table = table
        full = (n_pages, heads, page, dim)
        self.k, self.v = [], []
        store = {}
        for name in ("k", "v"):
            x = make_rows(gen, *full)
            if fmt == "bf16":
                held, t = x.double(), x.clone()
                if garbage:
                    used = torch.zeros(n_pages, page, dtype=torch.bool)
                    for b, n in enumerate(lens):
                        for j in range(n):
                            used[table[b, j // page], j % page] = True
                    bad = ~used[:, None, :, None].expand(full)
                    t[bad] = torch.tensor([float("nan"), float("inf"), -float("inf"), 3e38]).bfloat16()[
                        torch.randint(0, 4, (int(bad.sum()),), generator=gen)]
                store[name], store[name + "_par"] = t.cuda(), None
            else:
                u, s, m = ref.quantise(x, fmt)
                held = ref.values(u, s, m)
                par = torch.stack([s, m], -1)
                if garbage:
                    for g in set(range(n_pages)) - set(table[table >= 0].tolist()):
                        par[g] = float("nan")
                    for b, n in enumerate(lens):
                        if n % page:
                            par[table[b, n // page], :, n % page:] = float("nan")
                store[name], store[name + "_par"] = ref.pack(u, fmt).cuda(), par.cuda()
            seqs = []
            for b, n in enumerate(lens):
                j = torch.arange(n)
                seqs.append(held[table[b, j // page].long(), :, j % page])
            setattr(self, name, seqs)
        self.cache = PagedCache.from_tensors(fmt, store["k"], store["v"], store["k_par"], store["v_par"])
        self.start = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
        self.total = int(self.start[-1])
        self.batch = PagedBatch(table.cuda(), torch.from_numpy(self.start).cuda(),
                                torch.tensor(lens, dtype=torch.int32).cuda(), total_rows=self.total,
                                max_rows=max(rows) if max_rows is None else max_rows,
                                max_kv=max(lens) if max_kv is None else max_kv)


def bounds(fmt, weight, size, out, length, vmax):
    u_p, u_k = (2.0 ** -8, 2.0 ** -16) if fmt == "bf16" else (2.0 ** -10, 2.0 ** -11 + 2.0 ** -16)
    d = u_k * size[..., None]
    return 2.0 ** -8 * out.abs() + (u_p + torch.expm1(2 * d)) * weight * 1.02 + length * 2.0 ** -25 * vmax + 1e-30


def check_attend(s, q, got, lse, scale, causal=True, window=0, sinks=0):
    got, lse = got.double().cpu(), lse.double().cpu()
    for b, (n, length) in enumerate(zip(s.rows, s.lens)):
        at = slice(int(s.start[b]), int(s.start[b + 1]))
        o, l, weight, size = ref.attend(q[at].double(), s.k[b], s.v[b], scale, causal, window, sinks)
        vmax = float(s.v[b].abs().max()) if length else 0.0
        tol = bounds(s.fmt, weight, size, o, length, vmax)
        off = (got[at] - o).abs()
        assert torch.isfinite(got[at]).all(), (b, n, length)
        assert (off <= tol).all(), (b, n, length, float((off / tol.clamp(min=1e-30)).max()))
        empty = torch.isinf(l)
        assert torch.equal(lse[at][empty], l[empty])
        ltol = (size * (2.0 ** -16 if s.fmt == "bf16" else 2.0 ** -11 + 2.0 ** -16) + 2.0 ** -20 * (1 + l.abs()))[~empty]
        assert ((lse[at] - l)[~empty].abs() <= ltol).all(), (b, n, length)


def run_attend(s, share, seed, **kw):
    gen = torch.Generator().manual_seed(seed)
    q = (torch.randn((s.total, s.heads * share, s.dim), generator=gen) * 1.5).bfloat16()
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    s.cache.attend(q.cuda(), s.batch, out=out, lse=lse, **kw)
    torch.cuda.synchronize()
    return q, out, lse


# ------------------------------------------------------------ write and read back
WRITE_SHAPES = [  # fmt, dim, heads, page, (rows, kv)
    ("bf16", 128, 4, 16, [(1, 1), (0, 5), (17, 40), (33, 33)]),
    ("bf16", 80, 3, 32, [(5, 70), (64, 64)]),
    ("bf16", 8, 1, 64, [(3, 130)]),
    ("u8", 128, 4, 16, [(1, 1), (0, 0), (17, 40), (33, 33), (100, 257)]),
    ("u8", 64, 7, 64, [(1, 65), (200, 300)]),
    ("u4", 128, 4, 16, [(1, 1), (0, 0), (17, 40), (33, 33), (100, 257)]),
    ("u4", 64, 5, 128, [(1, 129), (300, 300)]),
    ("u4", 128, 28, 256, [(1, 1000)] * 9),
]


@pytest.mark.parametrize("fmt,dim,heads,page,seqs", WRITE_SHAPES)
def test_write_to_the_bit_and_read_back(fmt, dim, heads, page, seqs):
    gen = torch.Generator().manual_seed(len(seqs) * 1000 + dim)
    rows, lens = [r for r, _ in seqs], [n for _, n in seqs]
    s = Setup(gen, fmt, heads, dim, page, lens, rows, garbage=False)
    k_new, v_new = make_rows(gen, s.total, heads, dim), make_rows(gen, s.total, heads, dim, spread=False) * 0.3
    want = {}
    for name, x in (("k", k_new), ("v", v_new)):
        pool, par = getattr(s.cache, name).cpu().clone(), getattr(s.cache, name + "_par")
        par = None if par is None else par.cpu().clone()
        for b, (n, length) in enumerate(seqs):
            for i in range(n):
                j = length - n + i
                at = (int(s.table[b, j // page]), slice(None), j % page)
                if fmt == "bf16":
                    pool[at] = x[int(s.start[b]) + i]
                else:
                    u, st, m = ref.quantise(x[int(s.start[b]) + i], fmt)
                    pool[at], par[at] = ref.pack(u, fmt), torch.stack([st, m], -1)
        want[name] = (pool, par)
    s.cache.write(k_new.cuda(), v_new.cuda(), s.batch)
    k_back, v_back = s.cache.read(s.batch)
    for name, back, x in (("k", k_back, k_new), ("v", v_back, v_new)):
        pool, par = want[name]
        assert torch.equal(getattr(s.cache, name).cpu(), pool), name  # the whole pool: nothing else was touched
        if fmt == "bf16":
            assert torch.equal(back.cpu(), x)
        else:
            assert torch.equal(getattr(s.cache, name + "_par").cpu().view(torch.int16), par.view(torch.int16)), name
            u, st, m = ref.quantise(x, fmt)
            assert torch.equal(back.cpu(), ref.values(u, st, m).float().bfloat16()), name


@pytest.mark.parametrize("fmt", ["u8", "u4"])
def test_special_groups(fmt):
    """Constant, tiny, huge, signed-zero and marked groups; ties between levels."""
    gen = torch.Generator().manual_seed(3)
    x = make_rows(gen, 24, 1, 128, spread=False).float()
    x[0] = 0.0
    x[1] = -0.0
    x[2] = 2.5
    x[3] = -3e-9                                     # below fp16's smallest step
    x[4] *= 1e-7
    x[5] *= 8000.0
    x[5].clamp_(-32768, 32768)
    x[6, :, 3] = float("nan")
    x[7, :, 70] = float("inf")
    x[8, :, 5] = -float("inf")
    x[9, :, 100] = 32769.0 * 1.01
    x[10, :, 0] = 32768.0
    x[11] = torch.arange(128) % 64 * 0.5             # many values half way between levels
    x[12] = (torch.arange(128) % 31 - 15).float()
    x[13, :, :64] = torch.linspace(-1, 1, 64)
    x = x.bfloat16()
    cache = PagedCache(2, 16, 1, 128, fmt)
    batch = PagedBatch(torch.tensor([[1, 0]], dtype=torch.int32).cuda(), torch.tensor([0, 24], dtype=torch.int32).cuda(),
                       torch.tensor([24], dtype=torch.int32).cuda(), total_rows=24, max_rows=24, max_kv=32)
    cache.write(x.cuda(), x.cuda(), batch)
    back = cache.read(batch)[0].cpu()
    u, st, m = ref.quantise(x, fmt)
    want = ref.values(u, st, m)
    j = torch.arange(24)
    page = torch.tensor([1, 0])[j // 16]
    assert torch.equal(cache.k.cpu()[page, :, j % 16], ref.pack(u, fmt))
    par = cache.k_par.cpu()[page, :, j % 16]
    assert torch.equal(torch.isnan(par), torch.isnan(torch.stack([st, m], -1)))
    assert torch.equal(par.nan_to_num(0.0), torch.stack([st, m], -1).nan_to_num(0.0))
    assert torch.equal(torch.isnan(back), torch.isnan(want))
    assert torch.equal(back.nan_to_num(0.0), want.float().bfloat16().nan_to_num(0.0))
    for r, g in ((6, 0), (7, 1), (8, 0), (9, 1)):    # the marked group and only it
        nan = torch.isnan(back[r, 0]).reshape(2, 64)
        assert nan[g].all() and not nan[1 - g].any()


def test_write_drops_what_does_not_fit():
    """Rows before position 0, page numbers outside the pool, and new rows outside the packed ones are dropped;
    read gives zeros for the first two."""
    gen = torch.Generator().manual_seed(5)
    cache = PagedCache(3, 16, 2, 64, "bf16")
    cache.k.fill_(9.0), cache.v.fill_(9.0)
    table = torch.tensor([[0, 99], [-1, 1], [2, 2], [2, 2]], dtype=torch.int32).cuda()
    start = torch.tensor([0, 20, 40, 45, 90], dtype=torch.int32).cuda()   # the last one's rows end past the packed 60
    lens = torch.tensor([20, 20, 3, 16], dtype=torch.int32).cuda()        # the third has 5 new rows and 3 in all
    batch = PagedBatch(table, start, lens, total_rows=60, max_rows=20, max_kv=32)
    x = make_rows(gen, 60, 2, 64, spread=False)
    cache.write(x.cuda(), -x.cuda(), batch)
    want = torch.full((3, 2, 16, 64), 9.0).bfloat16()
    want[0] = x[:16].transpose(0, 1)
    want[1, :, :4] = x[36:40].transpose(0, 1)
    want[2, :, :3] = x[42:45].transpose(0, 1)
    assert torch.equal(cache.k.cpu(), want)
    k_out = torch.full((60, 2, 64), 5.0, dtype=torch.bfloat16, device="cuda")
    cache.read(batch, k_out, k_out.clone())
    back = torch.full((60, 2, 64), 5.0).bfloat16()
    back[:20] = torch.cat([x[:16], torch.zeros(4, 2, 64).bfloat16()])
    back[20:40] = torch.cat([torch.zeros(16, 2, 64).bfloat16(), x[36:40]])
    back[40:45] = torch.cat([torch.zeros(2, 2, 64).bfloat16(), x[42:45]])
    assert torch.equal(k_out.cpu(), back)


# ------------------------------------------------------------------- attention
def test_single_tokens_of_every_length():
    """Lengths around the step, page and split sizes, zero and one among them, in one batch."""
    lens = [0, 1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500, 1023, 1537]
    for fmt in ("bf16", "u8", "u4"):
        gen = torch.Generator().manual_seed(11)
        s = Setup(gen, fmt, 2, 128, 16, lens, [1] * len(lens))
        q, out, lse = run_attend(s, 7, 12)
        check_attend(s, q, out, lse, 128 ** -0.5)


ATTEND = [  # fmt, dim, heads, share, page, [(rows, kv)], kwargs
    ("bf16", 64, 4, 1, 16, [(1, 300), (1, 77)], {}),
    ("bf16", 128, 1, 8, 64, [(1, 3000)], {}),
    ("bf16", 128, 2, 5, 256, [(1, 700)] * 3, {"window": 64, "sinks": 4}),
    ("bf16", 80, 2, 3, 32, [(1, 100), (3, 200), (0, 50)], {}),
    ("bf16", 96, 1, 4, 64, [(5, 5), (2, 130)], {"window": 7, "sinks": 1}),
    ("bf16", 8, 3, 2, 16, [(9, 40)], {}),
    ("bf16", 120, 1, 16, 128, [(1, 1000)], {"causal": False}),
    ("u8", 64, 4, 2, 16, [(1, 300), (1, 77), (2, 2)], {}),
    ("u8", 128, 2, 7, 64, [(1, 2500), (1, 10)], {}),
    ("u8", 128, 1, 8, 32, [(2, 900)], {"window": 100, "sinks": 40}),
    ("u4", 64, 4, 4, 16, [(1, 300), (3, 77)], {}),
    ("u4", 128, 2, 8, 64, [(1, 2500), (1, 10)], {}),
    ("u4", 128, 1, 5, 32, [(1, 900), (4, 700)], {"window": 33, "sinks": 3}),
    ("bf16", 128, 2, 7, 64, [(40, 40), (61, 500), (1, 9), (130, 131)], {}),
    ("bf16", 64, 2, 4, 16, [(300, 300), (17, 600)], {"window": 50, "sinks": 5}),
    ("bf16", 64, 1, 1, 32, [(257, 1000)], {"causal": False}),
    ("bf16", 80, 2, 3, 16, [(100, 333), (9, 20)], {}),
    ("bf16", 128, 1, 8, 128, [(33, 2000)], {"window": 1, "sinks": 0}),
    ("u8", 128, 2, 7, 64, [(61, 700), (20, 20), (1, 300)], {}),
    ("u8", 64, 1, 3, 16, [(200, 450)], {"window": 30, "sinks": 17}),
    ("u4", 128, 2, 4, 32, [(61, 700), (140, 140)], {}),
    ("u4", 64, 2, 8, 256, [(90, 600)], {"causal": False}),
]


@pytest.mark.parametrize("fmt,dim,heads,share,page,seqs,kw", ATTEND)
def test_attend(fmt, dim, heads, share, page, seqs, kw):
    gen = torch.Generator().manual_seed(dim * 31 + share)
    s = Setup(gen, fmt, heads, dim, page, [n for _, n in seqs], [r for r, _ in seqs])
    q, out, lse = run_attend(s, share, 21, **kw)
    check_attend(s, q, out, lse, dim ** -0.5, **kw)


@pytest.mark.parametrize("fmt", ["bf16", "u8", "u4"])
@pytest.mark.parametrize("rows", [1, 30])
def test_rows_that_see_nothing(fmt, rows):
    """More new rows than cached ones: queries before position 0 get 0 and -inf, and NaN elsewhere in the pool
    does not reach them; an empty sequence, and one without new rows."""
    gen = torch.Generator().manual_seed(31)
    lens, n = [0, max(0, rows - 12), 40], [rows, rows, 0]
    s = Setup(gen, fmt, 2, 128, 16, lens, n)
    q, out, lse = run_attend(s, 4, 32)
    out, lse = out.cpu(), lse.cpu()
    hidden = rows - lens[1]
    assert (out[:rows + hidden] == 0).all() and (lse[:rows + hidden] == -math.inf).all()
    if lens[1]:
        at = slice(rows + hidden, 2 * rows)
        o, l, weight, size = ref.attend(q[at].double(), s.k[1], s.v[1], 128 ** -0.5)
        tol = bounds(fmt, weight, size, o, lens[1], float(s.v[1].abs().max()))
        assert ((out[at].double() - o).abs() <= tol).all()


def test_strided_pools_queries_and_outputs():
    """A pool laid out [page][row][head], queries and outputs that are slices of wider tensors."""
    gen = torch.Generator().manual_seed(41)
    lens, rows = [130, 47], [3, 20]
    s = Setup(gen, "bf16", 4, 64, 16, lens, rows)
    k, v = (t.permute(0, 2, 1, 3).contiguous().permute(0, 2, 1, 3) for t in (s.cache.k, s.cache.v))
    cache = PagedCache.from_tensors("bf16", k, v)
    wide = (torch.randn((s.total, 3, 8, 64), generator=gen) * 1.5).bfloat16()
    q = wide[:, 1]
    out_wide = torch.full((8, s.total, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.zeros((s.total, 8), device="cuda")
    cache.attend(wide.cuda()[:, 1], s.batch, out=out_wide.transpose(0, 1), lse=lse)
    check_attend(s, q, out_wide.transpose(0, 1), lse, 64 ** -0.5)
    kv = make_rows(gen, 2, s.total, 4, 64)
    wide = torch.zeros((s.total, 12, 64), dtype=torch.bfloat16)
    wide[:, 4:8], wide[:, 8:] = kv[0], kv[1]
    wide = wide.cuda()
    cache.write(wide[:, 4:8], wide[:, 8:], s.batch)
    back_k, back_v = cache.read(s.batch)
    assert torch.equal(back_k.cpu(), kv[0]) and torch.equal(back_v.cpu(), kv[1])


def test_a_live_half_of_the_ping_pong_cache():
    """One layer of a ping-pong cache attended to as it stands, no table, a capacity that is no power of two."""
    gen = torch.Generator().manual_seed(51)
    layers, heads, cap, dim, n = 3, 2, 300, 128, 287
    cache = PingPongCache(layers * heads, cap, dim, "bf16", patch_ids=False)
    cache.k[0] = make_rows(gen, layers * heads, cap, dim).cuda()
    cache.v[0] = make_rows(gen, layers * heads, cap, dim).cuda()
    cache.n_tokens = n
    pages = PagedCache.of_layer(cache, 1, layers, heads)
    for rows in (1, 25):
        batch = PagedBatch(None, torch.tensor([0, rows], dtype=torch.int32).cuda(),
                           torch.tensor([n], dtype=torch.int32).cuda(), total_rows=rows, max_rows=rows, max_kv=cap)
        q = (torch.randn((rows, 14, dim), generator=gen) * 1.5).bfloat16()
        lse = torch.zeros((rows, 14), device="cuda")
        out = pages.attend(q.cuda(), batch, lse=lse)
        o, l, weight, size = ref.attend(q.double(), cache.k[0, 2:4, :n].transpose(0, 1).double().cpu(),
                                        cache.v[0, 2:4, :n].transpose(0, 1).double().cpu(), dim ** -0.5)
        tol = bounds("bf16", weight, size, o, n, 1.0)
        assert ((out.double().cpu() - o).abs() <= tol).all()
        assert ((lse.double().cpu() - l).abs() <= size * 2.0 ** -16 + 2.0 ** -20 * (1 + l.abs())).all()


def test_marked_groups_reach_the_output():
    """A visible NaN is not hidden: a marked K or V group makes the queries that see it NaN."""
    gen = torch.Generator().manual_seed(61)
    s = Setup(gen, "u4", 1, 128, 16, [50], [1])
    s.cache.v_par[int(s.table[0, 1]), 0, 3, 1] = float("nan")
    _, out, _ = run_attend(s, 4, 62)
    assert torch.isnan(out[..., 64:]).all() and torch.isfinite(out[..., :64]).all()
    s.cache.k_par[int(s.table[0, 1]), 0, 3, 0] = float("nan")
    _, out, lse = run_attend(s, 4, 62)
    assert torch.isnan(out).all() and torch.isnan(lse).all()


def test_large_and_small_queries():
    """Query rows far outside fp16's range, in both directions, over codes; scores that overflow nothing."""
    gen = torch.Generator().manual_seed(71)
    for fmt in ("u8", "u4", "bf16"):
        s = Setup(gen, fmt, 2, 128, 16, [200, 90], [1, 20])
        q = (torch.randn((21, 8, 128), generator=gen)).bfloat16()
        q[:, 0] *= 2.0 ** 60
        q[:, 1] *= 2.0 ** -60
        q[:, 2] = 0
        q[:, 3] *= 1e5
        for scale in (2.0 ** -66, 2.0 ** -20):
            sub = q if scale < 2.0 ** -30 else q[:, [1, 2, 3, 4, 5, 6, 7, 1]]
            lse = torch.zeros((21, 8), device="cuda")
            out = s.cache.attend(sub.cuda(), s.batch, lse=lse, scale=scale)
            check_attend(s, sub, out, lse, scale)


@pytest.mark.parametrize("fmt", ["bf16", "u4"])
@pytest.mark.parametrize("scale", [0.0, -0.1])
def test_scales_that_are_not_positive(fmt, scale):
    gen = torch.Generator().manual_seed(75)
    for n in (1, 20):
        s = Setup(gen, fmt, 2, 128, 16, [200, 90], [1, n])
        q, out, lse = run_attend(s, 4, 76, scale=scale, window=50, sinks=3)
        check_attend(s, q, out, lse, scale, window=50, sinks=3)


def test_bits_do_not_change_between_runs_and_streams():
    gen = torch.Generator().manual_seed(81)
    s = Setup(gen, "u8", 2, 128, 64, [3000, 1700], [1, 1])
    q = make_rows(gen, 2, 14, 128).cuda()
    want = s.cache.attend(q, s.batch)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    ws = torch.empty(64 << 20, dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    for _ in range(3):
        out = torch.zeros_like(q)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            s.cache.attend(q, s.batch, out=out, workspace=ws)
        side.synchronize()
        assert torch.equal(out, want)


def test_a_decode_step_in_a_graph():
    """Write the token's rows and attend, captured once, replayed with lengths that grow on the device."""
    gen = torch.Generator().manual_seed(91)
    page, dim, heads = 16, 128, 2
    cache = PagedCache(20, page, heads, dim, "u8")
    table = torch.randperm(20, generator=gen).to(torch.int32)[None].cuda()
    kv_len = torch.tensor([0], dtype=torch.int32).cuda()
    batch = PagedBatch(table, torch.tensor([0, 1], dtype=torch.int32).cuda(), kv_len, total_rows=1, max_rows=1, max_kv=320)
    rows = make_rows(gen, 100, 2, heads, dim).cuda()
    k, v = rows[0, :1].clone(), rows[0, 1:].clone()
    q, out, lse = make_rows(gen, 1, 8, dim).cuda(), torch.zeros(1, 8, dim, dtype=torch.bfloat16).cuda(), torch.zeros(1, 8).cuda()

    def step():
        kv_len.add_(1)
        cache.write(k, v, batch)
        cache.attend(q, batch, out=out, lse=lse)

    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        step()
        kv_len.zero_()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            step()
    torch.cuda.synchronize()
    seen = []
    for i in range(100):
        k.copy_(rows[i, :1]), v.copy_(rows[i, 1:])
        graph.replay()
        seen.append((out.clone(), lse.clone()))
    torch.cuda.synchronize()
    assert int(kv_len) == 100
    u = ref.quantise(rows.cpu(), "u8")
    held = ref.values(*u)
    for i in (0, 1, 31, 32, 99):
        o, l, weight, size = ref.attend(q.double().cpu(), held[:i + 1, 0], held[:i + 1, 1], dim ** -0.5)
        assert ((seen[i][0].double().cpu() - o).abs() <= bounds("u8", weight, size, o, i + 1, 20.0)).all(), i


def test_offsets_past_32_bits():
    """Pages whose bytes lie more than 4 GiB apart, and rows whose numbers pass 2^31 bytes."""
    page, dim, heads = 64, 128, 1
    gen = torch.Generator().manual_seed(101)
    base = torch.zeros((3, 1 << 30), dtype=torch.bfloat16, device="cuda")  # 2 GiB apart each
    k = base.as_strided((3, heads, page, dim), (1 << 30, page * dim, dim, 1))
    v = base.as_strided((3, heads, page, dim), (1 << 30, page * dim, dim, 1), (1 << 29))
    cache = PagedCache.from_tensors("bf16", k, v)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32).cuda()
    n = 180
    rows = make_rows(gen, 2, n, heads, dim)
    fill = PagedBatch(table, torch.tensor([0, n], dtype=torch.int32).cuda(), torch.tensor([n], dtype=torch.int32).cuda(),
                      total_rows=n, max_rows=n, max_kv=192)
    cache.write(rows[0].cuda(), rows[1].cuda(), fill)
    assert torch.equal(k[2, 0].cpu(), rows[0, :64, 0]) and torch.equal(v[1, 0, :52].cpu(), rows[1, 128:, 0])
    for m in (1, 50):
        batch = PagedBatch(table, torch.tensor([0, m], dtype=torch.int32).cuda(), fill.kv_len, total_rows=m, max_rows=m, max_kv=192)
        q = make_rows(gen, m, 4, dim)
        out = cache.attend(q.cuda(), batch)
        o, l, weight, size = ref.attend(q.double(), rows[0].double(), rows[1].double(), dim ** -0.5)
        assert ((out.double().cpu() - o).abs() <= bounds("bf16", weight, size, o, n, 1.0)).all()


def test_refusals_on_the_gpu():
    """A workspace that is too small is refused before anything runs; empty batches are accepted."""
    gen = torch.Generator().manual_seed(111)
    s = Setup(gen, "bf16", 1, 128, 16, [20000], [1])  # long enough to need a workspace
    q = make_rows(gen, 1, 8, 128).cuda()
    with pytest.raises(ipv.IpvError, match="workspace"):
        s.cache.attend(q, s.batch, workspace=torch.empty(256, dtype=torch.uint8, device="cuda"))
    none = PagedBatch(None, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(0, dtype=torch.int32, device="cuda"),
                      total_rows=0, max_rows=0, max_kv=0)
    assert s.cache.attend(q[:0], none).shape == (0, 8, 128)
    s.cache.write(q[:0, :1], q[:0, :1], none)


def test_a_wait_that_runs_out_is_reported():
    """With no time to wait the many-row kernel gives up, says so and leaves the device usable."""
    gen = torch.Generator().manual_seed(121)
    s = Setup(gen, "bf16", 1, 128, 64, [900], [100])
    assert ipv.attend_error() == 0
    ipv.attend_wait_limit(1)
    try:
        run_attend(s, 8, 122)
        assert ipv.attend_error() != 0
    finally:
        ipv.attend_wait_limit(0)
    q, out, lse = run_attend(s, 8, 122)
    assert ipv.attend_error() == 0
    check_attend(s, q, out, lse, 128 ** -0.5)


SHARED_OUT = [  # fmt, dim, heads, share, page, sequences (rows, kv) as a function of an index, how many, kwargs
    ("bf16", 64, 1, 2, 16, lambda b: (1, (b * 37) % 190), 500, {}),              # more sequences than a block has threads
    ("u4", 64, 2, 8, 16, lambda b: (1, (b * 53) % 410), 40, {}),                  # more than a warp has lanes
    ("u8", 128, 1, 7, 32, lambda b: (b % 3, 60 + (b * 29) % 200), 150, {"window": 40, "sinks": 2}),
    ("bf16", 64, 1, 4, 16, lambda b: (5 + b % 60, 70 + (b * 31) % 100), 420, {}),  # tiled kernel, more tiles than threads
    ("bf16", 128, 2, 3, 64, lambda b: (100 * (b % 4), 300 * (b % 4) + 3), 37, {}),
    ("u4", 128, 1, 4, 64, lambda b: (90, 150 + 20 * b), 12, {"window": 64, "sinks": 10}),
    ("bf16", 128, 1, 1, 16, lambda b: (1, 40000), 1, {}),                         # one tile over every block
    ("u8", 64, 1, 3, 16, lambda b: (1, 33000 - 999 * b), 3, {}),
    ("bf16", 64, 1, 1, 64, lambda b: (24, 40000), 1, {}),
    ("bf16", 128, 1, 8, 256, lambda b: (700, 5000), 1, {}),                       # many tiles, several to a block
    ("bf16", 128, 5, 1, 64, lambda b: (2500, 2500), 1, {"window": 300, "sinks": 129}),
]


@pytest.mark.parametrize("case", range(len(SHARED_OUT)))
def test_work_shared_out_over_blocks(case):
    """Batches whose tiles, runs and parts fall on the blocks in every way: many small sequences, one long one,
    tiles that start, continue and end in different blocks."""
    fmt, dim, heads, share, page, seq, count, kw = SHARED_OUT[case]
    gen = torch.Generator().manual_seed(1000 + case)
    seqs = [seq(b) for b in range(count)]
    s = Setup(gen, fmt, heads, dim, page, [n for _, n in seqs], [min(r, max(n, 1)) for r, n in seqs])
    q, out, lse = run_attend(s, share, 1100 + case, **kw)
    check_attend(s, q, out, lse, dim ** -0.5, **kw)


@pytest.mark.parametrize("fmt,dim,heads,share,seqs,kw", [
    ("bf16", 128, 4, 7, [(1, 600)], {}),
    ("bf16", 64, 2, 8, [(1, 1500), (1, 3), (0, 40), (2, 4000)], {}),
    ("bf16", 96, 3, 3, [(5, 900), (1, 0)], {}),
    ("u8", 128, 2, 7, [(1, 4000), (1, 513)], {}),
    ("u8", 64, 1, 16, [(1, 8000)], {"causal": False}),
    ("u4", 128, 4, 5, [(1, 2000), (3, 700), (2, 1)], {"window": 600, "sinks": 33}),
    ("u4", 64, 8, 8, [(1, 5000)], {}),
])
def test_clusters(fmt, dim, heads, share, seqs, kw):
    """Row tiles that 8 blocks of a cluster share, some with fewer steps than blocks, or none."""
    gen = torch.Generator().manual_seed(dim + share)
    s = Setup(gen, fmt, heads, dim, 32, [n for _, n in seqs], [r for r, _ in seqs])
    q, out, lse = run_attend(s, share, 151, **kw)
    check_attend(s, q, out, lse, dim ** -0.5, **kw)


@pytest.mark.parametrize("fmt,dim,heads,share,seqs,kw", [
    ("bf16", 128, 2, 7, [(9, 9), (3, 200), (8, 450)], {}),                     # whole contexts, several row tiles
    ("bf16", 64, 1, 4, [(16, 3000)], {"window": 900, "sinks": 7}),             # clusters
    ("bf16", 112, 2, 3, [(20, 20000), (1, 5), (0, 9), (13, 777)], {}),         # shares
    ("u8", 128, 3, 8, [(8, 400), (2, 2)], {}),
    ("u8", 64, 1, 16, [(4, 2500)], {"causal": False}),
    ("u8", 128, 2, 7, [(9, 9000), (9, 300), (4, 4000)], {}),
    ("u4", 64, 2, 1, [(64, 64), (33, 500)], {"window": 20, "sinks": 1}),
    ("u4", 128, 1, 2, [(17, 1700), (32, 32)], {}),
    ("u4", 128, 4, 7, [(7, 3000 + 50 * b) for b in range(9)], {}),
])
def test_several_row_tiles(fmt, dim, heads, share, seqs, kw):
    """17 to 64 query rows per KV head: a few row tiles of 16, their last one ragged."""
    gen = torch.Generator().manual_seed(dim * 7 + share)
    s = Setup(gen, fmt, heads, dim, 32, [n for _, n in seqs], [r for r, _ in seqs])
    q, out, lse = run_attend(s, share, 161, **kw)
    check_attend(s, q, out, lse, dim ** -0.5, **kw)


@pytest.mark.parametrize("rows", [1, 40])
def test_bounds_may_be_loose(rows):
    """max_rows, max_kv and total_rows far above what the sequences have."""
    gen = torch.Generator().manual_seed(131)
    s = Setup(gen, "bf16", 2, 128, 16, [300, 0, 77], [rows, 0, min(rows, 30)], max_rows=3 * rows, max_kv=100000)
    s.batch = PagedBatch(s.batch.table, s.batch.row_start, s.batch.kv_len, total_rows=s.total + 50, max_rows=3 * rows, max_kv=100000)
    q = (torch.randn((s.total + 50, 6, 128), generator=gen) * 1.5).bfloat16()
    out = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full(q.shape[:2], 7.0, device="cuda")
    s.cache.attend(q.cuda(), s.batch, out=out, lse=lse)
    check_attend(s, q, out, lse, 128 ** -0.5)
    assert (out[s.total:] == 7.0).all() and (lse[s.total:] == 7.0).all()  # rows of no sequence are left alone


def test_stream_of_its_own_without_a_workspace_is_refused():
    gen = torch.Generator().manual_seed(141)
    s = Setup(gen, "bf16", 1, 128, 16, [20000], [1])  # long enough to need a workspace
    q = make_rows(gen, 1, 8, 128).cuda()
    side = torch.cuda.Stream()
    with pytest.raises(ValueError, match="workspace"):
        s.cache.attend(q, s.batch, stream=side)
    want = s.cache.attend(q, s.batch)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):  # the current stream's own workspace
        out = s.cache.attend(q, s.batch)
    torch.cuda.synchronize()
    assert torch.equal(out, want)


@pytest.mark.parametrize("fmt,rows", [("bf16", 1), ("bf16", 40), ("u4", 3), ("u8", 30)])
def test_sequences_that_share_their_pages(fmt, rows):
    """A table of one row, expanded: several questions over one cache, each from a length of its own."""
    gen = torch.Generator().manual_seed(171)
    s = Setup(gen, fmt, 2, 128, 16, [700], [1])
    lens = [700, 333, 40]
    batch = PagedBatch(s.batch.table.expand(3, -1), torch.tensor([0, rows, 2 * rows, 3 * rows], dtype=torch.int32).cuda(),
                       torch.tensor(lens, dtype=torch.int32).cuda(), total_rows=3 * rows, max_rows=rows, max_kv=700)
    q = (torch.randn((3 * rows, 8, 128), generator=gen) * 1.5).bfloat16()
    lse = torch.zeros((3 * rows, 8), device="cuda")
    out = s.cache.attend(q.cuda(), batch, lse=lse)
    s.k, s.v = [s.k[0][:n] for n in lens], [s.v[0][:n] for n in lens]
    s.rows, s.lens, s.start = [rows] * 3, lens, np.arange(4) * rows
    check_attend(s, q, out, lse, 128 ** -0.5)


@pytest.mark.parametrize("as_number", [False, True])
def test_new_results_on_a_named_stream(as_number):
    """The results of a call on a stream of its own are not touched by the current stream, which is far behind."""
    gen = torch.Generator().manual_seed(181)
    s = Setup(gen, "u8", 2, 128, 16, [300, 90], [1, 3])
    q = make_rows(gen, 4, 8, 128).cuda()
    want, rows = s.cache.attend(q, s.batch), s.cache.read(s.batch)
    assert want.abs().sum() > 0
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        torch.cuda._sleep(20_000_000)  # the current stream's work: about 10 ms
        at = side.cuda_stream if as_number else side
        out, (k, v) = s.cache.attend(q, s.batch, stream=at), s.cache.read(s.batch, stream=at)
        side.synchronize()
        with torch.cuda.stream(side):
            got = [t.clone() for t in (out, k, v)]
        torch.cuda.synchronize()
        for t in got, (out, k, v):
            assert torch.equal(t[0], want) and torch.equal(t[1], rows[0]) and torch.equal(t[2], rows[1])


def long_cache(gen, fmt="bf16", heads=1, kv=20000):
    """Single tokens over this need a workspace."""
    return Setup(gen, fmt, heads, 128, 64, [kv], [1])


def workspace_need(cache, batch, n_q_heads, **kw):
    args = ipv.AttendArgs(n_q_heads=n_q_heads, scale=1.0, causal=int(kw.get("causal", True)), window=kw.get("window", 0),
                          sinks=kw.get("sinks", 0))
    return ipv.attend_workspace(cache.ref, batch.ref, args)


def test_a_graph_keeps_its_workspace():
    """A captured step whose plan needs a workspace, replayed after the stream's kept workspace has been replaced by a
    larger one and the memory of the first one has gone to other tensors."""
    gen = torch.Generator().manual_seed(191)
    s = long_cache(gen)
    need = workspace_need(s.cache, s.batch, 8)
    chunk = PagedBatch(s.batch.table, torch.tensor([0, 90], dtype=torch.int32).cuda(), s.batch.kv_len, total_rows=90, max_rows=90,
                       max_kv=20000)
    assert 0 < need < workspace_need(s.cache, chunk, 8)
    q, big = make_rows(gen, 1, 8, 128).cuda(), make_rows(gen, 90, 8, 128).cuda()
    side, out = torch.cuda.Stream(), torch.zeros(1, 8, 128, dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        s.cache.attend(q, s.batch, out=out)
        want = out.clone()
        side.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            s.cache.attend(q, s.batch, out=out)
        after = s.cache.attend(big, chunk)
        others = [torch.full((need,), 77, dtype=torch.uint8, device="cuda") for _ in range(6)]
        for _ in range(3):
            out.zero_()
            graph.replay()
            assert torch.equal(out, want)
        assert all(bool((t == 77).all()) for t in others)
        assert torch.equal(s.cache.attend(big, chunk), after)


def test_two_graphs_and_two_streams_at_once():
    """Two graphs over one cache, captured one after the other, and eager calls on two more streams, all in flight
    together: none shares a workspace with another."""
    gen = torch.Generator().manual_seed(192)
    s = long_cache(gen, heads=2)
    assert workspace_need(s.cache, s.batch, 16) > 0
    q = [make_rows(gen, 1, 16, 128).cuda() for _ in range(4)]
    want = [s.cache.attend(x, s.batch).clone() for x in q]
    outs, graphs = [torch.zeros_like(x) for x in q], []
    torch.cuda.synchronize()
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            s.cache.attend(q[i], s.batch, out=outs[i])
        graphs.append(graph)
    streams = [torch.cuda.Stream() for _ in range(4)]
    for _ in range(50):
        for o in outs:
            o.fill_(7.0)
        torch.cuda.synchronize()
        for i, st in enumerate(streams):
            with torch.cuda.stream(st):
                for _ in range(4):
                    if i < 2:
                        graphs[i].replay()
                    else:
                        s.cache.attend(q[i], s.batch, out=outs[i])
        torch.cuda.synchronize()
        for o, w in zip(outs, want):
            assert torch.equal(o, w)


@pytest.mark.parametrize("fmt,rows,kv", [("bf16", 100, 900), ("u8", 70, 3000), ("bf16", 90, 300)])
def test_outputs_are_left_alone_when_a_wait_runs_out(fmt, rows, kv):
    """A block that gave up has no results: no query gets one made of what the workspace held, here an earlier call's
    parts of the same tiles (the last case: whole contexts, without parts)."""
    gen = torch.Generator().manual_seed(201)
    s = Setup(gen, fmt, 2, 128, 64, [kv], [rows])
    need = workspace_need(s.cache, s.batch, 16)
    ws = torch.empty(max(need, 256), dtype=torch.uint8, device="cuda")
    q, out, lse = run_attend(s, 8, 202, workspace=ws)
    check_attend(s, q, out, lse, 128 ** -0.5)
    assert ipv.attend_error() == 0
    ipv.attend_wait_limit(1)
    try:
        _, held, lse_held = run_attend(s, 8, 202, workspace=ws)
        assert ipv.attend_error() != 0
    finally:
        ipv.attend_wait_limit(0)
    assert (held == 7.0).all() and (lse_held == 7.0).all()
    _, again, lse_again = run_attend(s, 8, 202, workspace=ws)
    assert ipv.attend_error() == 0 and torch.equal(again, out) and torch.equal(lse_again, lse)


@pytest.mark.parametrize("fmt", ["bf16", "u8", "u4"])
@pytest.mark.parametrize("rows", [2, 120])
@pytest.mark.parametrize("sinks", [2 ** 31 - 1, 2 ** 31 - 128, 700])
def test_sinks_that_cover_everything(fmt, rows, sinks):
    """As many first rows as the header takes, and a workspace that is full of NaN."""
    gen = torch.Generator().manual_seed(211)
    s = Setup(gen, fmt, 1, 64, 64, [900], [rows])
    ws = torch.empty(max(256, workspace_need(s.cache, s.batch, 4, window=10, sinks=sinks)), dtype=torch.uint8, device="cuda").fill_(255)
    q, out, lse = run_attend(s, 4, 212, window=10, sinks=sinks, workspace=ws)
    check_attend(s, q, out, lse, 64 ** -0.5, window=10, sinks=sinks)


@pytest.mark.parametrize("fmt", ["bf16", "u8"])
def test_rows_rewritten_and_read_back_in_one_go(fmt):
    """Writes and reads of the same rows, launched one behind the other: each read returns what the write before it wrote."""
    gen = torch.Generator().manual_seed(221)
    cache = PagedCache(8, 16, 4, 128, fmt)
    table = torch.randperm(8, generator=gen).to(torch.int32)[None].cuda()
    batch = PagedBatch(table, torch.tensor([0, 40], dtype=torch.int32).cuda(), torch.tensor([100], dtype=torch.int32).cuda(),
                       total_rows=40, max_rows=40, max_kv=128)
    rows = make_rows(gen, 200, 40, 4, 128)
    x = rows.cuda()
    outs = torch.zeros((200, 2, 40, 4, 128), dtype=torch.bfloat16, device="cuda")
    torch.cuda.synchronize()
    for i in range(200):
        cache.write(x[i], x[199 - i], batch)
        cache.read(batch, outs[i, 0], outs[i, 1])
    torch.cuda.synchronize()
    want = rows if fmt == "bf16" else ref.values(*ref.quantise(rows, fmt)).float().bfloat16()
    assert torch.equal(outs[:, 0].cpu(), want) and torch.equal(outs[:, 1].cpu(), want.flip(0))


@pytest.mark.parametrize("fmt", ["bf16", "u8", "u4"])
@pytest.mark.parametrize("rows", [1, 20, 90])
def test_nothing_is_cached(fmt, rows):
    """No sequence holds a row, and the bound says so: 0 and -inf for every query."""
    gen = torch.Generator().manual_seed(231)
    s = Setup(gen, fmt, 2, 64, 16, [0, 0], [rows, 3])
    assert s.batch.max_kv == 0
    q, out, lse = run_attend(s, 4, 232)
    assert (out == 0).all() and (lse == -math.inf).all()


@pytest.mark.parametrize("seqs,rows,kv,tiled", [(1, 8, 9000, False), (16, 9, 600, True), (16, 3, 6000, True)])
def test_which_kernel_takes_a_few_rows_over_bf16_pages(seqs, rows, kv, tiled):
    """The measured cases that the limit between the two kernels was drawn from, 7 query heads for each of 4 KV heads:
    the workspace of parts is that of 256-row tiles, or of 16-row ones."""
    cache = PagedCache(1, 64, 4, 128)
    table = torch.zeros((seqs, -(-kv // 64)), dtype=torch.int32, device="cuda")
    batch = PagedBatch(table, torch.arange(seqs + 1, dtype=torch.int32, device="cuda") * rows,
                       torch.full((seqs,), kv, dtype=torch.int32, device="cuda"), total_rows=seqs * rows, max_rows=rows, max_kv=kv)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    per_sm = workspace_need(cache, batch, 28) / sms
    assert per_sm >= 2 * 256 * 128 * 4 if tiled else per_sm < 2 * 64 * 128 * 4


SHARED_LISTS = [  # fmt, dim, heads, share, page, sequences (rows, kv) as a function of an index, how many, kwargs
    # rows kernel, more (sequence, tile) pairs than a block's 128 threads
    ("bf16", 64, 1, 2, 16, lambda b: (1, 900 if b % 97 == 50 else (b * 37) % 190), 500, {}),
    ("u4", 64, 2, 8, 16, lambda b: (1, 4000 if b == 399 else (b * 53) % 410), 400, {}),
    ("u8", 128, 1, 7, 32, lambda b: (b % 3, 60 + (b * 29) % 800), 270, {"window": 640, "sinks": 2}),
    ("bf16", 128, 1, 16, 64, lambda b: (1 if b in (0, 299) else 0, 5000 if b in (0, 299) else 20), 300, {}),
    # tiled kernel, more pairs than its 384 threads
    ("bf16", 64, 1, 4, 16, lambda b: (5 + b % 60, 900 if b % 150 == 149 else 70 + (b * 31) % 100), 800, {}),
    ("u8", 64, 1, 3, 16, lambda b: (b % 31, 1500 if b == 0 else 40 + (b * 17) % 90), 450, {"window": 1000, "sinks": 3}),
    ("bf16", 128, 1, 1, 32, lambda b: (600 if b == 410 else 65 if b % 40 == 3 else 0, 700 if b == 410 else 66), 411, {}),
    # one pair more than a warp's lanes, a block's threads
    ("u4", 128, 2, 5, 64, lambda b: (1, 600 + b), 33, {}),
    ("bf16", 96, 1, 8, 16, lambda b: (1, 513 + b), 129, {}),
    ("bf16", 64, 1, 1, 64, lambda b: (65, 513 + b % 50), 385, {}),
]


@pytest.mark.parametrize("case", range(len(SHARED_LISTS)))
def test_long_lists_shared_out_over_blocks(case):
    """Batches with more sequences than a block looks at together, too long for whole contexts and too many for clusters:
    the blocks' shares are found in several passes over the list."""
    fmt, dim, heads, share, page, seq, count, kw = SHARED_LISTS[case]
    gen = torch.Generator().manual_seed(3000 + case)
    seqs = [seq(b) for b in range(count)]
    s = Setup(gen, fmt, heads, dim, page, [n for _, n in seqs], [min(r, max(n, 1)) for r, n in seqs])
    widened = 0
    if fmt != "bf16" and max(s.rows) * share > 64:
        widened = 2 * (-(-len(seqs) * heads * max(s.lens) * dim * 2 // 256) * 256)
    assert workspace_need(s.cache, s.batch, heads * share, **kw) > widened  # parts: the work is shared out
    q, out, lse = run_attend(s, share, 3100 + case, **kw)
    check_attend(s, q, out, lse, dim ** -0.5, **kw)


def test_sixteen_row_tiles_shared_out():
    """17 to 64 bf16 query rows per KV head in the rows kernel, too long for whole contexts and clusters."""
    gen = torch.Generator().manual_seed(241)
    seqs = [(20, 5000), (1, 5), (0, 9), (13, 777)]
    s = Setup(gen, "bf16", 2, 112, 32, [n for _, n in seqs], [r for r, _ in seqs])
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert 0 < workspace_need(s.cache, s.batch, 6) < sms * 2 * 256 * 112 * 4  # parts of 16 rows, not of 256
    q, out, lse = run_attend(s, 3, 242)
    check_attend(s, q, out, lse, 112 ** -0.5)


@pytest.mark.parametrize("fmt,dim,heads,share,lens,rows", [
    ("u8", 128, 2, 7, [9000, 17000], [1, 1]), ("u4", 64, 1, 5, [30000], [2]), ("bf16", 128, 1, 8, [20000], [1]),
    ("bf16", 128, 1, 7, [3000, 700], [61, 33]), ("u8", 128, 1, 7, [2000, 900], [40, 70])])
def test_what_a_workspace_held_does_not_matter(fmt, dim, heads, share, lens, rows):
    """The same bits from a workspace full of NaN and full of zeros, on the current stream and on another."""
    gen = torch.Generator().manual_seed(251)
    s = Setup(gen, fmt, heads, dim, 64, lens, rows)
    need = workspace_need(s.cache, s.batch, heads * share)
    assert need > 0
    q = make_rows(gen, s.total, heads * share, dim).cuda()
    want, side = s.cache.attend(q, s.batch), torch.cuda.Stream()
    ws = torch.empty(need, dtype=torch.uint8, device="cuda")
    for fill in (255, 0, 255):
        out = torch.zeros_like(q)
        ws.fill_(fill)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            s.cache.attend(q, s.batch, out=out, workspace=ws)
        side.synchronize()
        assert torch.equal(out, want)


@pytest.mark.parametrize("dim", [8, 40, 56])
@pytest.mark.parametrize("page,seqs,kw", [
    (16, [(70, 300), (3, 40), (100, 100)], {}), (128, [(200, 1500)], {"window": 130, "sinks": 9}), (64, [(90, 800)], {"causal": False})])
def test_narrow_heads_in_the_tiled_kernel(dim, page, seqs, kw):
    """Rows shorter than the 64 channels of a copy."""
    gen = torch.Generator().manual_seed(261 + dim)
    s = Setup(gen, "bf16", 2, dim, page, [n for _, n in seqs], [r for r, _ in seqs])
    q, out, lse = run_attend(s, 2, 262, **kw)
    check_attend(s, q, out, lse, dim ** -0.5, **kw)
