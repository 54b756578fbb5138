"""The calls around chosen pages at sizes that take other ways through the kernels than test_gpu_chosen.py's: rows by the
thousand, whole caches' bounds, more lists than blocks, lists of thousands of keys in one block, work that is shared out with a
workspace. Against the same float64 definitions, within the same bounds; plain forms of these sizes run on the GPU in float64."""
import math

import pytest

torch = pytest.importorskip("torch")

import chosen_ref as cref  # noqa: E402
from paper_2506_15745_gb300 import ipv  # noqa: E402
from paper_2506_15745_gb300.cache import PingPongCache  # noqa: E402
from paper_2506_15745_gb300.paged import PageBounds, PagedBatch, PagedCache, Rotary  # noqa: E402
from test_gpu_chosen import Choice, check_chosen, ints, parts, random_lists, run_chosen, same_bits, turns  # noqa: E402
from test_gpu_chosen_forms import chosen_need  # noqa: E402
from test_gpu_paged import Setup, make_rows  # noqa: E402

pytestmark = pytest.mark.gpu


def pool_and_batch(gen, fmt, heads, dim, page, seqs, spare_rows=0):
    """An empty pool and a batch over it of sequences of (rows, kv); spare packed rows behind the last one."""
    held = [-(-n // page) for _, n in seqs]
    order, at = torch.randperm(sum(held) + 2, generator=gen).to(torch.int32), 0
    table = torch.full((len(seqs), max(held)), -1, dtype=torch.int32)
    for b, n in enumerate(held):
        table[b, :n] = order[at:at + n]
        at += n
    start = [0]
    for r, _ in seqs:
        start.append(start[-1] + r)
    cache = PagedCache(sum(held) + 2, page, heads, dim, fmt)
    batch = PagedBatch(table.cuda(), ints(*start), ints(*[n for _, n in seqs]), total_rows=start[-1] + spare_rows,
                       max_rows=max(r for r, _ in seqs), max_kv=max(n for _, n in seqs))
    return cache, batch, start[-1]


# ------------------------------------------------------------------- rotated writes
def turned(x, weight, eps, table, at, sections, interleaved):
    """chosen_ref.turned for whole tensors."""
    x = x.double()
    rot = table.shape[1]
    if weight is not None:
        x = x * weight.double() / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    axis = torch.repeat_interleave(torch.arange(len(sections)), torch.tensor(sections)).to(x.device)
    f = torch.arange(rot // 2, device=x.device)
    places = at[axis].long()                                     # [frequencies, rows]
    c, s = (table.double()[places, f[:, None] + k].t()[:, None] for k in (0, rot // 2))
    i, j = (2 * f, 2 * f + 1) if interleaved else (f, f + rot // 2)
    a, b = x[..., i], x[..., j]
    out, size = x.clone(), x.abs()
    out[..., i], out[..., j] = a * c - b * s, b * c + a * s
    size[..., i], size[..., j] = (a * c).abs() + (b * s).abs(), (b * c).abs() + (a * s).abs()
    return out, size


FORMS = [  # dim, heads, share, page, rot, sections, interleaved, norms
    (128, 4, 7, 64, 128, [32, 16, 16], False, "qk"),
    (128, 3, 4, 32, 96, [48], False, "k"),
    (128, 2, 3, 16, 64, [16, 16], False, "qk"),
    (128, 4, 5, 64, 128, [64], True, "q"),
    (64, 5, 1, 32, 64, [32], False, "qk"),
    (64, 2, 8, 64, 32, [8, 8], True, ""),
]


@pytest.mark.parametrize("fmt", ["bf16", "u8", "u4"])
@pytest.mark.parametrize("rows", [1000, 2800])  # two warps for a row (above 912), one (above 2736)
@pytest.mark.parametrize("form", range(len(FORMS)))
def test_many_rotated_rows(form, rows, fmt):
    dim, heads, share, page, rot, sections, interleaved, norms = FORMS[form]
    gen = torch.Generator().manual_seed(rows + form)
    seqs = [(rows - 340, rows), (0, 7), (1, 1), (300, 1000), (39, 100)]
    cache, batch, total = pool_and_batch(gen, fmt, heads, dim, page, seqs, spare_rows=3)
    q, k, v = (make_rows(gen, total + 3, h, dim).cuda() for h in (heads * share, heads, heads))
    w = {x: (1 + 0.3 * torch.randn(dim, generator=gen)).bfloat16().cuda() if x in norms else None for x in "qk"}
    table, at = turns(gen, 50, rot).cuda(), torch.randint(0, 50, (len(sections), total + 3), generator=gen, dtype=torch.int32).cuda()
    rotary = Rotary(table, sections, interleaved)
    before = [t.clone() for t in parts(cache)]
    out = torch.full_like(q, 5.0)
    call = lambda c, o: c.write_rotated(q, k, v, batch, rotary, at, q_weight=w["q"], k_weight=w["k"], eps=1e-3, q_out=o)  # noqa: E731
    call(cache, out)
    assert (out[total:] == 5.0).all()
    tol = lambda want, size: 2.0 ** -8 * want.abs() + 2.0 ** -16 * size + 1e-38  # noqa: E731
    want, size = turned(q, w["q"], 1e-3, table, at, sections, interleaved)
    assert ((out.double() - want).abs() <= tol(want, size))[:total].all()
    plain = PagedCache(cache.n_pages, page, heads, dim)
    call(plain, out)
    k_back, v_back = plain.read(batch)
    want, size = turned(k, w["k"], 1e-3, table, at, sections, interleaved)
    assert ((k_back.double() - want).abs() <= tol(want, size))[:total].all() and same_bits(v_back[:total], v[:total])
    after = [t.clone() for t in parts(cache)]
    for t, old in zip(parts(cache), before):
        t.copy_(old)
    cache.write(k_back, v_back, batch)
    assert all(same_bits(a, t) for a, t in zip(after, parts(cache)))  # the whole pool: nothing else was touched
    again = q.clone()  # in place
    cache.write_rotated(again, k, v, batch, rotary, at, q_weight=w["q"], k_weight=w["k"], eps=1e-3, q_out=again)
    assert same_bits(again[:total], out[:total]) and same_bits(again[total:], q[total:])


# ------------------------------------------------------------------- bounds of whole caches
def bounds_of(k):
    """Keys [..., rows, dim] -> codes [..., 2, dim], steps [...], by chosen_ref's rule."""
    k = k.double()
    top = k.abs().amax((-1, -2))
    m, e = torch.frexp(top)  # top = m 2^e, 1/2 <= m < 1: at most 127 of 2^(e - 7) if m <= 127/128, else of 2^(e - 6)
    e = torch.where(m * 128.0 <= 127.0, e - 7, e - 6).clamp(min=-40).long()
    step = (e + 1023 << 52).view(torch.float64)  # 2^e to the bit, which a device's pow does not promise
    lo, hi = (k.amin(-2) / step[..., None]).floor(), (k.amax(-2) / step[..., None]).ceil()
    return torch.stack([lo, hi], -2), step


@pytest.mark.parametrize("fmt,dim,page", [("bf16", 128, 64), ("bf16", 64, 64), ("bf16", 72, 128), ("u8", 128, 64), ("u8", 64, 64), ("u4", 128, 64),
                                          ("u4", 64, 128)])
def test_bounds_of_a_whole_cache(fmt, dim, page):
    """More than 2048 pages and heads, of more rows than a warp reads at once: a warp for each, several rounds."""
    gen = torch.Generator().manual_seed(dim)
    heads, seqs = 16, [(page * 90 + 5,) * 2, (page * 50,) * 2, (page + 1,) * 2]
    cache, batch, total = pool_and_batch(gen, fmt, heads, dim, page, seqs)
    k, v = make_rows(gen, total, heads, dim).cuda(), make_rows(gen, total, heads, dim).cuda()
    if fmt == "bf16":
        for t in (cache.k, cache.v):
            t.fill_(math.nan)  # behind the last rows
    cache.write(k, v, batch)
    made = PageBounds(cache)
    made.codes.fill_(77), made.steps.fill_(77.0)
    made.update(cache, batch)
    k = cache.read(batch)[0]
    want_codes, want_steps = torch.full_like(made.codes, 77), torch.full_like(made.steps, 77.0)
    row = 0
    for b, (n, _) in enumerate(seqs):
        for i in range(-(-n // page)):
            g, rows = int(batch.table[b, i]), min(page, n - i * page)
            codes, step = bounds_of(k[row:row + rows].transpose(0, 1))
            want_codes[g] = 0
            want_codes[g, ..., :dim], want_steps[g] = codes.to(torch.int8), step.float()
            row += rows
    assert sum(-(-n // page) for n, _ in seqs) * heads > 2048 and len(set(made.steps.flatten().tolist())) > 2
    assert torch.equal(made.steps, want_steps) and torch.equal(made.codes, want_codes)


# ------------------------------------------------------------------- more lists than blocks
@pytest.mark.parametrize("levels", [60, 1])
@pytest.mark.parametrize("dim,heads,share,n,seqs", [
    (128, 4, 8, 24, [(1, 8000 - 150 * b) for b in range(45)]),             # tokens of ragged streams, up to 500 pages
    (128, 4, 7, 24, [(61, 6400), (0, 5000), (2, 30)]),                     # a question's rows, each with lists of its own
    (64, 8, 3, 96, [(1, 16 * 300 + b) for b in range(24)]),
    (80, 2, 16, 300, [(60, 16 * 700), (60, 16 * 129)]),                    # more chosen than threads
])
def test_many_lists_over_many_pages(dim, heads, share, n, seqs, levels):
    """One block for each list, several rounds of pages for each of its warps."""
    c = Choice(len(seqs), seqs, heads, share, dim, 16, levels)
    rows = sorted({0, 1, 2, 30, 59, 60})
    got, want = c.run(n, 1, 2).cpu(), c.want(n, 1, 2, rows)
    some = want[:, 0, 0] != -2
    assert sum(r for r, _ in seqs) * heads > 152 and torch.equal(got[some], want[some])


# ------------------------------------------------------------------- long lists
LONG = [  # fmt, dim, heads, share, page, [(rows, kv)], n, whether work is shared out with a workspace (three blocks per SM; None: not said)
    ("bf16", 128, 8, 2, 64, [(50, 5000)], 70, False),                      # a block for each tile: 35 steps for each warp
    ("bf16", 128, 8, 2, 64, [(70, 5000), (0, 9), (12, 4990)], 70, False),  # blocks in turn
    ("bf16", 128, 8, 1, 64, [(63, 5000)], 70, True),                       # shared out
    ("u8", 128, 8, 2, 64, [(50, 5000)], 70, False),
    ("u8", 128, 8, 2, 64, [(70, 5000), (0, 9), (12, 4990)], 70, False),
    ("u8", 128, 8, 1, 64, [(63, 5000)], 70, True),
    ("u8", 128, 8, 3, 16, [(60, 800), (3, 20), (28, 900)], 36, False),     # in turn, ragged, shorter
    ("u4", 128, 8, 2, 64, [(50, 5000)], 70, False),
    ("u4", 128, 8, 2, 64, [(70, 5000), (0, 9), (12, 4990)], 70, False),
    ("u4", 128, 8, 1, 64, [(63, 5000)], 70, True),
    ("u4", 128, 8, 3, 16, [(60, 800), (3, 20), (28, 900)], 36, False),
    ("bf16", 64, 8, 2, 64, [(36, 5000)], 70, None),
    ("bf16", 64, 8, 2, 64, [(70, 5000), (12, 4990)], 70, None),
    ("u8", 64, 8, 2, 32, [(50, 5000)], 140, None),
    ("u4", 64, 8, 2, 32, [(90, 5000)], 140, None),
    ("bf16", 128, 2, 16, 64, [(45, 5000)], 70, None),                      # tiles of 16 query rows
    ("u8", 128, 2, 16, 64, [(80, 5000)], 70, None),
    ("u4", 128, 2, 12, 64, [(80, 5000)], 70, None),
    ("bf16", 128, 1, 1, 16, [(1, 70000), (2, 40000)], 3000, True),         # 48000 keys over all blocks
    ("u8", 128, 1, 1, 16, [(1, 70000), (2, 40000)], 3000, True),
]


@pytest.mark.parametrize("junk", [False, True])
@pytest.mark.parametrize("case", range(len(LONG)))
def test_long_lists(case, junk):
    """A warp takes more steps than it looks up at once, several times over; rings go on into the next tile."""
    fmt, dim, heads, share, page, seqs, n, shared = LONG[case]
    gen = torch.Generator().manual_seed(1500 + case)
    s = Setup(gen, fmt, heads, dim, page, [k for _, k in seqs], [r for r, _ in seqs])
    chosen = random_lists(gen, s, n, junk)
    if shared is not None:
        assert (chosen_need(s.cache, s.batch, heads * share, n) > 0) == shared
    q, out, lse = run_chosen(s, share, chosen, 1600 + case)
    check_chosen(s, q, chosen, out, lse, dim ** -0.5)


# ------------------------------------------------------------------- workspaces
def shared_out(gen, fmt):
    """Lists that blocks share with a workspace: 19200 keys each."""
    s = Setup(gen, fmt, 2, 128, 16, [20000, 19500], [2, 1])
    chosen = random_lists(gen, s, 1200)
    need = chosen_need(s.cache, s.batch, 14, 1200)
    assert need > 0
    return s, chosen, need


@pytest.mark.parametrize("fmt", ["bf16", "u8", "u4"])
def test_what_a_workspace_holds_does_not_matter(fmt):
    """Bytes of ones and bytes that an earlier call of other sizes left, on another stream; nothing behind its end is touched."""
    gen = torch.Generator().manual_seed(1700)
    s, chosen, need = shared_out(gen, fmt)
    q, want, lse = run_chosen(s, 7, chosen, 1701)
    check_chosen(s, q, chosen, want, lse, 128 ** -0.5)
    other = random_lists(gen, s, 900).cuda()
    assert 0 < chosen_need(s.cache, s.batch, 14, 900) <= need
    q, chosen = q.cuda(), chosen.cuda()
    side, ws = torch.cuda.Stream(), torch.empty(need + 4096, dtype=torch.uint8, device="cuda").fill_(255)
    torch.cuda.synchronize()
    for k in range(6):
        if k % 2:
            s.cache.attend_chosen(q, s.batch, other, workspace=ws[:need], stream=side)
        out = s.cache.attend_chosen(q, s.batch, chosen, workspace=ws[:need], stream=side)
        side.synchronize()
        assert same_bits(out, want)
    assert (ws[need:] == 255).all()


def test_graphs_with_workspaces_of_their_own():
    """Two captured calls that are shared out, replayed at the same time on two streams, eager calls between and beside them."""
    gen = torch.Generator().manual_seed(1800)
    s, chosen, need = shared_out(gen, "bf16")
    lists = [chosen.cuda(), random_lists(gen, s, 1200).cuda()]
    q = [make_rows(gen, s.total, 14, 128).cuda() for _ in range(2)]
    want = [s.cache.attend_chosen(*x) for x in zip(q, (s.batch,) * 2, lists)]
    outs, graphs, streams = [torch.zeros_like(x) for x in q], [], [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    for i in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=streams[i]):
            s.cache.attend_chosen(q[i], s.batch, lists[i], out=outs[i])
        graphs.append(graph)
    torch.cuda.synchronize()
    for _ in range(5):
        for t in outs:
            t.zero_()
        torch.cuda.synchronize()
        for g, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                g.replay()
        again = s.cache.attend_chosen(q[0], s.batch, lists[0])
        torch.cuda.synchronize()
        assert same_bits(outs[0], want[0]) and same_bits(outs[1], want[1]) and same_bits(again, want[0])


# ------------------------------------------------------------------- weights over bf16 pages
@pytest.mark.parametrize("dim,share,rows,kv,n", [(128, 7, 1, 1000, 70), (64, 7, 1, 1000, 70), (128, 16, 1, 1000, 70), (128, 2, 1, 4000, 250),
                                                 (128, 1, 82, 1200, 80), (128, 2, 1, 20000, 1250)])
def test_weights_have_16_bits_over_bf16_pages(dim, share, rows, kv, n):
    """Weights next to where bf16 rounds one way or the other, under values that cancel: a weight of 8 bits would be off by up to
    2^-8 sum p |v| in one direction.

    Scores are -log2 of 1, or of 1/2 plus a little less or a little more than half a step of bf16 there, held to 2^-16 by two
    channels; values are 1 where the weight rounds down and -1 where it rounds up. Of sum p |v| an output may be off by 2^-16 for
    the two bf16 parts of a weight, by twice the scores' error (2^-16 of their products), and by 2^-16 for fp32 sums: an
    accumulator takes 4 products for each 32 keys of its warp, 40 at most here, each off by 2^-22 at most."""
    gen = torch.Generator().manual_seed(1900)
    heads = 8 if rows > 1 else 2
    s = Setup(gen, "bf16", heads, dim, 16, [kv], [rows], garbage=False)
    up = torch.rand(kv, generator=gen) < 0.5
    x = -torch.log2(torch.where(up, 0.5 + 2.0 ** -9 * 1.05, 0.5 + 2.0 ** -9 * 0.95).double())
    high = x.bfloat16()
    k, v = torch.zeros(kv, heads, dim).bfloat16(), torch.where(up, -1.0, 1.0)[:, None, None].expand(kv, heads, dim).bfloat16()
    k[:, :, 0], k[:, :, 1] = high[:, None], (x - high.double()).bfloat16()[:, None]
    k[0, :, :2] = 0  # the largest score, weight 1
    whole = PagedBatch(s.batch.table, ints(0, kv), s.batch.kv_len, total_rows=kv, max_rows=kv, max_kv=kv)
    s.cache.write(k.cuda(), v.contiguous().cuda(), whole)
    q = torch.zeros(rows, heads * share, dim).bfloat16()
    q[..., :2] = -1
    chosen = torch.full((rows, heads, n), -1, dtype=torch.int32)
    for i in range(rows):
        pages = (kv - rows + i) // 16 + 1
        chosen[i, :, :min(n, pages)] = torch.arange(min(n, pages), dtype=torch.int32)
    scale = math.log(2.0)
    out = s.cache.attend_chosen(q.cuda(), s.batch, chosen.cuda(), scale=scale).double().cpu()
    o, _, weight, size = cref.attend(q.double(), k.double(), v.double(), chosen, 16, scale)
    tol = 2.0 ** -8 * o.abs() + (2.0 ** -15 + torch.expm1(2.0 * 2.0 ** -16 * size[..., None])) * weight
    assert ((out - o).abs() <= tol).all(), float(((out - o).abs() / tol).max())
    # The bound tells: weights rounded once to bf16 are outside of it.
    p = torch.exp2(-(k[:, 0, 0].double() + k[:, 0, 1].double()))[:16 * n if rows == 1 else kv]
    once = float((p.bfloat16().double() * v[:len(p), 0, 0].double()).sum() / p.sum())
    if rows == 1:
        assert abs(once - float(o[0, 0, 0])) > 4.0 * float(tol.max())


# ------------------------------------------------------------------- the pass's compaction
def test_a_gather_of_the_kept_rows_is_the_compaction():
    """The rows that the pass keeps of contiguous slabs, and a gather by ipv_select's indices of the same rows in pages."""
    layers, heads, dim, grid, frames, budget = 3, 2, 64, 4, 14, 96
    p, n_slabs, n = grid * grid, layers * heads, grid * grid * frames
    gen = torch.Generator().manual_seed(2000)
    ipv.init(device=0, dtype="bf16", max_head_dim=dim, max_frame_tokens=p, max_slabs=n_slabs, token_capacity=n)
    pp = PingPongCache(n_slabs, n, dim, "bf16")
    pp.k[0], pp.v[0] = make_rows(gen, n_slabs, n, dim).cuda(), make_rows(gen, n_slabs, n, dim).cuda()
    pp.n_tokens = n
    tar, van = torch.empty((n_slabs, n), device="cuda"), torch.empty((n_slabs, n), device="cuda")
    ipv.score(*pp.structs(False), layers, heads, dim, n, grid, grid, tar, van)
    kept = torch.empty((n_slabs, budget), dtype=torch.int32, device="cuda")
    ipv.select(tar, van, n_slabs, n, grid, grid, budget, 0.5, kept)
    pool = PagedCache(40, 16, n_slabs, dim)
    pages = torch.randperm(40, generator=gen).to(torch.int32).cuda()
    source = PagedBatch(pages[None, :14], ints(0, n), ints(n), total_rows=n, max_rows=n, max_kv=n)
    pool.write(pp.k[0].transpose(0, 1).contiguous(), pp.v[0].transpose(0, 1).contiguous(), source)
    whole = PagedBatch(pages[None, 14:20], ints(0, budget), ints(budget), total_rows=budget, max_rows=budget, max_kv=budget)
    pool.gather(pool, source, whole, kept[None])
    done = torch.empty_like(kept)
    pp.compress(layers, heads, grid, grid, budget, 0.5, done, pid_valid=False)
    k, v = pool.read(whole)
    assert torch.equal(done, kept)
    assert same_bits(k.transpose(0, 1), pp.k_live[:, :budget]) and same_bits(v.transpose(0, 1), pp.v_live[:, :budget])
