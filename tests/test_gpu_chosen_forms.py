"""Rotated writes, choices and attention over chosen pages in the forms that a call may take beside the usual ones: one long page
for each sequence, one place on all axes, queries and results inside
wider tensors, first uses."""
import math
import os
import subprocess
import sys

import pytest

torch = pytest.importorskip("torch")

import chosen_ref as cref  # noqa: E402
from paper_2506_15745_gb300 import ipv  # noqa: E402
from paper_2506_15745_gb300.paged import PageBounds, PagedBatch, PagedCache, Rotary  # noqa: E402
from test_gpu_chosen import ints, random_lists, same_bits, turns  # noqa: E402
from test_gpu_paged import Setup, bounds, make_rows  # noqa: E402

pytestmark = pytest.mark.gpu


def chosen_need(cache, batch, n_q_heads, n_chosen):
    """Bytes of workspace that attend_chosen takes for these sizes; 0 where no tile is shared out."""
    return ipv.attend_chosen_workspace(cache.ref, batch.ref, ipv.AttendArgs(n_q_heads=n_q_heads, scale=1.0, causal=1), ipv.Chosen(n_chosen=n_chosen))


@pytest.mark.parametrize("fmt,held", [("bf16", 300), ("bf16", 3000), ("u8", 300), ("u4", 1000)])
def test_a_page_may_be_longer_than_the_sequence(fmt, held):
    """One page per sequence, as of_layer gives: the work goes by the rows held, not by the page's length, so a longer page is shared
    out in the same way and gives the same bits."""
    gen = torch.Generator().manual_seed(held)
    lens, rows, heads, share, dim = [held, held // 3, 1], [2, 1, 1], 2, 4, 128
    q = make_rows(gen, 4, heads * share, dim)
    k, v = (make_rows(gen, sum(lens), heads, dim) for _ in range(2))
    chosen = torch.zeros((4, heads, 1), dtype=torch.int32, device="cuda")
    made = []
    for size in (held, 9408):
        cache = PagedCache(3, size, heads, dim, fmt)
        whole = PagedBatch(None, ints(0, lens[0], sum(lens[:2]), sum(lens)), ints(*lens), total_rows=sum(lens), max_rows=held, max_kv=held)
        cache.write(k.cuda(), v.cuda(), whole)
        batch = PagedBatch(None, ints(0, 2, 3, 4), ints(*lens), total_rows=4, max_rows=2, max_kv=held)
        assert chosen_need(cache, batch, heads * share, 1) == 0
        lse = torch.zeros(4, heads * share, device="cuda")
        made.append((cache.attend_chosen(q.cuda(), batch, chosen, lse=lse), lse, *cache.read(whole)))
    assert all(same_bits(a, b) for a, b in zip(*made))
    out, lse, k_held, v_held = made[0]
    at, row = 0, 0
    for n, r in zip(lens, rows):
        kk, vv = k_held[at:at + n].double().cpu(), v_held[at:at + n].double().cpu()
        o, l, weight, size = cref.attend(q[row:row + r].double(), kk, vv, chosen[row:row + r].cpu(), 9408, dim ** -0.5)
        tol = bounds(fmt, weight, size, o, n, float(vv.abs().max()))
        if fmt != "bf16":  # `read` rounds the codes' values to bf16: scores by 2^-8 of their products, values by 2^-8; a weight times
            # its group's step is rounded by 2^-11 of itself, which stands before a code of up to (largest - least) / step
            spread = float((vv.amax(-1) - vv.amin(-1)).max())
            tol = tol + (2.0 ** -8 + torch.expm1(2.0 * 2.0 ** -8 * size[..., None])) * weight * 1.01 + 2.0 ** -11 * spread * 1.02
        assert ((out[row:row + r].double().cpu() - o).abs() <= tol).all() and not math.isnan(float(lse.sum()))
        at, row = at + n, row + r


@pytest.mark.parametrize("interleaved", [False, True])
def test_one_place_on_all_axes(interleaved):
    """A text token has one position on every axis: a row expanded over the axes turns as the same row repeated."""
    gen = torch.Generator().manual_seed(5)
    q, k, v = make_rows(gen, 40, 8, 128), make_rows(gen, 40, 2, 128), make_rows(gen, 40, 2, 128)
    table, at = turns(gen, 60, 128), torch.randint(0, 60, (1, 40), generator=gen, dtype=torch.int32)
    rotary = Rotary(table.cuda(), [24, 24, 16], interleaved)
    batch = PagedBatch(ints(2, 0, 1)[None], ints(0, 40), ints(45), total_rows=40, max_rows=40, max_kv=48)
    made = []
    for places in (at.cuda().expand(3, 40), at.expand(3, 40).contiguous().cuda()):
        cache = PagedCache(3, 16, 2, 128)
        made.append((cache.write_rotated(q.cuda(), k.cuda(), v.cuda(), batch, rotary, places), cache.k, cache.v))
    assert all(same_bits(a, b) for a, b in zip(*made))
    want, size = cref.turned(q, None, 0.0, table, at.expand(3, 40), [24, 24, 16], interleaved)
    assert ((made[0][0].double().cpu() - want).abs() <= 2.0 ** -8 * want.abs() + 2.0 ** -16 * size).all()


@pytest.mark.parametrize("fmt,dim,rows", [("bf16", 128, 3), ("bf16", 80, 70), ("u8", 128, 70), ("u4", 64, 3)])
def test_queries_and_results_inside_wider_tensors(fmt, dim, rows):
    """q a slice of a projection's rows, out one of another tensor's, heads first in one of them: the bits of contiguous ones, and
    nothing beside them is touched."""
    gen = torch.Generator().manual_seed(dim + rows)
    s = Setup(gen, fmt, 2, dim, 16, [700, 90], [rows, 1])
    made = PageBounds(s.cache)
    whole = PagedBatch(s.batch.table, ints(0, 700, 790), s.batch.kv_len, total_rows=790, max_rows=700, max_kv=700)
    made.update(s.cache, whole)
    q = make_rows(gen, s.total, 8, dim).cuda()
    wide = torch.full((s.total + 2, 14, dim), math.nan, dtype=torch.bfloat16, device="cuda")
    wide[:s.total, 3:11] = q
    inside = wide[:, 3:11]
    heads_first = torch.full((11, s.total, dim), 7.0, dtype=torch.bfloat16, device="cuda")
    lists = made.choose(q, s.batch, 9)
    assert torch.equal(made.choose(inside, s.batch, 9), lists)
    want = s.cache.attend_chosen(q, s.batch, lists)
    out = heads_first[1:9].transpose(0, 1)
    assert s.cache.attend_chosen(inside, s.batch, lists, out=out) is out
    assert same_bits(out, want) and (heads_first[0] == 7.0).all() and (heads_first[9:] == 7.0).all()
    chosen = random_lists(gen, s, 44).cuda()  # over 512 keys
    assert same_bits(s.cache.attend_chosen(inside, s.batch, chosen, out=out), s.cache.attend_chosen(q, s.batch, chosen))
    assert torch.isnan(wide[:, :3]).all() and torch.isnan(wide[:, 11:]).all()


def test_rotated_rows_into_one_page_per_sequence():
    """Without a table: what the same rows give through pages of 16."""
    gen = torch.Generator().manual_seed(9)
    q, k, v = make_rows(gen, 90, 4, 64).cuda(), make_rows(gen, 90, 2, 64).cuda(), make_rows(gen, 90, 2, 64).cuda()
    rotary, at = Rotary(turns(gen, 200, 64).cuda()), torch.randint(0, 200, (90,), generator=gen, dtype=torch.int32).cuda()
    made = []
    for cache, table in ((PagedCache(2, 333, 2, 64), None), (PagedCache(10, 16, 2, 64), ints(*range(9, -1, -1)).view(2, 5))):
        batch = PagedBatch(table, ints(0, 50, 90), ints(70, 40), total_rows=90, max_rows=50, max_kv=70)
        made.append((cache.write_rotated(q, k, v, batch, rotary, at), *cache.read(batch)))
    assert all(same_bits(a, b) for a, b in zip(*made))


FIRST_USES = """
import time
import torch
from paper_2506_15745_gb300 import ipv
from paper_2506_15745_gb300.paged import PagedBatch, PagedCache
ints = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
cache = PagedCache(4, 64, 2, 128)
batch = PagedBatch(ints(0, 1, 2, 3)[None], ints(0, 1), ints(200), total_rows=1, max_rows=1, max_kv=256)
args = ipv.AttendArgs(n_q_heads=8, scale=1.0, causal=1)
torch.cuda.synchronize()
at = [time.perf_counter()]
ipv.attend_workspace(cache.ref, batch.ref, args)
at.append(time.perf_counter())
ipv.attend_chosen_workspace(cache.ref, batch.ref, args, ipv.Chosen(n_chosen=2))
at.append(time.perf_counter())
print(at[1] - at[0], at[2] - at[1])
"""


def test_a_first_call_sets_its_own_kernels_up():
    """In a process of its own: the first use of attend does not wait for the kernels of chosen pages (2.7 ms with all, 1.7 alone;
    theirs 1.3), so that these cost something when they are first used; were they there already it would be under a hundredth."""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    said = subprocess.run([sys.executable, "-c", FIRST_USES], cwd=root, capture_output=True, text=True, timeout=300, check=True).stdout
    dense, chosen = map(float, said.split()[-2:])
    assert chosen > 0.1 * dense, (dense, chosen)
