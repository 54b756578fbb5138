"""Rotated writes, bounds of pages, chosen pages, copies and gathers refuse bad arguments on the host, before a GPU is
touched; the float64 definitions that the GPU tests use hold on worked cases."""
import ctypes
import math
import os

import pytest

torch = pytest.importorskip("torch")

import chosen_ref as cref  # noqa: E402
from paper_2506_15745_gb300 import build as ipv_build  # noqa: E402
from paper_2506_15745_gb300 import ipv  # noqa: E402
from test_paged_abi import ARGS, BAD_ARGS, BAD_BATCH, BAD_PAGES, BATCH, PAGES  # noqa: E402

BAD, OK = ipv.IPV_EINVAL, ipv.IPV_OK
ROTARY = dict(table=0xA0000, n_positions=100, rot_dim=128, interleaved=0, n_axes=3, sections=(32, 16, 16, 0))
ROTATE = dict(q=0x50000, q_out=0x60000, k_new=0x70000, v_new=0x80000, q_row_stride=3584, q_head_stride=128, out_row_stride=3584,
              out_head_stride=128, row_stride=512, head_stride=128, n_q_heads=28, eps=1e-6, q_weight=0x90000, k_weight=0x91000,
              positions=0x92000, positions_stride=5)
BOUNDS = dict(n_kv_heads=4, head_dim=128, page_size=64, n_pages=10, codes=0xA0000, steps=0xB0000)
CHOOSE = dict(q=0x50000, q_row_stride=3584, q_head_stride=128, n_q_heads=28, n_chosen=3, first=1, recent=2, out=0xC0000,
              out_row_stride=12, out_head_stride=3)
CHOSEN = dict(pages=0xD0000, n_chosen=3, row_stride=12, head_stride=3)


@pytest.fixture(scope="module")
def lib():
    ipv_build.build()
    return ipv.load()


def by(cls, base, **change):
    values = {**base, **change}
    if "sections" in values:
        values["sections"] = (ctypes.c_int * 4)(*values["sections"])
    return ctypes.byref(cls(**values))


def rotated(lib, pages=(), batch=(), rotary=(), args=()):
    return lib.ipv_pages_write_rotated(by(ipv.PagesDesc, PAGES, **dict(pages)), by(ipv.Batch, BATCH, **dict(batch)),
                                       by(ipv.RotaryDesc, ROTARY, **dict(rotary)), by(ipv.RotateArgs, ROTATE, **dict(args)), None)


def update(lib, bounds=(), pages=(), batch=()):
    return lib.ipv_bounds_update(by(ipv.BoundsDesc, BOUNDS, **dict(bounds)), by(ipv.PagesDesc, PAGES, **dict(pages)),
                                 by(ipv.Batch, BATCH, **dict(batch)), None)


def choose(lib, bounds=(), batch=(), args=()):
    return lib.ipv_bounds_choose(by(ipv.BoundsDesc, BOUNDS, **dict(bounds)), by(ipv.Batch, BATCH, **dict(batch)),
                                 by(ipv.ChooseArgs, CHOOSE, **dict(args)), None)


def attend(lib, pages=(), batch=(), args=(), chosen=()):
    return lib.ipv_attend_chosen(by(ipv.PagesDesc, PAGES, **dict(pages)), by(ipv.Batch, BATCH, **dict(batch)),
                                 by(ipv.AttendArgs, ARGS, **dict(args)), by(ipv.Chosen, CHOSEN, **dict(chosen)), None)


def workspace(lib, pages=(), batch=(), args=(), chosen=()):
    n = ctypes.c_int64(7)
    return lib.ipv_attend_chosen_workspace(by(ipv.PagesDesc, PAGES, **dict(pages)), by(ipv.Batch, BATCH, **dict(batch)),
                                           by(ipv.AttendArgs, ARGS, **dict(args)), by(ipv.Chosen, CHOSEN, **dict(chosen)),
                                           ctypes.byref(n)), n.value


def gather(lib, source=(), source_batch=(), pages=(), batch=(), kept=(0xE0000, 12, 3)):
    return lib.ipv_pages_gather(by(ipv.PagesDesc, PAGES, **dict(source)), by(ipv.Batch, BATCH, **dict(source_batch)),
                                by(ipv.PagesDesc, PAGES, **dict(pages)), by(ipv.Batch, BATCH, **dict(batch)), *kept, None)


def copy(lib, pages=(), lists=(0xE0000, 0xF0000), n=2):
    return lib.ipv_pages_copy(by(ipv.PagesDesc, PAGES, **dict(pages)), *lists, n, None)


@pytest.mark.parametrize("bad", BAD_PAGES + BAD_BATCH, ids=str)
def test_bad_pages_and_batches(lib, bad):
    pages = {k: v for k, v in bad.items() if k in PAGES}
    batch = {k: v for k, v in bad.items() if k in BATCH}
    assert rotated(lib, pages, batch) == BAD
    assert update(lib, {}, pages, batch) == BAD
    assert attend(lib, pages, batch) == BAD and workspace(lib, pages, batch) == (BAD, 0)
    assert gather(lib, pages, batch) == BAD and gather(lib, (), (), pages, batch) == BAD
    if batch:
        assert choose(lib, batch=batch) == BAD
    elif bad not in (dict(page_size=48), dict(page_size=8)):  # fit for one page per sequence, which a copy does not know
        assert copy(lib, pages) == BAD
    assert lib.ipv_last_error().startswith(b"IPV_EINVAL")


@pytest.mark.parametrize("bad", [dict(rot_dim=0), dict(rot_dim=24), dict(rot_dim=144), dict(rot_dim=64), dict(n_positions=0),
                                 dict(n_positions=1 << 31), dict(interleaved=2), dict(interleaved=-1), dict(n_axes=0), dict(n_axes=5),
                                 dict(n_axes=2), dict(sections=(32, 32, 0, 0)), dict(sections=(36, 12, 16, 0)),
                                 dict(sections=(72, -8, 0, 0)), dict(sections=(1 << 30, 1 << 30, 64, 0)), dict(table=None), dict(table=0xA0008)], ids=str)
def test_bad_rotaries(lib, bad):
    assert rotated(lib, rotary=bad) == BAD


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=0x50008), dict(q_out=None), dict(q_out=0x60002), dict(k_new=None), dict(v_new=None),
                                 dict(v_new=0x80004), dict(q_row_stride=3580), dict(q_head_stride=-128), dict(out_row_stride=4), dict(row_stride=516),
                                 dict(head_stride=-8), dict(n_q_heads=0), dict(n_q_heads=65536), dict(eps=math.nan), dict(eps=math.inf),
                                 dict(eps=-1e-6), dict(q_weight=0x90008), dict(k_weight=0x91002), dict(positions=None),
                                 dict(positions=0x92002), dict(positions_stride=4), dict(positions_stride=-5),
                                 dict(q_out=0x50000, out_row_stride=7168)], ids=str)
def test_bad_rotated_writes(lib, bad):
    assert rotated(lib, args=bad) == BAD


@pytest.mark.parametrize("bad", [dict(n_kv_heads=0), dict(n_kv_heads=65536), dict(n_kv_heads=3), dict(head_dim=0), dict(head_dim=136), dict(head_dim=100),
                                 dict(head_dim=64), dict(page_size=0), dict(page_size=32), dict(n_pages=0), dict(n_pages=1 << 31), dict(n_pages=9),
                                 dict(codes=None), dict(codes=0xA0008), dict(steps=None), dict(steps=0xB0002)], ids=str)
def test_bad_bounds(lib, bad):
    assert update(lib, bad) == BAD
    if not (bad in (dict(head_dim=64), dict(page_size=32), dict(n_pages=9))):  # bounds of other pages: choose sees no pages
        assert choose(lib, bad) == BAD


@pytest.mark.parametrize("bad", [dict(q=None), dict(q=0x50008), dict(q_row_stride=3580), dict(q_head_stride=-128), dict(n_q_heads=0), dict(n_q_heads=27),
                                 dict(n_q_heads=4 * 65), dict(n_chosen=0), dict(n_chosen=2), dict(first=-1), dict(first=2), dict(recent=0), dict(recent=3),
                                 dict(first=1 << 30, recent=(1 << 30) + 1, n_chosen=(1 << 31) - 1, out_row_stride=-1), dict(out=None),
                                 dict(out=0xC0002), dict(out_row_stride=-1), dict(out_head_stride=-1)], ids=str)
def test_bad_choices(lib, bad):
    assert choose(lib, args=bad) == BAD


def test_choices_over_too_many_pages(lib):
    wide = dict(max_pages=32769, table_stride=32769)
    assert choose(lib, batch=dict(**wide, max_kv=64 * 32768 + 1)) == BAD
    assert b"32768" in lib.ipv_last_error()


@pytest.mark.parametrize("bad", BAD_ARGS + [dict(causal=0), dict(window=5), dict(window=5, sinks=2), dict(sinks=1)], ids=str)
def test_bad_attention(lib, bad):
    assert attend(lib, args=bad) == BAD


@pytest.mark.parametrize("bad", [dict(pages=None), dict(pages=0xD0002), dict(n_chosen=0), dict(n_chosen=-3), dict(row_stride=-1), dict(head_stride=-1)], ids=str)
def test_bad_lists(lib, bad):
    assert attend(lib, chosen=bad) == BAD


def test_attention_over_too_long_a_cache(lib):
    pages = dict(page_size=1 << 30, page_stride=1, head_stride=1)
    assert attend(lib, pages, dict(max_pages=4, max_kv=(1 << 30) + 1)) == BAD
    assert b"2^30" in lib.ipv_last_error()


def test_bad_copies(lib):
    for lists in ((None, 0xF0000), (0xE0000, None), (0xE0002, 0xF0000), (0xE0000, 0xF0001), (0xE0000, 0xE0000)):
        assert copy(lib, lists=lists) == BAD
    assert copy(lib, n=-1) == BAD and copy(lib, n=1 << 40) == BAD
    assert copy(lib, dict(page_size=1 << 30, n_kv_heads=2, page_stride=1, head_stride=1)) == BAD  # more pieces than a page may have
    assert copy(lib, lists=(None, None), n=0) == OK


def test_bad_gathers(lib):
    for pages in (dict(format=1), dict(n_kv_heads=3), dict(head_dim=64)):
        assert gather(lib, pages) == BAD and gather(lib, (), (), pages) == BAD
    for kept in ((0xE0002, 12, 3), (0xE0000, -1, 3), (0xE0000, 12, -1)):
        assert gather(lib, kept=kept) == BAD
    assert gather(lib, source_batch=dict(n_seqs=1)) == BAD


def test_null_structures(lib):
    p, b, r = by(ipv.PagesDesc, PAGES), by(ipv.Batch, BATCH), by(ipv.RotaryDesc, ROTARY)
    w, s, c = by(ipv.RotateArgs, ROTATE), by(ipv.BoundsDesc, BOUNDS), by(ipv.ChooseArgs, CHOOSE)
    t, x = by(ipv.AttendArgs, ARGS), by(ipv.Chosen, CHOSEN)
    for call, args in ((lib.ipv_pages_write_rotated, (p, b, r, w)), (lib.ipv_bounds_update, (s, p, b)), (lib.ipv_bounds_choose, (s, b, c)),
                       (lib.ipv_attend_chosen, (p, b, t, x))):
        for i in range(len(args)):
            assert call(*args[:i], None, *args[i + 1:], None) == BAD
    for i in range(4):
        args = [p, b, p, b]
        args[i] = None
        assert lib.ipv_pages_gather(*args, None, 0, 0, None) == BAD
    assert lib.ipv_pages_copy(None, 0xE0000, 0xF0000, 2, None) == BAD
    n = ctypes.c_int64(0)
    assert lib.ipv_attend_chosen_workspace(p, b, t, None, ctypes.byref(n)) == BAD
    assert lib.ipv_attend_chosen_workspace(p, b, t, x, None) == BAD


def test_nothing_to_do(lib):
    for empty in (dict(n_seqs=0, row_start=None, kv_len=None), dict(max_rows=0), dict(total_rows=0)):
        assert rotated(lib, batch=empty) == OK and update(lib, batch=empty) == OK
        assert choose(lib, batch=empty) == OK and attend(lib, batch=empty) == OK
        assert workspace(lib, batch=empty) == (OK, 0)
        if "n_seqs" in empty:
            assert gather(lib, source_batch=empty, batch=empty) == OK
        else:
            assert gather(lib, batch=empty) == OK
    assert update(lib, batch=dict(max_kv=0)) == OK


def test_overlapping_kernels_read_coherently():
    """As the paged cache's other kernels: launched while a predecessor may still write what they are to read."""
    for name in ("rotate.cu", "bounds.cu", "move.cu", "attend_chosen.cu", "attend_rows.cuh", "paged_codes.cuh"):
        with open(os.path.join(ipv_build.CSRC, name)) as f:
            text = f.read()
        for banned in ("ld_stream(", "ld.global.nc", "__ldg("):
            assert banned not in text, (name, banned)


# ------------------------------------------------ the definitions, on worked cases
def test_turned_worked_case():
    """A quarter turn of frequency 0, none of the others; the norm of (3, 4, 0, ..)."""
    x = torch.zeros(1, 1, 32)
    x[0, 0, 0], x[0, 0, 1] = 3.0, 4.0
    table = torch.cat([torch.ones(2, 8), torch.zeros(2, 8)], 1)
    table[1, 0], table[1, 8] = 0.0, 1.0
    y, _ = cref.turned(x, None, 0.0, table, torch.tensor([[1]]), [8], True)
    assert y[0, 0, :2].tolist() == [-4.0, 3.0]
    y, _ = cref.turned(x, None, 0.0, table, torch.tensor([[1]]), [8], False)
    assert y[0, 0, [0, 8, 1]].tolist() == [0.0, 3.0, 4.0]
    w = torch.full((32,), 2.0)
    y, _ = cref.turned(x, w, 0.0, table, torch.tensor([[0]]), [8], False)
    assert torch.allclose(y[0, 0, :2], torch.tensor([6.0, 8.0]).double() / math.sqrt(25 / 32))
    assert torch.isnan(cref.turned(x, None, 0.0, table, torch.tensor([[2]]), [8], False)[0][0, 0, :16]).all()


def test_bounds_worked_cases():
    lo, hi, step = cref.bounds(torch.tensor([[1.0, -3.0], [2.0, 0.0]]))
    assert step == 2.0 ** -5 and lo.tolist() == [32, -96] and hi.tolist() == [64, 0]
    assert cref.exponent(127.0) == 0 and cref.exponent(127.5) == 1 and cref.exponent(63.5) == -1 and cref.exponent(0.0) == -40
    assert math.isnan(cref.bounds(torch.tensor([[math.inf]]))[2])


def test_choice_worked_cases():
    lo, hi = torch.tensor([[-1, 0], [0, 2], [0, 2], [5, 5]]), torch.tensor([[1, 1], [3, 4], [3, 4], [6, 6]])
    s = cref.scores(torch.tensor([[127.0, -127.0]]), lo, hi, torch.tensor([1.0, 1.0, 1.0, math.nan]).double())
    assert s[:3].tolist() == [127.0, 127.0, 127.0] and math.isnan(s[3])
    assert cref.choose(s, 2, 0, 1) == [0, 3] and cref.choose(s, 3, 0, 1) == [0, 1, 3] and cref.choose(s, 5, 1, 1) == [0, 1, 2, 3, -1]
    assert cref.choose(torch.tensor([1.0, math.nan, -math.inf, 0.0]), 2, 0, 1) == [0, 3]
    assert cref.choose(torch.tensor([math.nan, math.nan, -5.0, 0.0]), 2, 0, 1) == [2, 3]


def test_attention_worked_case():
    q = torch.ones(1, 1, 8).double()
    k = torch.ones(3, 1, 8).double()
    v = torch.arange(3.0).double()[:, None, None].expand(3, 1, 8)
    for chosen, want in (([0, 1], 1.0), ([1, -1], 2.0), ([1, 1], 2.0), ([0, 0], 0.5), ([5, -1], 0.0), ([0, 7], 0.5)):
        out, lse, _, _ = cref.attend(q, k, v, torch.tensor([[chosen]]), 2, 0.5)
        assert torch.allclose(out, torch.full_like(out, want)), chosen
    assert lse[0, 0] == math.log(2) + 4.0
