"""The binding of rotated writes, page bounds, chosen pages, copies and gathers on the CPU: what it passes to the
library, and what it refuses before anything is passed. Tensors and streams are stand-ins, as in test_paged_binding.py."""
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2506_15745_gb300 import build as ipv_build  # noqa: E402
from paper_2506_15745_gb300 import ipv  # noqa: E402
from paper_2506_15745_gb300.paged import PageBounds, PagedBatch, PagedCache, Rotary  # noqa: E402
from test_paged_binding import SIDE, Handle, Streams, gpu, ints  # noqa: E402


@pytest.fixture(scope="module", autouse=True)
def built():
    ipv_build.build()


PAGES, BATCH = ipv.PagesDesc, ipv.Batch
STRUCTURES = {  # what a call's first arguments point to
    "ipv_pages_write_rotated": (PAGES, BATCH, ipv.RotaryDesc, ipv.RotateArgs), "ipv_bounds_update": (ipv.BoundsDesc, PAGES, BATCH),
    "ipv_bounds_choose": (ipv.BoundsDesc, BATCH, ipv.ChooseArgs), "ipv_attend_chosen": (PAGES, BATCH, ipv.AttendArgs, ipv.Chosen),
    "ipv_attend": (PAGES, BATCH, ipv.AttendArgs), "ipv_pages_copy": (PAGES,), "ipv_pages_gather": (PAGES, BATCH, PAGES, BATCH)}


class Library:
    """Notes what it is given; structures, by reference or address, as dicts."""

    def __init__(self, log):
        self.log = log

    def __getattr__(self, name):
        def call(*args):
            read = []
            for a, cls in zip(args, STRUCTURES[name]):
                x = a._obj if hasattr(a, "_obj") else cls.from_address(a)
                read.append({f: getattr(x, f) for f, _ in cls._fields_})
            self.log.append((name, *read, *args[len(read):]))
            return 0
        return call


@pytest.fixture
def world(monkeypatch):
    class World:
        log, need = [], 0

    w = World()
    w.streams = Streams(w.log, monkeypatch)
    monkeypatch.setattr(ipv, "attend_chosen_workspace", lambda *_: w.need)
    monkeypatch.setattr(torch.Tensor, "record_stream", lambda self, stream: w.log.append(("used on", self.data_ptr(), stream.cuda_stream)))
    rows = lambda *shape: gpu(torch.ones(shape, dtype=torch.bfloat16))  # noqa: E731
    w.rows = rows
    w.cache = PagedCache.from_tensors("bf16", rows(4, 2, 16, 64), rows(4, 2, 16, 64))
    w.bounds = PageBounds.from_tensors(gpu(torch.zeros(4, 2, 2, 64, dtype=torch.int8)), gpu(torch.zeros(4, 2)), 16, 64)
    w.cache._lib = w.bounds._lib = Library(w.log)
    w.batch = PagedBatch(ints(0, 1, 2, 3).view(1, 4), ints(0, 3), ints(50), total_rows=3, max_rows=3, max_kv=64)
    w.q, w.k, w.v = rows(3, 4, 64), rows(3, 2, 64), rows(3, 2, 64)
    w.rotary = Rotary(gpu(torch.zeros(100, 64)), [16, 8, 8])
    w.at = gpu(torch.zeros(3, 3, dtype=torch.int32))
    w.chosen = gpu(torch.zeros(3, 2, 3, dtype=torch.int32))
    return w


def cpu(t):
    return t.as_subclass(torch.Tensor)


def test_what_a_rotated_write_passes(world):
    w = world
    wide = w.rows(3, 8, 64)
    positions = gpu(torch.zeros(3, 9, dtype=torch.int32))
    weight = w.rows(64)
    out = w.cache.write_rotated(wide[:, 2:6], w.k, w.v, w.batch, w.rotary, positions[:, 2:5], q_weight=weight, eps=0.5, stream=SIDE)
    name, pages, batch, rotary, args, stream = w.log[-1]
    assert name == "ipv_pages_write_rotated" and stream == SIDE
    assert args["q"] == wide.data_ptr() + 2 * 128 and args["q_row_stride"] == 512 and args["q_head_stride"] == 64 and args["n_q_heads"] == 4
    assert args["q_out"] == out.data_ptr() and args["out_row_stride"] == 256 and out.shape == (3, 4, 64)
    assert (args["k_new"], args["v_new"], args["row_stride"], args["head_stride"]) == (w.k.data_ptr(), w.v.data_ptr(), 128, 64)
    assert (args["q_weight"], args["k_weight"], args["eps"]) == (weight.data_ptr(), None, 0.5)
    longer = [w.rows(5, 4, 64), w.rows(5, 2, 64), w.rows(5, 2, 64)]  # packed tensors may be longer than the batch
    w.cache.write_rotated(*longer, w.batch, w.rotary, positions, q_out=w.rows(9, 4, 64))
    assert w.log[-1][4]["q"] == longer[0].data_ptr() and w.log[-1][4]["eps"] == ctypes.c_float(1e-6).value
    assert args["positions"] == positions.data_ptr() + 8 and args["positions_stride"] == 9
    assert list(rotary["sections"])[:3] == [16, 8, 8] and rotary["n_axes"] == 3 and rotary["n_positions"] == 100 and rotary["rot_dim"] == 64
    assert ("used on", out.data_ptr(), 0) in w.log  # made on the call's stream
    other = Rotary(gpu(torch.zeros(9, 32)), interleaved=True)
    w.cache.write_rotated(w.q, w.k, w.v, w.batch, other, w.at[0], q_out=w.q)
    _, _, _, rotary, args, stream = w.log[-1]
    assert stream == 0 and args["q_out"] == args["q"] == w.q.data_ptr() and args["q_weight"] is None
    assert list(rotary["sections"])[:1] == [16] and rotary["interleaved"] == 1 and rotary["n_axes"] == 1


def test_rotated_writes_that_are_refused(world):
    w = world
    good = dict(q=w.q, k_new=w.k, v_new=w.v, batch=w.batch, rotary=w.rotary, positions=w.at)
    for bad, what in ((dict(q=cpu(w.q)), "q must"), (dict(q=w.q.float()), "q must"), (dict(q=w.q[0]), "q must"), (dict(q=w.q[:2]), "q must"),
                      (dict(q=w.rows(3, 64, 4).transpose(1, 2)), "q must"), (dict(q_out=w.rows(3, 2, 64)), "q_out"), (dict(q_out=cpu(w.q)), "q_out"),
                      (dict(k_new=w.rows(3, 3, 64)), "k_new"), (dict(v_new=w.rows(3, 2, 32)), "v_new"), (dict(v_new=cpu(w.v)), "v_new"),
                      (dict(v_new=w.rows(3, 4, 64)[:, ::2]), "strides"),
                      (dict(positions=w.at.long()), "positions"), (dict(positions=cpu(w.at)), "positions"), (dict(positions=w.at[:2]), "positions"),
                      (dict(positions=w.at[0]), "positions"), (dict(positions=w.at[:, :2]), "positions"),
                      (dict(positions=gpu(torch.zeros(3, 6, dtype=torch.int32))[:, ::2]), "positions"),
                      (dict(q_weight=w.rows(32)), "q_weight"), (dict(k_weight=w.rows(64).float()), "k_weight"),
                      (dict(k_weight=cpu(w.rows(64))), "k_weight"), (dict(q_weight=w.rows(128)[::2]), "q_weight")):
        with pytest.raises(ValueError, match=what):
            w.cache.write_rotated(**{**good, **bad})
    assert not any(e[0].startswith("ipv_") for e in w.log)


def test_rotaries_that_are_refused():
    table = gpu(torch.zeros(10, 64))
    for bad in (cpu(table), table.double(), table[0], table.t(), table[:, ::2]):
        with pytest.raises(ValueError, match="table"):
            Rotary(bad)
    for sections in ([], [8, 8, 8, 4, 4]):
        with pytest.raises(ValueError, match="axes"):
            Rotary(table, sections)
    with pytest.raises(ValueError, match="section"):
        Rotary(table, [(1 << 32) + 16, 16])


def test_what_bounds_pass(world):
    w = world
    w.bounds.update(w.cache, w.batch, stream=Handle(SIDE))
    name, bounds, pages, batch, stream = w.log[-1]
    assert name == "ipv_bounds_update" and stream == SIDE
    assert bounds == dict(n_kv_heads=2, head_dim=64, page_size=16, n_pages=4, codes=w.bounds.codes.data_ptr(), steps=w.bounds.steps.data_ptr())
    out = w.bounds.choose(w.q, w.batch, 3, first=0, recent=2, stream=SIDE)
    name, _, _, args, stream = w.log[-1]
    assert name == "ipv_bounds_choose" and stream == SIDE
    assert out.dtype is torch.int32 and out.shape == (3, 2, 3) and (out == -1).all() and ("used on", out.data_ptr(), 0) in w.log
    assert args == dict(q=w.q.data_ptr(), q_row_stride=256, q_head_stride=64, n_q_heads=4, n_chosen=3, first=0, recent=2, out=out.data_ptr(),
                        out_row_stride=6, out_head_stride=3)
    lists = gpu(torch.zeros(2, 3, 8, dtype=torch.int32)).transpose(0, 1)
    assert w.bounds.choose(w.q, w.batch, 5, out=lists[..., 1:6]) is not None
    args = w.log[-1][3]
    assert args["out"] == lists.data_ptr() + 4 and args["out_row_stride"] == 8 and args["out_head_stride"] == 24


def test_bounds_and_choices_that_are_refused(world):
    w = world
    codes, steps = w.bounds.codes, w.bounds.steps
    for bad in (cpu(codes), codes.to(torch.uint8), codes[:, :, :1], codes[0], codes[:, ::2], gpu(torch.zeros(4, 2, 2, 128, dtype=torch.int8))):
        with pytest.raises(ValueError, match="codes"):
            PageBounds.from_tensors(bad, steps, 16, 64)
    for bad in (cpu(steps), steps.half(), steps[:3], gpu(torch.zeros(2, 4)).t()):
        with pytest.raises(ValueError, match="steps"):
            PageBounds.from_tensors(codes, bad, 16, 64)
    with pytest.raises(ValueError, match="page_size"):
        PageBounds.from_tensors(codes, steps, (1 << 32) + 16, 64)
    for bad in (dict(q=cpu(w.q)), dict(q=w.q.float()), dict(q=w.q[:2]), dict(q=w.q[0]), dict(n_chosen=0), dict(n_chosen=(1 << 32) + 3),
                dict(first=1 << 32), dict(recent=(1 << 32) + 1), dict(out=w.chosen[..., :2]), dict(out=w.chosen.long()), dict(out=cpu(w.chosen)),
                dict(out=w.chosen[:2]), dict(out=w.chosen[:, :1]), dict(out=gpu(torch.zeros(3, 2, 6, dtype=torch.int32))[..., ::2])):
        with pytest.raises(ValueError):
            w.bounds.choose(**{**dict(q=w.q, batch=w.batch, n_chosen=3), **bad})
    assert not any(e[0].startswith("ipv_") for e in w.log)


def test_what_chosen_attention_passes(world):
    w = world
    lse = gpu(torch.zeros(3, 4))
    out = w.cache.attend_chosen(w.q, w.batch, w.chosen, lse=lse, scale=0.25, stream=SIDE)
    name, _, _, args, lists, stream = w.log[-1]
    assert name == "ipv_attend_chosen" and stream == SIDE and ("used on", out.data_ptr(), 0) in w.log
    assert lists == dict(pages=w.chosen.data_ptr(), n_chosen=3, row_stride=6, head_stride=3)
    assert (args["q"], args["out"], args["lse"], args["scale"], args["causal"]) == (w.q.data_ptr(), out.data_ptr(), lse.data_ptr(), 0.25, 1)
    w.cache.attend_chosen(w.q, w.batch, w.chosen[:, :, :2])
    args, lists = w.log[-1][3:5]
    assert lists["n_chosen"] == 2 and lists["row_stride"] == 6 and args["lse"] is None and args["scale"] == 0.125
    w.cache.attend_chosen(w.q, w.batch, w.chosen[:, :1].expand(3, 2, 3))  # one list for all heads
    assert w.log[-1][4]["head_stride"] == 0


def test_chosen_attention_that_is_refused(world):
    w = world
    for bad in (dict(q=cpu(w.q)), dict(q=w.q.float()), dict(q=w.q[:2]), dict(chosen=cpu(w.chosen)), dict(chosen=w.chosen.long()),
                dict(chosen=w.chosen[:2]), dict(chosen=w.chosen[:, :1]), dict(chosen=w.chosen[0]), dict(out=w.rows(3, 2, 64)), dict(out=cpu(w.q)),
                dict(lse=gpu(torch.zeros(3, 4, dtype=torch.float64))), dict(lse=gpu(torch.zeros(4, 3)).t()), dict(lse=torch.zeros(3, 4)),
                dict(chosen=gpu(torch.zeros(3, 2, 6, dtype=torch.int32))[..., ::2])):
        with pytest.raises(ValueError):
            w.cache.attend_chosen(**{**dict(q=w.q, batch=w.batch, chosen=w.chosen), **bad})
    w.need = 4096
    with pytest.raises(ValueError, match="workspace"):
        w.cache.attend_chosen(w.q, w.batch, w.chosen[..., :1], stream=SIDE)  # a stream that is not the current one
    assert not any(e[0].startswith("ipv_") for e in w.log)


def test_calls_of_both_attentions_do_not_share_arguments(world, monkeypatch):
    """The same sizes, with and without lists."""
    w = world
    monkeypatch.setattr(ipv, "attend_workspace", lambda *_: 0)
    for _ in range(2):
        w.cache.attend(w.q, w.batch, window=3)
        assert w.log[-1][0] == "ipv_attend" and w.log[-1][3]["window"] == 3
        w.cache.attend_chosen(w.q, w.batch, w.chosen)
        assert w.log[-1][0] == "ipv_attend_chosen" and w.log[-1][3]["window"] == 0
        w.cache.attend(w.q, w.batch)
        assert w.log[-1][3]["window"] == 0


def test_what_copies_and_gathers_pass(world):
    w = world
    w.cache.copy_pages(ints(1, 2), ints(0, 3), stream=SIDE)
    name, _, _, _, n, stream = w.log[-1]
    assert name == "ipv_pages_copy" and n == 2 and stream == SIDE
    for bad in ((ints(1), ints(0, 3)), (ints(1, 2).long(), ints(0, 3)), (ints(1, 2), cpu(ints(0, 3))), (ints(1, 2).view(1, 2), ints(0, 3).view(1, 2)),
                (ints(1, 0, 2, 0)[::2], ints(0, 3))):
        with pytest.raises(ValueError):
            w.cache.copy_pages(*bad)
    other = PagedCache.from_tensors("bf16", w.rows(6, 2, 16, 64), w.rows(6, 2, 16, 64))
    held = PagedBatch(ints(0, 1, 2).view(1, 3), ints(0, 0), ints(40), total_rows=0, max_rows=0, max_kv=48)
    kept = gpu(torch.zeros(1, 2, 5, dtype=torch.int32))
    w.cache.gather(other, held, w.batch, kept[..., 1:])
    name, pages, batch, to, to_batch, at, seq, head, stream = w.log[-1]
    assert name == "ipv_pages_gather" and pages["n_pages"] == 6 and to["n_pages"] == 4 and batch["total_rows"] == 0 and to_batch["total_rows"] == 3
    assert (at, seq, head, stream) == (kept.data_ptr() + 4, 10, 5, 0)
    w.cache.gather(other, held, w.batch, kept[:, :1].expand(1, 2, 5))  # one list for all heads
    assert w.log[-1][6:8] == (10, 0) or w.log[-1][7] == 0
    w.cache.gather(other, held, w.batch)
    assert w.log[-1][5:8] == (None, 0, 0)
    n = len(w.log)
    for bad in (kept.long(), cpu(kept), kept[:, :1], kept[..., :2], kept[0], gpu(torch.zeros(1, 2, 10, dtype=torch.int32))[..., ::2]):
        with pytest.raises(ValueError, match="kept"):
            w.cache.gather(other, held, w.batch, bad)
    assert len(w.log) == n
