"""The binding of the paged cache on the CPU: what it passes to the library, and
what it refuses before anything is passed.

The tensors live on the host and say that they are on the GPU; the library, the
streams and the capture state are stand-ins that record what they are given."""
import contextlib
import ctypes

import pytest

torch = pytest.importorskip("torch")

from paper_2506_15745_gb300 import build as ipv_build  # noqa: E402
from paper_2506_15745_gb300 import ipv  # noqa: E402
from paper_2506_15745_gb300 import paged  # noqa: E402
from paper_2506_15745_gb300.paged import PagedBatch, PagedCache  # noqa: E402


class OnGpu(torch.Tensor):
    is_cuda = property(lambda self: True)


def gpu(t):
    return t.as_subclass(OnGpu)


def ints(*x):
    return gpu(torch.tensor(x, dtype=torch.int32))


@pytest.fixture(scope="module", autouse=True)
def built():
    ipv_build.build()


# ------------------------------------------------------------------ page tables
def batch_of(table, n):
    return PagedBatch(table, ints(*range(n + 1)), ints(*[9] * n), total_rows=n, max_rows=1, max_kv=9)


def entries(batch):
    """What the kernels read: entry i of sequence b at table + b * table_stride + i, inside the tensor's storage."""
    s, t = batch.struct, batch.table
    end = t.untyped_storage().data_ptr() + t.untyped_storage().nbytes()
    out = []
    for b in range(s.n_seqs):
        at = s.table + 4 * b * s.table_stride
        assert at + 4 * s.max_pages <= end, f"sequence {b} reads behind the table"
        out.append(list((ctypes.c_int32 * s.max_pages).from_address(at)))
    return out


def test_a_table_that_all_sequences_share():
    table = ints(5, 3, 8).view(1, 3).expand(4, 3)
    assert entries(batch_of(table, 4)) == [[5, 3, 8]] * 4


def test_tables_that_are_slices():
    wide = gpu(torch.arange(40, dtype=torch.int32).view(4, 10))
    assert entries(batch_of(wide[:, 2:5], 4)) == [[2, 3, 4], [12, 13, 14], [22, 23, 24], [32, 33, 34]]
    assert entries(batch_of(wide[::2, :4], 2)) == [[0, 1, 2, 3], [20, 21, 22, 23]]
    assert entries(batch_of(wide[1:2, 7:], 1)) == [[17, 18, 19]]


def test_rows_of_a_table_that_overlap_are_refused():
    flat = gpu(torch.arange(16, dtype=torch.int32))
    with pytest.raises(ValueError, match="table"):
        batch_of(flat.as_strided((4, 3), (2, 1)), 4)


# ---------------------------------------------------------- the calls that launch
class Library:
    """Stands in for libipv.so: notes what it is given."""

    def __init__(self, log):
        self.log = log

    def ipv_pages_read(self, pages, batch, k, v, row, head, stream):
        self.log.append(("read", k, v, stream))
        return 0

    def ipv_attend(self, pages, batch, args, stream):
        a = args._obj
        self.log.append(("attend", a.out, a.workspace, a.workspace_bytes, stream))
        return 0


class Streams:
    """PyTorch's streams as numbers; fills are noted with the stream that is current."""

    def __init__(self, log, monkeypatch):
        self.log, self.at, self.capturing = log, 0, False
        monkeypatch.setattr(ipv, "_stream", lambda s: self.at if s is None else s if isinstance(s, int) else s.cuda_stream)
        monkeypatch.setattr(torch.cuda, "stream", self.enter)
        monkeypatch.setattr(torch.cuda, "ExternalStream", lambda handle, *_: Handle(handle))
        monkeypatch.setattr(torch.cuda, "current_stream", lambda *_: Handle(self.at))
        monkeypatch.setattr(torch.cuda, "is_current_stream_capturing", lambda: self.capturing)

    @contextlib.contextmanager
    def enter(self, stream):
        before, self.at = self.at, stream.cuda_stream
        yield
        self.at = before


class Handle:
    def __init__(self, cuda_stream):
        self.cuda_stream = cuda_stream


NEED = 4096


@pytest.fixture
def world(monkeypatch):
    """(cache, batch, q, log, streams); attention needs NEED bytes of workspace until `world.need` says otherwise."""
    log = []

    class World:
        need = NEED

    class Traced(OnGpu):
        @classmethod
        def __torch_function__(cls, func, types, args=(), kwargs=None):
            out = super().__torch_function__(func, types, args, kwargs or {})
            if func.__name__ in ("zeros_like", "new_zeros", "zero_", "fill_"):
                log.append(("fill", out.data_ptr(), World.streams.at))
            return out

        def record_stream(self, stream):
            log.append(("used on", self.data_ptr(), stream.cuda_stream))

    empty = torch.empty
    monkeypatch.setattr(paged.torch, "empty", lambda *a, **k: empty(*a, **{**k, "device": "cpu"}).as_subclass(Traced))
    World.streams = Streams(log, monkeypatch)
    monkeypatch.setattr(ipv, "attend_workspace", lambda *_: World.need)
    World.tensor = staticmethod(lambda *shape: torch.ones(shape, dtype=torch.bfloat16).as_subclass(Traced))
    World.cache = PagedCache.from_tensors("bf16", World.tensor(4, 2, 16, 64), World.tensor(4, 2, 16, 64))
    World.cache._lib = Library(log)
    World.batch = PagedBatch(ints(0, 1, 2, 3).view(1, 4), ints(0, 3), ints(50), total_rows=3, max_rows=3, max_kv=64)
    World.q, World.log = World.tensor(3, 4, 64), log
    return World


def aligned(n):
    t = torch.zeros(n + 256, dtype=torch.uint8)
    at = -t.data_ptr() % 256
    return t[at:at + n]


def test_a_workspace_is_gpu_memory_that_is_really_there(world):
    w = gpu(aligned(2 * NEED))
    world.cache.attend(world.q, world.batch, workspace=w)
    assert world.log[-1][2:4] == (w.data_ptr(), 2 * NEED)
    for bad in (aligned(NEED),                                      # host memory
                gpu(aligned(1)).expand(NEED),                       # one byte that says it is many
                gpu(aligned(2 * NEED))[::2]):
        n = len(world.log)
        with pytest.raises(ValueError, match="workspace"):
            world.cache.attend(world.q, world.batch, workspace=bad)
        assert not any(e[0] == "attend" for e in world.log[n:])


SIDE = 0x5000


def test_results_are_made_on_the_stream_that_writes_them(world):
    """Named streams: the fill of new results precedes the kernel on its stream, and their memory is not handed on
    while the current stream may still use them."""
    world.need = 0
    for call in (lambda: [world.cache.attend(world.q, world.batch, stream=SIDE)],
                 lambda: world.cache.read(world.batch, stream=SIDE),
                 lambda: world.cache.read(world.batch, stream=Handle(SIDE))):
        del world.log[:]
        made = {t.data_ptr() for t in call()}
        assert made == {e[1] for e in world.log if e[0] == "fill"}
        assert all(e[2] == SIDE for e in world.log if e[0] == "fill"), world.log
        assert made == {e[1] for e in world.log if e[0] == "used on" and e[2] == 0}
        assert world.log[-1][0] in ("attend", "read") and world.log[-1][-1] == SIDE
        assert world.streams.at == 0


def test_results_on_the_current_stream(world):
    out = world.cache.attend(world.q, world.batch, stream=0)
    k, v = world.cache.read(world.batch)
    assert [e for e in world.log if e[0] == "fill"] == [("fill", t.data_ptr(), 0) for t in (out, k, v)]
    assert not any(e[0] == "used on" for e in world.log)


def last(log, kind):
    return next(e for e in reversed(log) if e[0] == kind)


def test_a_captured_call_does_not_use_the_kept_workspace(world):
    """A graph's workspace is the graph's: it is not the one that later calls on the stream use, replace and free."""
    attend = lambda: (world.cache.attend(world.q, world.batch), last(world.log, "attend")[2])[1]  # noqa: E731
    kept = attend()
    assert attend() == kept and list(world.cache._workspaces) == [0]
    held = world.cache._workspaces[0]
    world.streams.capturing = True
    assert attend() != kept
    assert world.cache._workspaces == {0: held}
    world.streams.at = SIDE
    attend()
    assert world.cache._workspaces == {0: held}
    world.streams.capturing, world.streams.at = False, 0
    assert attend() == kept
    world.streams.capturing = True  # a workspace that is given is used
    w = gpu(aligned(NEED))
    world.cache.attend(world.q, world.batch, workspace=w)
    assert last(world.log, "attend")[2] == w.data_ptr()


# ------------------------------------------------------------- sizes past 32 bits
@pytest.mark.parametrize("bad", [dict(max_kv=1 << 32), dict(max_kv=1 << 31), dict(max_rows=(1 << 32) + 1), dict(total_rows=1 << 64),
                                 dict(max_kv=-(1 << 32) + 9)], ids=str)
def test_bounds_that_32_bits_do_not_hold_are_refused(bad):
    sizes = {**dict(total_rows=1, max_rows=1, max_kv=9), **bad}
    with pytest.raises(ValueError, match=next(iter(bad))):
        PagedBatch(ints(0, 1).view(1, 2), ints(0, 1), ints(9), **sizes)


@pytest.mark.parametrize("bad", [dict(window=1 << 32), dict(window=(1 << 32) + 5), dict(sinks=1 << 32, window=4), dict(window=1 << 31)], ids=str)
def test_masks_that_32_bits_do_not_hold_are_refused(world, bad):
    with pytest.raises(ValueError, match=next(iter(bad))):
        world.cache.attend(world.q, world.batch, workspace=gpu(aligned(NEED)), **bad)
