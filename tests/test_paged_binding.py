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
