"""The books of a paged cache's pages: which sequence holds which, and how many hold each.

The host side of PagedCache (paged.py). Sequences forked from one another share
pages; a page that several hold is copied before one of them writes to it, and
one that nobody holds any more is handed out again. The books only say what to
do: the caller enqueues the copies (PagedCache.copy_pages) and the gather of a
compaction (PagedCache.gather). Pages are handed out again at once, which is right
as long as all calls on the pool go to one stream.
"""
from __future__ import annotations

from collections import Counter

import torch

from .paged import PagedBatch


class OutOfPages(RuntimeError):
    """The pool has too few free pages; nothing was changed."""


class Sequences:
    """Sequences over a pool of n_pages pages of page_size rows. A sequence is known by the number that `add` or `fork`
    returned."""

    def __init__(self, n_pages: int, page_size: int):
        if n_pages < 1 or page_size < 1:
            raise ValueError("n_pages and page_size must be positive")
        self.n_pages, self.page_size = n_pages, page_size
        self._free = list(range(n_pages - 1, -1, -1))  # the last one goes first
        self._holders = [0] * n_pages
        self._lent = Counter()  # pages that `replace` returned and `release` has not seen, each as often as it was lent
        self._pages, self._rows = {}, {}
        self._next = 0

    # ------------------------------------------------------------ what is held
    def __len__(self) -> int:
        return len(self._rows)

    def __contains__(self, seq) -> bool:
        return seq in self._rows

    @property
    def free_pages(self) -> int:
        return len(self._free)

    def rows(self, seq: int) -> int:
        """Rows that the sequence holds."""
        self._known(seq)
        return self._rows[seq]

    def pages(self, seq: int) -> list[int]:
        """Its pages, in order."""
        self._known(seq)
        return list(self._pages[seq])

    def holders(self, page: int) -> int:
        return self._holders[page]

    # ------------------------------------------------------------ changes
    def add(self, rows: int = 0) -> int:
        """A new sequence with room for `rows` rows, which the caller writes."""
        self._count(rows)
        pages = self._take(-(-rows // self.page_size))
        return self._new(pages, rows)

    def fork(self, seq: int) -> int:
        """A new sequence that holds the same rows in the same pages."""
        self._known(seq)
        for page in self._pages[seq]:
            self._holders[page] += 1
        return self._new(list(self._pages[seq]), self._rows[seq])

    def extend(self, seq: int, rows: int) -> list[tuple[int, int]]:
        """Room for `rows` more rows. Returns the (page, its copy) pairs to copy before they are written: the last page, if it is
        partly filled and others hold it too."""
        self._known(seq)
        self._count(rows)
        pages, held = self._pages[seq], self._rows[seq]
        last = held // self.page_size
        shared = rows > 0 and held % self.page_size != 0 and self._holders[pages[last]] > 1
        # Every page that `held` rows leave unused is behind the last one (truncate gives them back).
        more = -(-(held + rows) // self.page_size) - len(pages)
        new = self._take(more + shared)
        copies = []
        if shared:
            copies.append((pages[last], new[0]))
            self._drop(pages[last])
            pages[last] = new.pop(0)
        pages += new
        self._rows[seq] = held + rows
        return copies

    def truncate(self, seq: int, rows: int) -> None:
        """The sequence keeps its first `rows` rows."""
        self._known(seq)
        self._count(rows)
        if rows > self._rows[seq]:
            raise ValueError(f"sequence {seq} holds {self._rows[seq]} rows, not {rows}")
        keep = -(-rows // self.page_size)
        for page in self._pages[seq][keep:]:
            self._drop(page)
        del self._pages[seq][keep:]
        self._rows[seq] = rows

    def replace(self, seq: int, rows: int) -> list[int]:
        """New pages for `rows` rows in place of the sequence's own, for a gather to fill. Returns the pages that it held, from which
        the gather reads: they are held until `release` is called with them."""
        self._known(seq)
        self._count(rows)
        new = self._take(-(-rows // self.page_size))
        old, self._pages[seq], self._rows[seq] = self._pages[seq], new, rows
        self._lent.update(old)
        return list(old)

    def release(self, pages) -> None:
        """Gives back pages that `replace` returned, after the calls that read them have been enqueued. Each lending is given back
        once: with any other page nothing is changed."""
        back = Counter(map(int, pages))
        for page, times in back.items():
            if times > self._lent[page]:
                raise ValueError(f"page {page} is lent to nobody, or was given back already")
        self._lent -= back
        for page in back.elements():
            self._drop(page)

    def remove(self, seq: int) -> None:
        """The sequence is over."""
        self._known(seq)
        for page in self._pages.pop(seq):
            self._drop(page)
        del self._rows[seq]

    # ------------------------------------------------------------ for the calls
    def table(self, seqs, max_pages: int | None = None) -> torch.Tensor:
        """int32 [sequences, max_pages] on the host, -1 behind a sequence's pages; as wide as the longest if None."""
        pages = [self.pages(s) for s in seqs]
        longest = max([1] + [len(p) for p in pages])
        wide = longest if max_pages is None else max_pages
        if wide < longest:
            raise ValueError(f"a sequence holds {longest} pages, the table {wide}")
        return torch.tensor([p + [-1] * (wide - len(p)) for p in pages], dtype=torch.int32).reshape(len(pages), wide)

    def batch(self, seqs, new_rows, device="cuda") -> PagedBatch:
        """A PagedBatch of these sequences whose last new_rows[i] rows are new."""
        seqs, new_rows = list(seqs), list(new_rows)
        if len(seqs) != len(new_rows):
            raise ValueError("one number of new rows for each sequence")
        start, lens = [0], []
        for s, n in zip(seqs, new_rows):
            if not 0 <= n <= self.rows(s):
                raise ValueError(f"sequence {s} holds {self.rows(s)} rows, {n} of them new")
            start.append(start[-1] + n)
            lens.append(self.rows(s))
        return PagedBatch(self.table(seqs).to(device), torch.tensor(start, dtype=torch.int32).to(device),
                          torch.tensor(lens, dtype=torch.int32).to(device), total_rows=start[-1], max_rows=max([0] + new_rows),
                          max_kv=max([0] + lens))

    # ------------------------------------------------------------ within
    def _known(self, seq):
        if seq not in self._rows:
            raise KeyError(f"no sequence {seq}")

    @staticmethod
    def _count(rows):
        if rows < 0:
            raise ValueError("rows must not be negative")

    def _new(self, pages, rows):
        seq, self._next = self._next, self._next + 1
        self._pages[seq], self._rows[seq] = pages, rows
        return seq

    def _take(self, n):
        if n > len(self._free):
            raise OutOfPages(f"{n} pages wanted, {len(self._free)} free")
        out = [self._free.pop() for _ in range(n)]
        for page in out:
            self._holders[page] = 1
        return out

    def _drop(self, page):
        self._holders[page] -= 1
        if not self._holders[page]:
            self._free.append(page)
