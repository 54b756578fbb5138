"""A paged key/value cache and attention over it, on PyTorch tensors.

A PagedCache holds rows in pages of bf16, or of 8-bit or 4-bit codes with a
step and a minimum for each 64 channels; a PagedBatch says which pages a set of
sequences uses and which of their rows are new. `write` puts new rows into
pages, `read` reads them back, `attend` attends with new rows' queries over
all the rows that their sequences hold. `write_rotated` takes rows as a model's
projections leave them: norms and position rotation (Rotary) on the way.
PageBounds keeps bounds of each page's keys, by which `choose` picks the pages
that a query is to see, and `attend_chosen` attends to those alone.
`copy_pages` and `gather` move pages and rows; sequences.py keeps the books.
Everything runs in libipv.so's kernels
(include/ipv.h, ipv_pages_write and on); this module allocates with PyTorch
and passes pointers. A half of a PingPongCache is a paged cache as it stands:
`PagedCache.of_layer`.
"""
from __future__ import annotations

import ctypes
import struct

import torch

from . import ipv

GROUP = 64  # channels that share a step and a minimum
FORMATS = {"bf16": ipv.IPV_PAGES_BF16, "u8": ipv.IPV_PAGES_U8, "u4": ipv.IPV_PAGES_U4}


# Small calls take as long as the host does, so the ones below check a tensor with few reads of its attributes, spell out what is
# wrong only then (_packed and its like), and write a structure's fields at once. ctypes lays structures out as these do.
_ROTATE = struct.Struct("@4P6qi4x3Pq").pack_into  # but eps
_CHOOSE = struct.Struct("@P2q4iP2q").pack_into
_ATTEND = struct.Struct("@3P4qi").pack_into  # the fields before scale
_LISTS = struct.Struct("@Pi2q").pack_into


def _fields(structure):
    """A ctypes structure's memory, for these."""
    return (ctypes.c_char * ctypes.sizeof(structure)).from_buffer(structure)


def _need(ok: bool, what: str) -> None:
    if not ok:
        raise ValueError(what)


def _fits(bits: int, **values: int) -> None:
    """ctypes cuts what a C integer does not hold."""
    for name, x in values.items():
        _need(-(1 << (bits - 1)) <= x < 1 << (bits - 1), f"{name} {x} does not fit {bits} bits")


class PagedBatch:
    """Sequences and their new rows (ipv_batch).

    table: int32 [n_seqs, max_pages] page numbers, or None (one page per
    sequence, page b for sequence b); a row expanded to n_seqs is one set of
    pages that all sequences read. row_start: int32 [n_seqs + 1], the new
    rows' places in packed tensors. kv_len: int32 [n_seqs], rows held, new ones
    included. The three are read on the GPU when a call runs and may be
    updated in place between calls; total_rows, max_rows and max_kv bound
    them on the host (the packed rows, one sequence's new rows, one sequence's
    rows)."""

    def __init__(self, table, row_start: torch.Tensor, kv_len: torch.Tensor, *, total_rows: int,
                 max_rows: int, max_kv: int):
        for name, t in (("table", table), ("row_start", row_start), ("kv_len", kv_len)):
            if t is not None:
                _need(t.dtype == torch.int32 and t.is_cuda, f"{name} must be an int32 CUDA tensor")
                _need(t.numel() == 0 or t.stride(-1) == 1, f"{name} must be contiguous along its last dimension")
        _need(kv_len.dim() == 1 and row_start.shape == (kv_len.shape[0] + 1,),
              "kv_len is [n_seqs], row_start [n_seqs + 1]")
        n = kv_len.shape[0]
        _need(table is None or (table.dim() == 2 and table.shape[0] == n and table.shape[1] >= 1),
              "table is [n_seqs, max_pages]")
        # 0: an expanded row, all sequences read it. Anything else below a row's length has no meaning; the stride of
        # a table of one row is never used.
        table_stride = 1 if table is None else table.stride(0) if n > 1 else table.shape[1]
        _need(table is None or table_stride == 0 or table_stride >= table.shape[1],
              "the rows of table overlap; table.contiguous() separates them")
        _fits(32, max_rows=max_rows, max_kv=max_kv)
        _fits(64, total_rows=total_rows)
        self.table, self.row_start, self.kv_len = table, row_start, kv_len
        self.n_seqs, self.total_rows, self.max_rows, self.max_kv = n, total_rows, max_rows, max_kv
        self.max_pages = 1 if table is None else table.shape[1]
        self.struct = ipv.Batch(n, self.max_pages, ipv._ptr(table), table_stride, ipv._ptr(row_start),
                                ipv._ptr(kv_len), total_rows, max_rows, max_kv)
        self.ref, self.at = ctypes.byref(self.struct), ctypes.addressof(self.struct)
        self.sizes = (n, self.max_pages, total_rows, max_rows, max_kv)


class Rotary:
    """Position rotation (ipv_rotary). table: fp32 [n_positions, rot_dim], a
    position's rot_dim / 2 cosines and then its sines. Frequency f turns channels
    f and f + rot_dim / 2, or 2f and 2f + 1 if interleaved. sections: how many
    frequencies go by each axis of the positions (multiples of 8); one axis if
    None."""

    def __init__(self, table: torch.Tensor, sections=None, interleaved: bool = False):
        _need(table.dim() == 2 and table.dtype is torch.float32 and table.is_cuda and table.is_contiguous(),
              "table must be a contiguous fp32 CUDA tensor [n_positions, rot_dim]")
        sections = [table.shape[1] // 2] if sections is None else [int(n) for n in sections]
        _need(1 <= len(sections) <= 4, "positions have 1 to 4 axes")
        _fits(32, **{f"section {i}": n for i, n in enumerate(sections)})
        self.table, self.sections, self.axes, self.interleaved = table, sections, len(sections), bool(interleaved)
        self.struct = ipv.RotaryDesc(table.data_ptr(), table.shape[0], table.shape[1], int(self.interleaved), len(sections),
                                     (ctypes.c_int * 4)(*sections))
        self.at = ctypes.addressof(self.struct)

    @classmethod
    def of_base(cls, base: float, n_positions: int, rot_dim: int, sections=None, interleaved: bool = False,
                device="cuda") -> "Rotary":
        """Angles position * base^(-2f / rot_dim), taken in 64 bits."""
        f = torch.arange(rot_dim // 2, dtype=torch.float64, device=device)
        angle = torch.arange(n_positions, dtype=torch.float64, device=device)[:, None] * base ** (-2.0 * f / rot_dim)
        return cls(torch.cat([angle.cos(), angle.sin()], 1).float(), sections, interleaved)


class PageBounds:
    """Bounds of the keys of a pool's pages (ipv_bounds): codes int8 [n_pages,
    n_kv_heads, 2 (lower, upper), 64 or 128], steps fp32 [n_pages, n_kv_heads]. They say
    nothing of a page before `update` has seen it; copy_pages and gather leave them to the next update."""

    def __init__(self, cache: "PagedCache"):
        padded = 64 if cache.head_dim <= 64 else 128
        codes = torch.zeros((cache.n_pages, cache.n_kv_heads, 2, padded), dtype=torch.int8, device=cache.k.device)
        self._set(codes, torch.zeros((cache.n_pages, cache.n_kv_heads), device=cache.k.device), cache.page_size, cache.head_dim)

    @classmethod
    def from_tensors(cls, codes: torch.Tensor, steps: torch.Tensor, page_size: int, head_dim: int) -> "PageBounds":
        """Bounds over contiguous tensors that the caller keeps."""
        self = cls.__new__(cls)
        self._set(codes, steps, page_size, head_dim)
        return self

    def _set(self, codes, steps, page_size, head_dim):
        padded = 64 if head_dim <= 64 else 128
        _need(codes.dim() == 4 and codes.shape[2:] == (2, padded) and codes.dtype is torch.int8 and codes.is_cuda and codes.is_contiguous(),
              f"codes must be a contiguous int8 CUDA tensor [n_pages, n_kv_heads, 2, {padded}]")
        _need(steps.shape == codes.shape[:2] and steps.dtype is torch.float32 and steps.is_cuda and steps.is_contiguous(),
              "steps must be a contiguous fp32 CUDA tensor [n_pages, n_kv_heads]")
        _fits(32, page_size=page_size, head_dim=head_dim)
        self.codes, self.steps, self.page_size, self.head_dim = codes, steps, page_size, head_dim
        self.n_pages, self.n_kv_heads = codes.shape[:2]
        self.struct = ipv.BoundsDesc(self.n_kv_heads, head_dim, page_size, self.n_pages, codes.data_ptr(), steps.data_ptr())
        self.at, self._lib = ctypes.addressof(self.struct), ipv.load()
        self._args = ipv.ChooseArgs()
        self._args_at, self._args_fields = ctypes.addressof(self._args), _fields(self._args)

    def update(self, cache: "PagedCache", batch: PagedBatch, stream=None) -> None:
        """ipv_bounds_update: the bounds of the pages that hold the batch's new rows, after these were written."""
        status = self._lib.ipv_bounds_update(self.at, cache.at, batch.at, ipv._stream(stream))
        if status:
            ipv._check(status)

    def choose(self, q, batch: PagedBatch, n_chosen: int, *, first: int = 1, recent: int = 1, out=None, stream=None):
        """ipv_bounds_choose: for each new row and KV head the n_chosen pages of its sequence (columns of the table)
        that attend_chosen is to read: the first `first`, the last `recent` and those whose bounds promise the largest
        products with q, bf16 [total_rows, n_q_heads, head_dim]. int32 [total_rows, n_kv_heads, n_chosen], ascending,
        then -1; allocated if out is None, with -1 where a row belongs to no sequence. One host thread at a time
        uses the object."""
        shape, qs = q.shape, q.stride()
        if (len(shape) != 3 or shape[0] < batch.total_rows or shape[2] != self.head_dim or q.dtype is not torch.bfloat16 or not q.is_cuda or
                qs[2] != 1):
            PagedCache._packed("q", q, batch, shape[1] if len(shape) == 3 else 0, self.head_dim)
        if not (0 < n_chosen < 1 << 31 and 0 <= first < 1 << 31 and 0 < recent < 1 << 31):
            raise ValueError(f"n_chosen {n_chosen}, first {first}, recent {recent}: n_chosen and recent must be positive, first at least 0, "
                             "and fit 32 bits")
        at = ipv._stream(stream)
        if out is None:
            out, = PagedCache._results(q, [(batch.total_rows, self.n_kv_heads, n_chosen)], stream, at, torch.int32, -1)
        os = _lists("out", out, batch, self.n_kv_heads, n_chosen)
        _CHOOSE(self._args_fields, 0, q.data_ptr(), qs[0], qs[1], shape[1], n_chosen, first, recent, out.data_ptr(), os[0], os[1])
        status = self._lib.ipv_bounds_choose(self.at, batch.at, self._args_at, at)
        if status:
            ipv._check(status)
        return out


def _lists(name, t, batch, heads, n=None):
    """Strides of int32 [total_rows, heads, n] lists."""
    shape, strides = t.shape, t.stride()
    if (len(shape) != 3 or shape[0] < batch.total_rows or shape[1] != heads or (n is not None and shape[2] != n) or
            (strides[2] != 1 and shape[2] > 1) or t.dtype is not torch.int32 or not t.is_cuda):
        raise ValueError(f"{name} must be an int32 CUDA tensor [{batch.total_rows}, {heads}, {'n' if n is None else n}], contiguous "
                         "along its last dimension")
    return strides


class PagedCache:
    """A pool of pages (ipv_pages): k, v [n_pages, n_kv_heads, page_size,
    head_dim] bf16, or codes uint8 [..., head_dim (u8) or head_dim / 2 (u4)]
    with k_par, v_par fp16 [n_pages, n_kv_heads, page_size, head_dim / 64, 2]
    (step, minimum)."""

    def __init__(self, n_pages: int, page_size: int, n_kv_heads: int, head_dim: int, fmt: str = "bf16",
                 device="cuda"):
        _need(fmt in FORMATS, f"fmt is one of {sorted(FORMATS)}")
        shape = (n_pages, n_kv_heads, page_size)
        if fmt == "bf16":
            k = torch.zeros(shape + (head_dim,), dtype=torch.bfloat16, device=device)
            self._set(fmt, k, torch.zeros_like(k), None, None)
        else:
            _need(head_dim % GROUP == 0, "codes need head_dim 64 or 128")
            k = torch.zeros(shape + (head_dim // (1 if fmt == "u8" else 2),), dtype=torch.uint8, device=device)
            par = torch.zeros(shape + (head_dim // GROUP, 2), dtype=torch.float16, device=device)
            self._set(fmt, k, torch.zeros_like(k), par, torch.zeros_like(par))

    @classmethod
    def from_tensors(cls, fmt: str, k, v, k_par=None, v_par=None) -> "PagedCache":
        """A pool over tensors that the caller keeps. They may be views (a
        permuted [n_pages, page_size, n_kv_heads, ...] pool, a slice of one) as long
        as a row is contiguous and all strides are whole rows, the same ones in
        every tensor."""
        self = cls.__new__(cls)
        _need(fmt in FORMATS, f"fmt is one of {sorted(FORMATS)}")
        self._set(fmt, k, v, k_par, v_par)
        return self

    @classmethod
    def of_layer(cls, cache, layer: int, n_layers: int, n_kv_heads: int, n_streams: int = 1) -> "PagedCache":
        """One layer of a PingPongCache's live half (bf16), without a copy: page b
        is the layer's rows of stream b (PagedBatch with table=None). Valid
        until the next compression pass flips the cache or writes this half."""
        _need(cache.dtype == "bf16", "attention takes bf16 caches")
        _need(cache.n_slabs == n_streams * n_layers * n_kv_heads and 0 <= layer < n_layers,
              "the cache's slabs are streams x layers x KV heads")
        k, v = (t.view(n_streams, n_layers, n_kv_heads, cache.capacity, cache.head_dim)[:, layer]
                for t in (cache.k_live, cache.v_live))
        return cls.from_tensors("bf16", k, v)

    def _set(self, fmt, k, v, k_par, v_par):
        codes = fmt != "bf16"
        want = torch.uint8 if codes else torch.bfloat16
        for name, t in (("k", k), ("v", v)):
            _need(t.dim() == 4 and t.dtype == want and t.is_cuda, f"{name} must be a 4-d {want} CUDA tensor")
        _need(k.shape == v.shape, "k and v must have one shape")
        width = k.shape[3]
        self.fmt, self.k, self.v, self.k_par, self.v_par = fmt, k, v, k_par, v_par
        self.n_pages, self.n_kv_heads, self.page_size = k.shape[0], k.shape[1], k.shape[2]
        self.head_dim = width * (2 if fmt == "u4" else 1)
        rows = self._row_strides(k, width)
        _need(self._row_strides(v, width) == rows, "k and v must have the same strides")
        if codes:
            groups = self.head_dim // GROUP
            for name, t in (("k_par", k_par), ("v_par", v_par)):
                _need(t is not None and t.dtype == torch.float16 and t.is_cuda and
                      t.shape == k.shape[:3] + (groups, 2), f"{name} must be fp16 {tuple(k.shape[:3]) + (groups, 2)}")
                _need(t.stride(4) == 1 and t.stride(3) == 2, f"{name}: a row's pairs must be contiguous")
                _need(self._row_strides(t, 2 * groups) == rows, f"{name} must have k's strides, in rows")
        self.struct = ipv.PagesDesc(FORMATS[fmt], self.n_kv_heads, self.head_dim, self.page_size, self.n_pages, *rows,
                                    k.data_ptr(), v.data_ptr(), ipv._ptr(k_par), ipv._ptr(v_par))
        self.ref, self.at = ctypes.byref(self.struct), ctypes.addressof(self.struct)
        self._workspaces, self._calls, self._lib = {}, {}, ipv.load()
        self._rotate_args = ipv.RotateArgs()
        self._rotate_at, self._rotate_fields = ctypes.addressof(self._rotate_args), _fields(self._rotate_args)

    @staticmethod
    def _row_strides(t, width):
        _need(t.dim() == 5 or t.stride(3) == 1, "a row must be contiguous")
        out = []
        for i in range(3):
            s = t.stride(i) if t.shape[i] > 1 else width * (1 if i == 2 else t.shape[2])
            _need(s % width == 0, "strides must be whole rows")
            out.append(s // width)
        return tuple(out)

    @staticmethod
    def _packed(name, t, batch, heads, dim):
        shape, strides = t.shape, t.stride()
        if (t.dtype is not torch.bfloat16 or not t.is_cuda or len(shape) != 3 or strides[2] != 1 or
                shape[0] < batch.total_rows or shape[1] != heads or shape[2] != dim):
            raise ValueError(f"{name} must be a bf16 CUDA tensor [{batch.total_rows}, {heads}, {dim}] with contiguous rows")
        return strides

    def _alike(self, k, v, batch):
        """The strides of K's and V's rows where they are just what most calls give; None: _pair is to look closer."""
        shape, strides, bf16 = k.shape, k.stride(), torch.bfloat16
        if (shape == (batch.total_rows, self.n_kv_heads, self.head_dim) and v.shape == shape and strides[2] == 1 and v.stride() == strides and
                k.dtype is bf16 and v.dtype is bf16 and k.is_cuda and v.is_cuda):
            return strides
        return None

    def _pair(self, k_name, k, v_name, v, batch):
        strides = self._packed(k_name, k, batch, self.n_kv_heads, self.head_dim)
        if v.shape != k.shape or v.dtype is not torch.bfloat16 or not v.is_cuda:
            self._packed(v_name, v, batch, self.n_kv_heads, self.head_dim)
        if v.stride() != strides:
            raise ValueError(f"{k_name} and {v_name} must have the same strides")
        return strides

    @staticmethod
    def _results(like, shapes, stream, at, dtype=torch.bfloat16, fill=0):
        """New tensors, filled (zeroed), for a call on stream `at`. Made on that stream: the fill comes before the kernel, and
        the memory belongs to it; the current stream may use them as well."""
        make = lambda shape: like.new_full(shape, fill, dtype=dtype) if fill else like.new_zeros(shape, dtype=dtype)  # noqa: E731
        if stream is None or at == ipv._stream(None):
            return [make(shape) for shape in shapes]
        here = torch.cuda.current_stream()
        with torch.cuda.stream(torch.cuda.ExternalStream(at)):
            out = [make(shape) for shape in shapes]
        for t in out:
            t.record_stream(here)
        return out

    def write(self, k_new, v_new, batch: PagedBatch, stream=None) -> None:
        """ipv_pages_write: k_new, v_new bf16 [total_rows, n_kv_heads, head_dim] into the batch's pages."""
        strides = self._alike(k_new, v_new, batch) or self._pair("k_new", k_new, "v_new", v_new, batch)
        status = self._lib.ipv_pages_write(self.at, batch.at, k_new.data_ptr(), v_new.data_ptr(), strides[0], strides[1],
                                           ipv._stream(stream))
        if status:
            ipv._check(status)

    def read(self, batch: PagedBatch, k_out=None, v_out=None, stream=None):
        """ipv_pages_read: the batch's new rows, bf16 [total_rows, n_kv_heads, head_dim] each. Packed rows that
        belong to no sequence are left as they are (new tensors: zero). New tensors belong to the call's stream."""
        at = ipv._stream(stream)
        if k_out is None or v_out is None:
            shape = (batch.total_rows, self.n_kv_heads, self.head_dim)
            new = self._results(self.k, [shape] * ((k_out is None) + (v_out is None)), stream, at)
            k_out = new.pop(0) if k_out is None else k_out
            v_out = new.pop(0) if v_out is None else v_out
        strides = self._alike(k_out, v_out, batch) or self._pair("k_out", k_out, "v_out", v_out, batch)
        status = self._lib.ipv_pages_read(self.at, batch.at, k_out.data_ptr(), v_out.data_ptr(), strides[0], strides[1], at)
        if status:
            ipv._check(status)
        return k_out, v_out

    def attend(self, q, batch: PagedBatch, *, out=None, lse=None, scale: float | None = None, causal: bool = True,
               window: int = 0, sinks: int = 0, workspace=None, stream=None):
        """ipv_attend: attention of q, bf16 [total_rows, n_q_heads, head_dim], over the rows that the batch's
        sequences hold. out: bf16 like q (allocated if None, on the call's stream); lse: fp32
        [total_rows, n_q_heads], filled if given. workspace: a contiguous uint8 tensor
        that no call on another stream uses at the same time; without one the cache keeps one of its own for
        each stream that is current in a call. ipv.attend_workspace tells its size; many rows over codes (above 64
        per sequence and KV head) need 4 * n_seqs * n_kv_heads * max_kv * head_dim bytes for the widened codes, which
        the layers' caches of a model share if they are given one tensor. A call that torch.cuda.graph captures takes its workspace from the
        graph's memory; if one is given, it has to live as long as the graph, and graphs that share it may not be
        replayed at the same time. One host thread at a time uses a cache object."""
        n_q_heads = q.shape[1]
        qs = self._packed("q", q, batch, n_q_heads, self.head_dim)
        at = ipv._stream(stream)
        if out is None:
            out, = self._results(q, [q.shape], stream, at)
        os = self._packed("out", out, batch, n_q_heads, self.head_dim)
        if lse is not None:
            self._check_lse(lse, batch, n_q_heads)
        # Arguments and workspace need are kept for each set of sizes that they depend on.
        sizes = (batch.sizes, n_q_heads, causal, window, sinks)
        kept = self._calls.get(sizes)
        if kept is None:
            kept = self._first_call(batch, sizes)
        args, ref, need = kept
        args.q, args.out, args.lse = q.data_ptr(), out.data_ptr(), None if lse is None else lse.data_ptr()
        args.q_row_stride, args.q_head_stride, args.out_row_stride, args.out_head_stride = qs[0], qs[1], os[0], os[1]
        args.scale = self.head_dim ** -0.5 if scale is None else scale
        if need:
            self._give_workspace(args, need, workspace, stream, at, q.device)
        status = self._lib.ipv_attend(self.ref, batch.ref, ref, at)
        if status:
            ipv._check(status)
        return out

    def _give_workspace(self, args, need, workspace, stream, at, device):
        if workspace is None:
            _need(stream is None or at == ipv._stream(None), "a stream that is not the current one needs a workspace")
            if torch.cuda.is_current_stream_capturing():
                # From the graph's own memory, which lives as long as the graph: a kept one would be shared with
                # other graphs and calls, and freed when a later call needs a larger one.
                workspace = torch.empty(need, dtype=torch.uint8, device=device)
            else:
                workspace = self._workspaces.get(at)
                if workspace is None or workspace.numel() < need:
                    workspace = self._workspaces[at] = torch.empty(need, dtype=torch.uint8, device=device)
        elif not (workspace.is_cuda and workspace.dtype is torch.uint8 and workspace.is_contiguous()):
            raise ValueError("workspace must be a contiguous uint8 CUDA tensor")
        args.workspace, args.workspace_bytes = workspace.data_ptr(), workspace.numel()

    def attend_chosen(self, q, batch: PagedBatch, chosen, *, out=None, lse=None, scale: float | None = None, workspace=None, stream=None):
        """ipv_attend_chosen: attention of each new row over the rows that it sees of its own pages alone. chosen:
        int32 [total_rows, n_kv_heads, n], columns of the batch's table, as PageBounds.choose gives them (a list
        shorter than the row's pages; entries that are none of them, -1 say, are skipped). q, out, lse, workspace and
        captured calls as in attend."""
        shape, qs = q.shape, q.stride()
        n_q_heads = shape[1] if len(shape) == 3 else 0
        if not n_q_heads or shape[0] < batch.total_rows or shape[2] != self.head_dim or q.dtype is not torch.bfloat16 or not q.is_cuda or qs[2] != 1:
            self._packed("q", q, batch, n_q_heads, self.head_dim)
        cs, n_chosen = _lists("chosen", chosen, batch, self.n_kv_heads), chosen.shape[2]
        at = ipv._stream(stream)
        if out is None:
            out, = self._results(q, [shape], stream, at)
        os = out.stride()
        if out.shape != shape or out.dtype is not torch.bfloat16 or not out.is_cuda or os[2] != 1:
            self._packed("out", out, batch, n_q_heads, self.head_dim)  # may be longer
        if lse is not None and (lse.shape != shape[:2] or lse.dtype is not torch.float32 or not lse.is_cuda or not lse.is_contiguous()):
            self._check_lse(lse, batch, n_q_heads)  # may be longer
        sizes = (batch.sizes, n_q_heads, n_chosen)
        kept = self._calls.get(sizes)
        if kept is None:
            _fits(32, n_chosen=n_chosen)
            args = ipv.AttendArgs(n_q_heads=n_q_heads, scale=1.0, causal=1)
            lists = ipv.Chosen(n_chosen=n_chosen)
            need = ipv.attend_chosen_workspace(self.ref, batch.ref, args, lists)
            kept = args, ctypes.addressof(args), _fields(args), lists, ctypes.addressof(lists), _fields(lists), need
            self._keep_call(sizes, kept)
        args, args_at, args_fields, _, lists_at, lists_fields, need = kept
        _ATTEND(args_fields, 0, q.data_ptr(), out.data_ptr(), 0 if lse is None else lse.data_ptr(), qs[0], qs[1], os[0], os[1], n_q_heads)
        args.scale = self.head_dim ** -0.5 if scale is None else scale
        _LISTS(lists_fields, 0, chosen.data_ptr(), n_chosen, cs[0], cs[1])
        if need:
            self._give_workspace(args, need, workspace, stream, at, q.device)
        status = self._lib.ipv_attend_chosen(self.at, batch.at, args_at, lists_at, at)
        if status:
            ipv._check(status)
        return out

    @staticmethod
    def _check_lse(lse, batch, n_q_heads):
        _need(lse.dtype is torch.float32 and lse.is_cuda and lse.is_contiguous() and lse.dim() == 2 and
              lse.shape[0] >= batch.total_rows and lse.shape[1] == n_q_heads,
              "lse must be a contiguous fp32 CUDA tensor [total_rows, n_q_heads]")

    def _check_weight(self, name, w):
        if w.dtype is not torch.bfloat16 or not w.is_cuda or w.shape != (self.head_dim,) or not w.is_contiguous():
            raise ValueError(f"{name} must be a contiguous bf16 CUDA tensor [{self.head_dim}]")

    def write_rotated(self, q, k_new, v_new, batch: PagedBatch, rotary: Rotary, positions, *, q_weight=None, k_weight=None,
                      eps: float = 1e-6, q_out=None, stream=None):
        """ipv_pages_write_rotated: k_new (normalised with k_weight if given, rotated) and v_new into the batch's pages,
        and q, bf16 [total_rows, n_q_heads, head_dim], normalised with q_weight if given and rotated, into q_out
        (allocated if None, on the call's stream; q itself will do), which is returned. positions: int32
        [total_rows] or [axes, total_rows] (one row expanded to all axes will do), places in the rotary's table: a row's place
        in the stream, which a compacted cache does not tell. weights: bf16 [head_dim]. One host thread at a time uses a cache object."""
        rows, dim, bf16 = batch.total_rows, self.head_dim, torch.bfloat16
        shape, qs = q.shape, q.stride()
        n_q_heads = shape[1] if len(shape) == 3 else 0
        if not n_q_heads or shape[0] < rows or shape[2] != dim or q.dtype is not bf16 or not q.is_cuda or qs[2] != 1:
            self._packed("q", q, batch, n_q_heads, dim)
        strides = self._alike(k_new, v_new, batch) or self._pair("k_new", k_new, "v_new", v_new, batch)
        at_shape, at_strides, axes = positions.shape, positions.stride(), rotary.axes
        if len(at_shape) == 1 and axes == 1:
            at_shape, at_strides = (1, at_shape[0]), (at_shape[0], at_strides[0])
        if (len(at_shape) != 2 or at_shape[0] != axes or at_shape[1] < rows or (at_strides[1] != 1 and at_shape[1] > 1) or
                positions.dtype is not torch.int32 or not positions.is_cuda):
            raise ValueError(f"positions must be an int32 CUDA tensor [{axes}, {rows}], contiguous along its last dimension")
        if q_weight is not None:
            self._check_weight("q_weight", q_weight)
        if k_weight is not None:
            self._check_weight("k_weight", k_weight)
        at = ipv._stream(stream)
        if q_out is None:
            q_out, = self._results(q, [shape], stream, at)
        os = q_out.stride()
        if q_out.shape != shape or q_out.dtype is not bf16 or not q_out.is_cuda or os[2] != 1:
            self._packed("q_out", q_out, batch, n_q_heads, dim)  # may be longer
        _ROTATE(self._rotate_fields, 0, q.data_ptr(), q_out.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), qs[0], qs[1], os[0], os[1],
                strides[0], strides[1], n_q_heads, 0 if q_weight is None else q_weight.data_ptr(),
                0 if k_weight is None else k_weight.data_ptr(), positions.data_ptr(), at_strides[0])
        self._rotate_args.eps = eps
        status = self._lib.ipv_pages_write_rotated(self.at, batch.at, rotary.at, self._rotate_at, at)
        if status:
            ipv._check(status)
        return q_out

    def copy_pages(self, source, target, stream=None) -> None:
        """ipv_pages_copy: page target[i] becomes a copy of page source[i], int32 CUDA tensors [n]. No page is in target
        twice, or in target and at another place in source."""
        n = source.shape
        if (source.dtype is not torch.int32 or target.dtype is not torch.int32 or not source.is_cuda or not target.is_cuda or len(n) != 1 or
                not source.is_contiguous() or not target.is_contiguous()):
            raise ValueError("source and target must be contiguous int32 CUDA tensors [n]")
        if target.shape != n:
            raise ValueError("source and target must have one length")
        status = self._lib.ipv_pages_copy(self.at, source.data_ptr(), target.data_ptr(), n[0], ipv._stream(stream))
        if status:
            ipv._check(status)

    def gather(self, source: "PagedCache", source_batch: PagedBatch, batch: PagedBatch, kept=None, stream=None) -> None:
        """ipv_pages_gather: new row i of sequence b of `batch`, for KV head h, becomes row kept[b, h, i] of sequence b of
        source_batch in the cache `source` (which may be this one), as it is held; row i without kept. kept: int32
        [n_seqs, n_kv_heads, >= max_rows], indices of ipv.select, say. Pages that are written may not be among those that
        are read."""
        kept_strides = (0, 0)
        if kept is not None:
            shape, kept_strides = kept.shape, kept.stride()
            if (len(shape) != 3 or shape[0] < batch.n_seqs or shape[1] != self.n_kv_heads or shape[2] < min(batch.max_rows, batch.total_rows) or
                    (kept_strides[2] != 1 and shape[2] > 1) or kept.dtype is not torch.int32 or not kept.is_cuda):
                raise ValueError("kept must be an int32 CUDA tensor [n_seqs, n_kv_heads, max_rows], contiguous along its last dimension")
        status = self._lib.ipv_pages_gather(source.at, source_batch.at, self.at, batch.at, ipv._ptr(kept), kept_strides[0],
                                            kept_strides[1], ipv._stream(stream))
        if status:
            ipv._check(status)

    def _first_call(self, batch, sizes):
        _, n_q_heads, causal, window, sinks = sizes
        _fits(32, window=window, sinks=sinks)
        args = ipv.AttendArgs(n_q_heads=n_q_heads, scale=1.0, causal=int(causal), window=window, sinks=sinks)
        kept = args, ctypes.byref(args), ipv.attend_workspace(self.ref, batch.ref, args)
        self._keep_call(sizes, kept)
        return kept

    def _keep_call(self, sizes, kept):
        if len(self._calls) >= 1024:
            self._calls.clear()
        self._calls[sizes] = kept
