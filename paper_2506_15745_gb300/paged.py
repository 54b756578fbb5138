"""A paged key/value cache and attention over it, on PyTorch tensors.

A PagedCache holds rows in pages of bf16, or of 8-bit or 4-bit codes with a
step and a minimum for each 64 channels; a PagedBatch says which pages a set of
sequences uses and which of their rows are new. `write` puts new rows into
pages, `read` reads them back, `attend` attends with new rows' queries over
all the rows that their sequences hold. Everything runs in libipv.so's kernels
(include/ipv.h, ipv_pages_write and on); this module allocates with PyTorch
and passes pointers. A half of a PingPongCache is a paged cache as it stands:
`PagedCache.of_layer`.
"""
from __future__ import annotations

import ctypes

import torch

from . import ipv

GROUP = 64  # channels that share a step and a minimum
FORMATS = {"bf16": ipv.IPV_PAGES_BF16, "u8": ipv.IPV_PAGES_U8, "u4": ipv.IPV_PAGES_U4}


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
        self.ref = ctypes.byref(self.struct)
        self.sizes = (n, self.max_pages, total_rows, max_rows, max_kv)


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
        self.ref = ctypes.byref(self.struct)
        self._workspaces, self._calls, self._lib = {}, {}, ipv.load()

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

    def _pair(self, k_name, k, v_name, v, batch):
        strides = self._packed(k_name, k, batch, self.n_kv_heads, self.head_dim)
        if v.shape != k.shape or v.dtype is not torch.bfloat16 or not v.is_cuda:
            self._packed(v_name, v, batch, self.n_kv_heads, self.head_dim)
        _need(v.stride() == strides, f"{k_name} and {v_name} must have the same strides")
        return strides

    @staticmethod
    def _results(like, shapes, stream, at):
        """New zeroed bf16 tensors for a call on stream `at`. Made on that stream: the fill comes before the kernel, and
        the memory belongs to it; the current stream may use them as well."""
        if stream is None or at == ipv._stream(None):
            return [like.new_zeros(shape, dtype=torch.bfloat16) for shape in shapes]
        here = torch.cuda.current_stream()
        with torch.cuda.stream(torch.cuda.ExternalStream(at)):
            out = [like.new_zeros(shape, dtype=torch.bfloat16) for shape in shapes]
        for t in out:
            t.record_stream(here)
        return out

    def write(self, k_new, v_new, batch: PagedBatch, stream=None) -> None:
        """ipv_pages_write: k_new, v_new bf16 [total_rows, n_kv_heads, head_dim] into the batch's pages."""
        strides = self._pair("k_new", k_new, "v_new", v_new, batch)
        status = self._lib.ipv_pages_write(self.ref, batch.ref, k_new.data_ptr(), v_new.data_ptr(), strides[0], strides[1],
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
        strides = self._pair("k_out", k_out, "v_out", v_out, batch)
        status = self._lib.ipv_pages_read(self.ref, batch.ref, k_out.data_ptr(), v_out.data_ptr(), strides[0], strides[1], at)
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
            _need(lse.dtype is torch.float32 and lse.is_cuda and lse.is_contiguous() and lse.dim() == 2 and
                  lse.shape[0] >= batch.total_rows and lse.shape[1] == n_q_heads,
                  "lse must be a contiguous fp32 CUDA tensor [total_rows, n_q_heads]")
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
            if workspace is None:
                _need(stream is None or at == ipv._stream(None), "a stream that is not the current one needs a workspace")
                if torch.cuda.is_current_stream_capturing():
                    # From the graph's own memory, which lives as long as the graph: a kept one would be shared with
                    # other graphs and calls, and freed when a later call needs a larger one.
                    workspace = torch.empty(need, dtype=torch.uint8, device=q.device)
                else:
                    workspace = self._workspaces.get(at)
                    if workspace is None or workspace.numel() < need:
                        workspace = self._workspaces[at] = torch.empty(need, dtype=torch.uint8, device=q.device)
            elif not (workspace.is_cuda and workspace.dtype is torch.uint8 and workspace.is_contiguous()):
                raise ValueError("workspace must be a contiguous uint8 CUDA tensor")
            args.workspace, args.workspace_bytes = workspace.data_ptr(), workspace.numel()
        status = self._lib.ipv_attend(self.ref, batch.ref, ref, at)
        if status:
            ipv._check(status)
        return out

    def _first_call(self, batch, sizes):
        _, n_q_heads, causal, window, sinks = sizes
        _fits(32, window=window, sinks=sinks)
        args = ipv.AttendArgs(n_q_heads=n_q_heads, scale=1.0, causal=int(causal), window=window, sinks=sinks)
        kept = args, ctypes.byref(args), ipv.attend_workspace(self.ref, batch.ref, args)
        if len(self._calls) >= 1024:
            self._calls.clear()
        self._calls[sizes] = kept
        return kept
