"""A paged K/V cache: pools of pages on the device, the page table that says
which pages hold a sequence, and the calls that write rows into them, read them
back and attend to them.  `PageTable` hands pages out on the host; `PagedCache`
marshals buffers for ebd_paged_write, ebd_paged_read and ebd_paged_attention of
one layer.  What a sequence caches may grow row by row, and pages of sequences
that have ended serve others.

    table = PagedCache(h, n_pages=4096, sequences=64, max_pages=128, dtype="e4m3")
    table.reserve(3, 700)                       # pages for positions [0, 700) of sequence 3
    table.write(cu_rows, row_pos, k, v)         # rows of new tokens, of any projection's strides
    table.attention(q, cu_rows, kv_len, out, causal=True)
    table.release(3)
"""
from __future__ import annotations

from typing import List, Optional

import numpy as np
import torch

from . import _ebd as E
from . import runtime as rt

DTYPES = {"bf16": E.EBD_KV_BF16, "e4m3": E.EBD_KV_E4M3}


class OutOfPages(RuntimeError):
    """The pools hold no page more; nothing was reserved."""


class PageTable:
    """Pages of `sequences` sequences, at most `max_pages` each, out of `n_pages`.
    Pages given back are handed out again last in, first out."""

    def __init__(self, n_pages: int, sequences: int, max_pages: int, page_size: int):
        if min(n_pages, sequences, max_pages) < 1:
            raise ValueError("n_pages, sequences and max_pages must be positive")
        if page_size < 16 or page_size > 256 or page_size & (page_size - 1):
            raise ValueError("page_size must be a power of two from 16 to 256")
        self.n_pages, self.page_size = n_pages, page_size
        self.table = np.full((sequences, max_pages), -1, np.int32)
        self.held = np.zeros(sequences, np.int64)  # pages of each sequence
        self._free: List[int] = list(range(n_pages - 1, -1, -1))

    @property
    def free(self) -> int:
        return len(self._free)

    def reserve(self, seq: int, length: int) -> bool:
        """Pages for positions [0, length) of a sequence; those it has stay.
        Says whether the table changed."""
        self._check(seq, length)
        need = (length + self.page_size - 1) // self.page_size
        have = int(self.held[seq])
        if need > self.table.shape[1]:
            raise ValueError(f"{length} positions are more than {self.table.shape[1]} pages hold")
        if need - have > len(self._free):
            raise OutOfPages(f"{need - have} pages wanted, {len(self._free)} free")
        for i in range(have, need):
            self.table[seq, i] = self._free.pop()
        self.held[seq] = max(have, need)
        return need > have

    def release(self, seq: int, length: int = 0) -> bool:
        """Gives back the pages past position `length`: of the whole sequence,
        or of what a rejected draft cached.  Says whether the table changed."""
        self._check(seq, length)
        keep, have = (length + self.page_size - 1) // self.page_size, int(self.held[seq])
        for i in range(have - 1, keep - 1, -1):
            self._free.append(int(self.table[seq, i]))
            self.table[seq, i] = -1
        self.held[seq] = min(have, keep)
        return keep < have

    def _check(self, seq: int, length: int):
        if not 0 <= seq < self.table.shape[0]:
            raise ValueError(f"no sequence {seq}")
        if length < 0:
            raise ValueError(f"a length of {length}")


def _rows(t: torch.Tensor, what: str, heads: int, dim: int) -> int:
    """Stride between the rows of a [rows][heads][dim] tensor of bf16 values
    (or of their bits), which may be a slice of a wider row."""
    if t.dtype not in (torch.bfloat16, torch.int16) or t.dim() != 3 or t.shape[1:] != (heads, dim):
        raise ValueError(f"{what}: bf16 [rows][{heads}][{dim}] expected, not {t.dtype} {list(t.shape)}")
    if t.shape[0] and (t.stride(2) != 1 or t.stride(1) != dim):
        raise ValueError(f"{what}: a row's heads must be contiguous")
    if t.shape[0] < 2:
        return 0
    if t.stride(0) < heads * dim:  # rows that overlap; a stride of 0 (an expanded row) is dense to the C calls
        raise ValueError(f"{what}: rows must not overlap (stride {t.stride(0)} of rows of {heads * dim})")
    return t.stride(0)


class PagedCache:
    """One layer's pools, and the calls on the first sequences of the table.
    `h`: a handle of ebd_config.paged = 1; its heads are the cache's."""

    def __init__(self, h: rt.Handle, n_pages: int, sequences: int, max_pages: int,
                 page_size: int = 64, dtype: str = "bf16", device="cuda"):
        if dtype not in DTYPES:
            raise ValueError("dtype must be 'bf16' or 'e4m3'")
        c = h.cfg
        self.h, self.dtype, self.page_size = h, dtype, page_size
        self.heads_q, self.heads, self.dim = c.n_heads_q, c.n_heads_kv, c.head_dim
        self.pages = PageTable(n_pages, sequences, max_pages, page_size)
        shape = (n_pages, self.heads, page_size)
        el = torch.uint8 if dtype == "e4m3" else torch.bfloat16
        self.k = torch.zeros(shape + (self.dim,), dtype=el, device=device)
        self.v = torch.zeros_like(self.k)
        self.k_scale = self.v_scale = None
        if dtype == "e4m3":
            self.k_scale = torch.zeros(shape, dtype=torch.uint8, device=device)
            self.v_scale = torch.zeros_like(self.k_scale)
        self.table = torch.from_numpy(self.pages.table.copy()).to(device)
        self._struct = self.struct()

    # ------------------------------------------------------------ pages
    def reserve(self, seq: int, length: int, stream: Optional[torch.cuda.Stream] = None):
        """Pages for positions [0, length); later calls on `stream` see them."""
        if self.pages.reserve(seq, length):
            self._upload(seq, stream)

    def release(self, seq: int, length: int = 0, stream: Optional[torch.cuda.Stream] = None):
        """Gives back the pages past `length`; calls before it on `stream` still use them."""
        if self.pages.release(seq, length):
            self._upload(seq, stream)

    def _upload(self, seq, stream):
        with torch.cuda.stream(stream or torch.cuda.current_stream()):
            self.table[seq].copy_(torch.from_numpy(self.pages.table[seq].copy()))

    def struct(self) -> E.ebd_kv_pages:
        """The cache as the C calls take it."""
        c = E.ebd_kv_pages()
        c.k, c.v, c.page_table = self.k.data_ptr(), self.v.data_ptr(), self.table.data_ptr()
        c.k_scale, c.v_scale = rt.ptr(self.k_scale), rt.ptr(self.v_scale)
        c.dtype, c.page_size = DTYPES[self.dtype], self.page_size
        c.n_pages, c.max_pages = self.pages.n_pages, self.table.shape[1]
        return c

    # ------------------------------------------------------------ calls
    def _call(self, fn, a, stream):
        if a.batch > self.table.shape[0]:
            raise ValueError("more sequences than the table has")
        E.check(fn(self.h.h, self._struct, a, rt.stream_handle(stream)), self.h.h)

    def _here(self, **tensors):
        for what, t in tensors.items():
            if t.device != self.k.device:
                raise ValueError(f"{what} is on {t.device}, the cache on {self.k.device}")

    def _args(self, rows: int, cu_rows: torch.Tensor) -> E.ebd_paged_args:
        _ints(cu_rows, "cu_rows")
        self._here(cu_rows=cu_rows)
        a = E.ebd_paged_args()
        a.batch, a.rows, a.cu_rows = cu_rows.numel() - 1, rows, cu_rows.data_ptr()
        return a

    def _kv(self, cu_rows, row_pos, k, v):
        a = self._args(k.shape[0], cu_rows)
        stride = _rows(k, "k", self.heads, self.dim)
        if _rows(v, "v", self.heads, self.dim) != stride or v.shape != k.shape:
            raise ValueError("k and v must have the same rows and strides")
        if row_pos.numel() != k.shape[0]:
            raise ValueError("row_pos: one position per row")
        _ints(row_pos, "row_pos")
        self._here(row_pos=row_pos, k=k, v=v)
        a.row_pos, a.k, a.v, a.kv_stride = row_pos.data_ptr(), k.data_ptr(), v.data_ptr(), stride
        return a

    def write(self, cu_rows, row_pos, k, v, skip=None, stream=None):
        """Rows k, v [rows][heads][dim] into the pages, those with a non-zero
        byte of `skip` left out.  cu_rows [B + 1], row_pos [rows]: int32."""
        a = self._kv(cu_rows, row_pos, k, v)
        if skip is not None:
            if skip.dtype not in (torch.uint8, torch.bool) or skip.numel() != a.rows or not skip.is_contiguous():
                raise ValueError("skip: one byte per row")
            self._here(skip=skip)
            a.skip = skip.data_ptr()
        self._call(E.ebd_paged_write, a, stream)

    def read(self, cu_rows, row_pos, k, v, stream=None):
        """The rows at row_pos into k and v."""
        self._call(E.ebd_paged_read, self._kv(cu_rows, row_pos, k, v), stream)

    def attention(self, q, cu_rows, kv_len, out, causal=False, scale=0.0, max_new=0, stream=None):
        """out [rows][heads_q][dim] = attention of q's rows over the first
        kv_len [B] positions of their sequences (ebd_paged_attention)."""
        a = self._args(q.shape[0], cu_rows)
        _ints(kv_len, "kv_len")
        if kv_len.numel() != a.batch:
            raise ValueError("kv_len: one length per sequence")
        a.q_stride = _rows(q, "q", self.heads_q, self.dim)
        _rows(out, "out", self.heads_q, self.dim)
        if out.shape != q.shape or not out.is_contiguous():
            raise ValueError("out: contiguous, of q's shape")
        self._here(q=q, kv_len=kv_len, out=out)
        a.q, a.out, a.kv_len = q.data_ptr(), out.data_ptr(), kv_len.data_ptr()
        a.causal, a.scale, a.max_new = int(causal), scale, max_new
        self._call(E.ebd_paged_attention, a, stream)


def _ints(t: torch.Tensor, what: str):
    if t.dtype != torch.int32 or not t.is_contiguous():
        raise ValueError(f"{what}: contiguous int32 expected")
